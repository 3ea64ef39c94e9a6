// Embedding lookup and the gradient of its table (gfx950).
//
// Forward: out[t] = scale * table[token[t]], a gather of rows: bound by memory, every element is touched once.  8192 rows of 2048 in bf16 10 us, 7.0 TB/s with the
// tokens' repetitions; eight rows 2.3, a launch.
//
// Backward: d_table[v] = scale * sum of d_out[t] over the places t with token[t] = v.  Every row of the table is written, most of
// them as zeros, and every row of d_out is read once; no atomics, one order of every sum.  What is done:
//   1. sort   chunks of 1024 places are sorted by (token, place) in shared memory; meanwhile other workgroups write zeros
//   2. merge  (more than one chunk) the rank of a place is its rank in its chunk and, by bisection, in the others: up to 32 sorted
//             runs become one, again and again until one is left
//   3. reduce the sorted places are cut into segments of equal length, whatever the tokens are.  A run of one token that lies within a segment is
//             added up and written; one that goes on over an end leaves a line of fp32 sums
//   4. join   adds up the lines of every run that crosses an end, in order
// So a token that is every second one costs what others do.  The zeros are most of the bytes: written beside the sorting, which few
// workgroups do and which waits most of its time, they hide it.  8192 places of 2048 columns, a table of 32000 rows in bf16: 12 us of sorting and clearing, 10 of merging and
// clearing (131 MB in the two: 6.0 TB/s), 12 of reading (34 MB), 8 of joining, 39 in all in arrays that come again, 48 in ones that do not.
#include "sdl_operand.h"

namespace {

using namespace sdl_device;

constexpr uint32_t kNone = 0xffffffffu;     // token of a place that is not in the table: behind all others

struct Tokens {
    const void* at;
    uint32_t wide, vocab;       // 64 bits each; rows of the table
    // the token, or kNone
    __device__ __forceinline__ uint32_t get(uint32_t i) const
    {
        const int64_t t = wide ? static_cast<const int64_t*>(at)[i] : (int64_t) static_cast<const int32_t*>(at)[i];
        return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : kNone;
    }
};

struct Places {
    Div tokens;                 // n = batch * tokens places
    uint32_t n, width;
    View rows;                  // out or d_out
};

template <typename T>
__device__ __forceinline__ T* place_row(const Places& p, uint32_t i)
{
    const uint32_t b = div(i, p.tokens), t = i - b * p.tokens.d;
    return reinterpret_cast<T*>(p.rows.data) + ((int64_t)b * p.rows.batch + (int64_t)t * p.rows.token);
}

struct LookupArgs {
    Places places;
    Tokens tokens;
    const char* table;
    int64_t stride;
    float scale;
};

// Eight columns of a row of W: the last ones of a row come as the eight at its end, whose first ones a neighbour has too (and makes the same of).  A load that takes what is
// there element by element is waited for on the spot.  TINY: rows of less than eight.
template <bool TINY>
__device__ __forceinline__ uint32_t columns(uint32_t at, uint32_t W)
{
    return TINY ? at : min(at, W - 8);
}
template <bool TINY, typename T>
__device__ __forceinline__ Eight<T> load_columns(const T* row, uint32_t at, uint32_t W)
{
    return load8(row, at, TINY ? W : ~0u);
}
template <bool TINY, typename T>
__device__ __forceinline__ void store_columns(T* row, uint32_t at, uint32_t W, const float* v)
{
    store8(row, at, TINY ? W : ~0u, v);
}

// LPR lanes a row, ROWS rows at a time each, so that their loads are under way together.
template <typename P, typename T, int LPR, int ROWS, bool TINY>
__global__ void __launch_bounds__(256) sdl_embedding_kernel(const LookupArgs a)
{
    constexpr uint32_t kTeams = 256 / LPR;
    const uint32_t lane = threadIdx.x % LPR, W = a.places.width;
    const uint32_t first = (workgroup() * kTeams + threadIdx.x / LPR) * ROWS;
    uint32_t v[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) v[r] = first + r < a.places.n ? a.tokens.get(first + r) : kNone;
    for (uint32_t from = lane * 8; from < W; from += LPR * 8) {
        const uint32_t at = columns<TINY>(from, W);
        Eight<P> e[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            e[r] = Eight<P>{};
            if (v[r] != kNone) e[r] = load_columns<TINY>(reinterpret_cast<const P*>(a.table) + (int64_t)v[r] * a.stride, at, W);
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (first + r >= a.places.n) break;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = v[r] == kNone ? 0.0f : e[r].get(j) * a.scale;
            store_columns<TINY>(place_row<T>(a.places, first + r), at, W, x);
        }
    }
}

// ------------------------------------------------------------------------------------------------------ backward

constexpr uint32_t kChunk = 1024;           // places that a workgroup sorts, one a thread (10 bits)
constexpr uint32_t kFan = 32;               // sorted runs that become one
constexpr uint32_t kFill = 1024 * 8;        // elements of a table without gaps that a workgroup clears at a time

struct Table {
    char* data;
    int64_t stride;
    uint32_t vocab, width;
};

// A share of the table's zeros: pieces [lo, hi) of a table without gaps, or rows.
struct Fill {
    Table table;
    uint64_t lo, hi;
    uint32_t dense;
};

template <typename P>
__device__ __forceinline__ void fill(const Fill& f, uint32_t group, uint32_t groups)
{
    const float zero[8] = {};
    if (f.dense) {
        const uint64_t numel = (uint64_t)f.table.vocab * f.table.width;
        for (uint64_t i = f.lo + group; i < f.hi; i += groups) {
            const uint64_t at = i * kFill;
            const uint32_t n = (uint32_t)min((uint64_t)kFill, numel - at);
            if (threadIdx.x * 8 < n) store8(reinterpret_cast<P*>(f.table.data) + at, threadIdx.x * 8, n, zero);
        }
    } else {
        for (uint64_t i = f.lo + group; i < f.hi; i += groups)
            for (uint32_t at = threadIdx.x * 8; at < f.table.width; at += 1024 * 8)
                store8(reinterpret_cast<P*>(f.table.data) + (int64_t)i * f.table.stride, at, f.table.width, zero);
    }
}

struct SortArgs {
    Tokens tokens;
    uint32_t n, chunks;
    uint64_t* keys;             // token << 32 | place
    Fill fill;
};

// x of lane ^ J
template <int J>
__device__ __forceinline__ uint32_t of_lane(uint32_t x)
{
#define SDL_DPP(v, ctrl) (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v), ctrl, 0xf, 0xf, true)
    if constexpr (J == 1) return SDL_DPP(x, 0xb1);
    else if constexpr (J == 2) return SDL_DPP(x, 0x4e);
    else if constexpr (J == 4) return SDL_DPP(SDL_DPP(x, 0x141), 0x1b);      // the other end of eight, and of four
    else if constexpr (J == 8) return SDL_DPP(x, 0x128);                      // half of sixteen around
    else if constexpr (J == 16) {
        const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x, x, false, false));
        return threadIdx.x & 16 ? p[0] : p[1];
    } else {
        static_assert(J == 32, "a lane of the wavefront");
        const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(x, x, false, false));
        return threadIdx.x & 32 ? p[0] : p[1];
    }
#undef SDL_DPP
}

constexpr uint32_t log2_of(uint32_t x) { return x <= 1 ? 0 : 1 + log2_of(x / 2); }

// One exchange of a bitonic sort: places J apart, in runs of S that go up and down in turn.
template <uint32_t S, uint32_t J, typename K>
__device__ __forceinline__ void exchange(K& key, K (*lds)[kChunk])
{
    K other;
    if constexpr (J >= (uint32_t)kWave) {
        // two arrays in turn, so that one barrier is enough: the exchanges of S = 128, 256, .. through shared memory are 1, 2, .., counted from the first
        constexpr uint32_t kStage = log2_of(S) - 7, kNumber = kStage * (kStage + 1) / 2 + log2_of(S / 2) - log2_of(J);
        K* at = lds[kNumber % 2];
        at[threadIdx.x] = key;
        __syncthreads();
        other = at[threadIdx.x ^ J];
    } else if constexpr (sizeof(K) == 4) {
        other = of_lane<(int)J>(key);
    } else {
        other = (uint64_t)of_lane<(int)J>((uint32_t)(key >> 32)) << 32 | of_lane<(int)J>((uint32_t)key);
    }
    const bool least = ((threadIdx.x & J) == 0) == ((threadIdx.x & S) == 0);
    key = (other < key) == least ? other : key;
    if constexpr (J > 1) exchange<S, J / 2>(key, lds);
}

// Bitonic sort of one chunk (K. E. Batcher, Sorting networks and their applications, 1968): keys differ, so that equal tokens keep their order.
template <uint32_t S, typename K>
__device__ __forceinline__ void sort_runs(K& key, uint32_t n, K (*lds)[kChunk])
{
    exchange<S, S / 2>(key, lds);
    if constexpr (S < kChunk)
        if (S < n) sort_runs<2 * S>(key, n, lds);
}

// K: what a key is while it is sorted, 32 bits where the token fits beside the place in the chunk (4551 places 26 us instead of 27, in all).
constexpr uint32_t kMostShort = (1u << 22) - 1;        // rows of a table whose tokens do, and the token of no row then
template <typename P, typename K>
__global__ void __launch_bounds__(1024) sdl_embedding_sort_kernel(const SortArgs a)
{
    __shared__ K lds[2][kChunk];
    if (blockIdx.x >= a.chunks) {
        fill<P>(a.fill, blockIdx.x - a.chunks, gridDim.x - a.chunks);
        return;
    }
    const uint32_t i = blockIdx.x * kChunk + threadIdx.x, n = min(kChunk, a.n - blockIdx.x * kChunk);
    K key = (K)~(K)0;
    if (threadIdx.x < n) {
        const uint32_t v = a.tokens.get(i);
        if constexpr (sizeof(K) == 4) key = min(v, kMostShort) << 10 | threadIdx.x;
        else key = (uint64_t)v << 32 | i;
    }
    sort_runs<2>(key, n, lds);
    if (threadIdx.x >= n) return;
    if constexpr (sizeof(K) == 4) {
        const uint32_t v = key >> 10;
        a.keys[i] = (uint64_t)(v == kMostShort ? kNone : v) << 32 | (blockIdx.x * kChunk + key % kChunk);
    } else {
        a.keys[i] = key;
    }
}

struct MergeArgs {
    const uint64_t* from;
    uint64_t* to;
    uint32_t n, run, groups;    // length of the sorted runs, a power of two; workgroups that merge
    Fill fill;
};

// A place's rank is its place in its run and the number of lesser keys in each of the others, by bisection; four lanes share a place, each with every fourth run.
// Chunks are looked through in shared memory, eight of them at a time: a search in memory waits ten times, for 1 us each.
template <typename P>
__global__ void __launch_bounds__(1024) sdl_embedding_merge_kernel(const MergeArgs a)
{
    constexpr uint32_t kHeld = 8;
    __shared__ uint64_t held[kHeld * kChunk];
    if (blockIdx.x >= a.groups) {
        fill<P>(a.fill, blockIdx.x - a.groups, gridDim.x - a.groups);
        return;
    }
    // a workgroup's places are of one chunk
    const uint32_t share = threadIdx.x % 4, p = blockIdx.x * 256 + threadIdx.x / 4, own = blockIdx.x * 256 / kChunk, first = own / kFan * kFan;
    const uint32_t runs = min((a.n - 1) / kChunk + 1 - first, kFan);
    const uint64_t key = a.from[min(p, a.n - 1)];
    uint32_t rank = share == 0 ? p - own * kChunk : 0;
    for (uint32_t r0 = first; r0 < first + runs; r0 += kHeld) {
        if (r0 > first) __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kHeld; ++i) {
            const uint64_t k = (uint64_t)(r0 + i) * kChunk + threadIdx.x;
            held[i * kChunk + threadIdx.x] = k < a.n ? a.from[k] : ~0ull;
        }
        __syncthreads();
#pragma unroll
        for (uint32_t i = 0; i < kHeld; i += 4) {
            const uint32_t r = r0 + i + share;
            if (r == own || r >= first + runs) continue;
            const uint64_t* run = held + (i + share) * kChunk;
            uint32_t lesser = 0;
#pragma unroll
            for (uint32_t step = kChunk / 2; step; step /= 2) lesser += run[lesser + step - 1] < key ? step : 0;
            rank += lesser + (run[lesser] < key);
        }
    }
    rank += __shfl_xor(rank, 1);
    rank += __shfl_xor(rank, 2);
    if (p < a.n && share == 0) a.to[first * kChunk + rank] = key;
}

// The same for longer runs, in memory: eight searches a lane wait together, and take three keys at a time, which divide what is left by four.
__global__ void __launch_bounds__(1024) sdl_embedding_merge_long_kernel(const MergeArgs a)
{
    const uint32_t share = threadIdx.x % 4;
    const uint32_t p = blockIdx.x * 256 + threadIdx.x / 4, own = blockIdx.x * 256 / a.run, first = own / kFan * kFan;
    const uint32_t runs = min((a.n - 1) / a.run + 1 - first, kFan);
    const uint64_t key = a.from[min(p, a.n - 1)];
    uint32_t rank = share == 0 ? p - own * a.run : 0;
    constexpr int kSearches = 8;
    static_assert(kSearches * 4 == kFan, "all of a group's runs at once");
    uint32_t at[kSearches];         // keys in front of it are lesser ones
#pragma unroll
    for (int i = 0; i < kSearches; ++i) at[i] = (first + i * 4 + share) * a.run;
    // no load waits for a comparison: a last run that is shorter goes on with what counts as more than all
    const auto load = [&](int i, uint32_t offset) { return a.from[min(at[i] + offset, a.n - 1)]; };
    const auto less = [&](int i, uint32_t offset, uint64_t k) { return (uint32_t)(k < key && at[i] + offset < a.n); };
    uint32_t left = a.run;
    for (; left >= 4; left /= 4) {
        uint64_t k[kSearches][3];
#pragma unroll
        for (int i = 0; i < kSearches; ++i)
            if (i * 4u < runs)
#pragma unroll
                for (int q = 0; q < 3; ++q) k[i][q] = load(i, left / 4 * (q + 1) - 1);
#pragma unroll
        for (int i = 0; i < kSearches; ++i)
            if (i * 4u < runs) {
                uint32_t lesser = 0;
#pragma unroll
                for (int q = 0; q < 3; ++q) lesser += less(i, left / 4 * (q + 1) - 1, k[i][q]);
                at[i] += lesser * (left / 4);
            }
    }
#pragma unroll
    for (int i = 0; i < kSearches; ++i) {
        const uint32_t r = first + i * 4 + share;
        if (i * 4u >= runs) break;
        if (left == 2) at[i] += less(i, 0, load(i, 0));
        at[i] += less(i, 0, load(i, 0));
        if (r != own && i * 4 + share < runs) rank += at[i] - r * a.run;
    }
    rank += __shfl_xor(rank, 1);
    rank += __shfl_xor(rank, 2);
    if (p < a.n && share == 0) a.to[first * a.run + rank] = key;
}

struct ReduceArgs {
    Places places;
    Table table;
    const uint64_t* keys;
    float* lines;               // [segments][2][width]: sums of the run that comes in over a segment's start, and of the one that leaves over its end
    Div slices;                 // parts of LPR * 8 columns
    uint32_t segments, length;
    float scale;
};

__device__ __forceinline__ uint32_t token_of(uint64_t key) { return (uint32_t)(key >> 32); }

template <bool TINY, typename P>
__device__ __forceinline__ void write_row(const Table& t, uint32_t v, uint32_t at, float scale, const float* acc)
{
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = acc[j] * scale;
    store_columns<TINY>(reinterpret_cast<P*>(t.data) + (int64_t)v * t.stride, at, t.width, x);
}

// LPR lanes have eight columns each of one segment; eight rows are under way at a time.
template <typename T, typename P, int LPR, bool TINY>
__global__ void __launch_bounds__(256) sdl_embedding_reduce_kernel(const ReduceArgs a)
{
    constexpr uint32_t kTeams = 256 / LPR;
    const uint32_t unit = blockIdx.x * kTeams + threadIdx.x / LPR, seg = div(unit, a.slices);
    const uint32_t lane_at = ((unit - seg * a.slices.d) * LPR + threadIdx.x % LPR) * 8, W = a.table.width, at = columns<TINY>(lane_at, W);
    if (seg >= a.segments || lane_at >= W) return;
    const uint32_t s0 = seg * a.length, s1 = min(s0 + a.length, a.places.n);
    // the keys around the segment with those of its first places: nothing waits for one after the other
    const uint64_t before = s0 > 0 ? a.keys[s0 - 1] : ~0ull, behind = s1 < a.places.n ? a.keys[s1] : ~0ull;
    uint64_t k[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j] = s0 + j < s1 ? a.keys[s0 + j] : ~0ull;
    uint32_t cur = token_of(k[0]);
    if (cur == kNone) return;
    bool open = s0 > 0 && token_of(before) == cur;        // begun in front of this segment
    float acc[8] = {};
    for (uint32_t p = s0; p < s1; p += 8) {
        uint64_t next[8];
        Eight<T> e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            e[j] = Eight<T>{};
            if (token_of(k[j]) != kNone) e[j] = load_columns<TINY>(place_row<const T>(a.places, (uint32_t)k[j]), at, W);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) next[j] = p + 8 + j < s1 ? a.keys[p + 8 + j] : ~0ull;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (p + j >= s1) break;
            const uint32_t v = token_of(k[j]);
            if (v != cur) {
                if (cur != kNone) {
                    if (open)
                        store_columns<TINY>(a.lines + (uint64_t)seg * 2 * W, at, W, acc);
                    else
                        write_row<TINY, P>(a.table, cur, at, a.scale, acc);
                }
                open = false;
                cur = v;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += e[j].get(i);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) k[j] = next[j];
    }
    if (cur == kNone) return;
    const bool on = token_of(behind) == cur;
    if (open || on)
        store_columns<TINY>(a.lines + ((uint64_t)seg * 2 + (open ? 0 : 1)) * W, at, W, acc);
    else
        write_row<TINY, P>(a.table, cur, at, a.scale, acc);
}

// The lines of the runs that leave their first segments: a wavefront a segment, which adds up a few lines in order; of many, all eight of the workgroup a share each, and
// then the shares.  (A workgroup a segment and part of the columns: 17 us for 4000 that have nothing to do.)  With sixteen wavefronts a workgroup 4551 places, a third of
// them of one token, take 26.0 us in all, with eight 24.8, with four 25.1; 16384 of one token 44.0, 44.7 and 52.0.
constexpr uint32_t kJoined = 8, kFew = 8;

template <typename P, bool TINY>
__global__ void __launch_bounds__(kJoined * kWave) sdl_embedding_join_kernel(const ReduceArgs a)
{
    __shared__ f32x4_t sums[kJoined][kWave];
    __shared__ uint32_t many[kJoined], tokens[kJoined];          // lines, where they are many
    const uint32_t group = div(blockIdx.x, a.slices), lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const uint32_t lane_at = ((blockIdx.x - group * a.slices.d) * kWave + lane) * 4, W = a.table.width, seg = group * kJoined + wave;
    const uint32_t at = TINY ? lane_at : min(lane_at, W - 4);
    const auto add = [&](uint32_t s, uint32_t from, uint32_t to) {
        const float* line = a.lines + (uint64_t)s * 2 * W + at;
        f32x4_t acc = {};
        for (uint32_t l = from; l < to; l += 8) {
            f32x4_t e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = f32x4_t{};
                if (l + j < to) {
                    const float* p = line + ((uint64_t)(l + j) * 2 + (l + j == 0)) * W;
                    if constexpr (TINY) {
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i) e[j][i] = at + i < W ? p[i] : 0.0f;
                    } else {
                        const f32x4_elem x = *reinterpret_cast<const f32x4_elem*>(p);
                        e[j] = f32x4_t{x.x, x.y, x.z, x.w};
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) acc += e[j];
        }
        return acc;
    };
    const auto write = [&](uint32_t v, const f32x4_t& x) {
        P* row = reinterpret_cast<P*>(a.table.data) + (int64_t)v * a.table.stride + at;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (!TINY || at + i < W) row[i] = (P)(x[i] * a.scale);
    };
    uint32_t lines = 0, v = kNone;
    if (seg + 1 < a.segments) {
        const uint32_t s0 = seg * a.length, s1 = s0 + a.length;
        const uint64_t before = s0 > 0 ? a.keys[s0 - 1] : ~0ull, last = a.keys[s1 - 1];
        // first tokens of the segments that follow, four a lane: the run goes on through those that have its own
        const auto follow = [&](uint32_t s) { return s < a.segments ? token_of(a.keys[s * a.length]) : kNone; };
        uint32_t other[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) other[i] = follow(seg + 1 + i * kWave + lane);
        v = token_of(last);
        // (all of a segment may be one run from further up)
        if (v != kNone && !(s0 > 0 && token_of(before) == v)) {
            for (lines = 1;;) {                 // this segment's second line, and the others' first ones
                uint32_t more = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) more += (uint32_t)__popcll(__ballot(other[i] == v));
                lines += more;
                if (more < 4u * kWave) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) other[i] = follow(seg + lines + i * kWave + lane);
            }
            if (lines > 1 && lines <= kFew && lane_at < W) write(v, add(seg, 0, lines));
        }
    }
    if (lane == 0) {
        many[wave] = lines > kFew ? lines : 0;
        tokens[wave] = v;
    }
    __syncthreads();
    for (uint32_t k = 0; k < kJoined; ++k) {
        const uint32_t n = many[k];
        if (n == 0) continue;
        const uint32_t each = (n + kJoined - 1) / kJoined, from = min(wave * each, n);
        sums[wave][lane] = lane_at < W ? add(group * kJoined + k, from, min(from + each, n)) : f32x4_t{};
        __syncthreads();
        if (wave == k && lane_at < W) {
            f32x4_t acc = {};
#pragma unroll
            for (uint32_t w = 0; w < kJoined; ++w) acc += sums[w][lane];
            write(tokens[k], acc);
        }
        __syncthreads();
    }
}

// -------------------------------------------------------------------------------------------------------- host

constexpr uint32_t kSlice = kWave * 4;      // columns of a wavefront that joins

// Places of a segment: enough of them that a device has work for all its compute units, and not so many that the join of one token's lines
// takes longer than the reading.  (Twice as long: 1000 places 19.1 us instead of 17.1, 16384 of words 37.3 instead of 34.8, of one token 40.8 instead of 44.9.)
uint32_t segment_length(uint64_t n)
{
    const uint64_t each = (n + 1023) / 1024;
    return each <= 8 ? 8 : (uint32_t)((each + 7) / 8 * 8);
}

struct Space {
    size_t keys, lines, bytes;
    uint32_t length, segments;
};

Space space_of(uint64_t n, uint32_t width)
{
    Space s{};
    s.length = segment_length(n);
    s.segments = (uint32_t)((n + s.length - 1) / s.length);
    s.keys = ((size_t)n * sizeof(uint64_t) + 15) / 16 * 16;
    s.lines = s.segments > 1 ? (size_t)s.segments * 2 * width * sizeof(float) : 0;
    s.bytes = (n > kChunk ? 2 : 1) * s.keys + s.lines;
    return s;
}

int check_shape(uint32_t batch, uint32_t tokens, uint32_t vocab, uint32_t width, sdl_dtype_t dtype, sdl_dtype_t table_dtype, sdl_index_t index)
{
    if (!known(dtype) || !known(table_dtype) || (index != SDL_INDEX_INT32 && index != SDL_INDEX_INT64) || width == 0) return SDL_ERR_INVALID_ARG;
    if (width > SDL_EMBEDDING_MAX_WIDTH || vocab > 0x7fffffffu || (uint64_t)batch * tokens > 0x7fffffffu) return SDL_ERR_UNSUPPORTED;
    return SDL_OK;
}

size_t index_size(sdl_index_t t) { return t == SDL_INDEX_INT64 ? 8 : 4; }
bool finite(float x) { return x - x == 0.0f; }

template <typename P, typename T>
int lookup(const LookupArgs& a, hipStream_t st)
{
    const uint32_t n = a.places.n, W = a.places.width;
    const auto groups = [n](uint32_t rows) { return grid_of(((uint64_t)n + rows - 1) / rows); };
    // a row for a workgroup while they are few: 64 rows of 2048 2.4 us instead of 3.6, 2900 4.7 instead of 5.8, but 6000 9.1 instead of 8.8; where all of its lanes have no column each
    // sooner, of 768 columns 2048 rows 3.0 instead of 3.2, 4096 4.1 instead of 3.8.  Narrow rows with lanes to suit: 65536 of 64 columns 4.1 us instead of 9.9, of 256 11.6 instead of 12.9.
    const bool few = n <= (W >= 2048 ? 4096u : 2048u);
#define SDL_LAUNCH(LPR, ROWS, TINY) hipLaunchKernelGGL((sdl_embedding_kernel<P, T, LPR, ROWS, TINY>), groups(256 / LPR * ROWS), dim3(256), 0, st, a)
    if (W < 8) SDL_LAUNCH(8, 1, true);
    else if (W <= 64) SDL_LAUNCH(8, 1, false);
    else if (W <= 256) SDL_LAUNCH(32, 1, false);
    else if (few) SDL_LAUNCH(256, 1, false);
    else SDL_LAUNCH(64, 2, false);
#undef SDL_LAUNCH
    return launched();
}

// Workgroups that clear while others sort or merge (256 to 4096 take the same time).
constexpr uint32_t kFillGroups = 1024;

template <typename T, typename P>
int gradient(const Places& places, const Tokens& tokens, const Table& table, float scale, char* workspace, hipStream_t st)
{
    const uint32_t n = places.n, chunks = (n + kChunk - 1) / kChunk;
    const Space s = space_of(n, table.width);
    uint64_t *keys = reinterpret_cast<uint64_t*>(workspace), *other = reinterpret_cast<uint64_t*>(workspace + s.keys);
    float* lines = reinterpret_cast<float*>(workspace + (n > kChunk ? 2 : 1) * s.keys);
    const bool dense = table.stride == (int64_t)table.width || table.vocab <= 1;
    const uint64_t pieces = dense ? ((uint64_t)table.vocab * table.width + kFill - 1) / kFill : table.vocab;
    const uint64_t half = chunks > 1 ? pieces / 2 : pieces;
    const auto fillers = [](uint64_t share) { return (uint32_t)(share < kFillGroups ? share : kFillGroups); };
    if (chunks || half) {
        const SortArgs a{tokens, n, chunks, keys, Fill{table, 0, half, dense}};
        const dim3 groups(chunks + fillers(half));
        if (table.vocab <= kMostShort) hipLaunchKernelGGL((sdl_embedding_sort_kernel<P, uint32_t>), groups, dim3(1024), 0, st, a);
        else hipLaunchKernelGGL((sdl_embedding_sort_kernel<P, uint64_t>), groups, dim3(1024), 0, st, a);
        if (launched() != SDL_OK) return SDL_ERR_DEVICE;
    }
    if (n == 0) return SDL_OK;
    for (uint64_t run = kChunk; run < n; run *= kFan) {
        const uint32_t groups = (n + 255) / 256;
        const MergeArgs a{keys, other, n, (uint32_t)run, groups, Fill{table, half, pieces, dense}};
        if (run == kChunk)
            hipLaunchKernelGGL((sdl_embedding_merge_kernel<P>), dim3(groups + fillers(pieces - half)), dim3(1024), 0, st, a);
        else
            hipLaunchKernelGGL(sdl_embedding_merge_long_kernel, dim3(groups), dim3(1024), 0, st, a);
        if (launched() != SDL_OK) return SDL_ERR_DEVICE;
        uint64_t* t = keys;
        keys = other;
        other = t;
    }
    ReduceArgs r{places, table, keys, lines, make_div(1), s.segments, s.length, scale};
    const uint32_t W = table.width;
#define SDL_LAUNCH(LPR, TINY)                                                                                                     \
    do {                                                                                                                          \
        r.slices = make_div((W + LPR * 8 - 1) / (LPR * 8));                                                                       \
        const uint32_t teams = 256 / LPR, units = r.slices.d * s.segments;                                                        \
        hipLaunchKernelGGL((sdl_embedding_reduce_kernel<T, P, LPR, TINY>), dim3((units + teams - 1) / teams), dim3(256), 0, st, r); \
    } while (0)
    // (narrow rows with a wavefront a segment: 16384 of 64 columns 31.4 us instead of 27.2)
    if (W < 8) SDL_LAUNCH(8, true);
    else if (W <= 64) SDL_LAUNCH(8, false);
    else if (W <= 256) SDL_LAUNCH(32, false);
    else SDL_LAUNCH(64, false);
#undef SDL_LAUNCH
    if (launched() != SDL_OK) return SDL_ERR_DEVICE;
    if (s.segments > 1) {
        r.slices = make_div((W + kSlice - 1) / kSlice);
        const dim3 groups(r.slices.d * ((s.segments + kJoined - 1) / kJoined));
        if (W < 8)
            hipLaunchKernelGGL((sdl_embedding_join_kernel<P, true>), groups, dim3(kJoined * kWave), 0, st, r);
        else
            hipLaunchKernelGGL((sdl_embedding_join_kernel<P, false>), groups, dim3(kJoined * kWave), 0, st, r);
    }
    return launched();
}

}  // namespace

extern "C" {

int sdl_embedding(const void* table, int64_t table_stride, uint32_t vocab, uint32_t width, sdl_dtype_t table_dtype, const void* tokens, sdl_index_t index,
                  uint32_t batch, uint32_t tokens_of_batch, float scale, const sdl_view_t* out, sdl_dtype_t dtype, void* stream)
{
    int rc = check_shape(batch, tokens_of_batch, vocab, width, dtype, table_dtype, index);
    if (rc != SDL_OK) return rc;
    if (!finite(scale)) return SDL_ERR_INVALID_ARG;
    if (batch == 0 || tokens_of_batch == 0) return SDL_OK;
    if (!tokens || (vocab && !table)) return SDL_ERR_INVALID_ARG;
    if ((rc = check_output(out, dtype, batch, tokens_of_batch, 1)) != SDL_OK) return rc;
    if (!aligned_to(table, dtype_size(table_dtype)) || !aligned_to(tokens, index_size(index))) return SDL_ERR_ALIGNMENT;
    const LookupArgs a{Places{make_div(tokens_of_batch), batch * tokens_of_batch, width, kernel_view(out)},
                       Tokens{tokens, index == SDL_INDEX_INT64, vocab}, static_cast<const char*>(table), table_stride, scale};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (table_dtype == SDL_DTYPE_BF16) return dtype == SDL_DTYPE_BF16 ? lookup<__bf16, __bf16>(a, st) : lookup<__bf16, float>(a, st);
    return dtype == SDL_DTYPE_BF16 ? lookup<float, __bf16>(a, st) : lookup<float, float>(a, st);
}

size_t sdl_embedding_workspace_bytes(uint64_t places, uint32_t width)
{
    return places == 0 || places > SDL_EMBEDDING_MAX_PLACES || width > SDL_EMBEDDING_MAX_WIDTH ? 0 : space_of(places, width).bytes;
}

int sdl_embedding_backward(const sdl_view_t* d_out, sdl_dtype_t dtype, const void* tokens, sdl_index_t index, uint32_t batch, uint32_t tokens_of_batch,
                           float scale, void* d_table, int64_t table_stride, uint32_t vocab, uint32_t width, sdl_dtype_t table_dtype, void* workspace,
                           size_t workspace_bytes, void* stream)
{
    int rc = check_shape(batch, tokens_of_batch, vocab, width, dtype, table_dtype, index);
    if (rc != SDL_OK) return rc;
    if (!finite(scale)) return SDL_ERR_INVALID_ARG;
    if (vocab == 0) return SDL_OK;
    if (!d_table || (vocab > 1 && table_stride == 0)) return SDL_ERR_INVALID_ARG;
    if (!aligned_to(d_table, dtype_size(table_dtype))) return SDL_ERR_ALIGNMENT;
    if ((uint64_t)batch * tokens_of_batch > SDL_EMBEDDING_MAX_PLACES) return SDL_ERR_UNSUPPORTED;
    const uint32_t n = batch * tokens_of_batch;
    Places places{make_div(tokens_of_batch ? tokens_of_batch : 1), n, width, View{}};
    if (n) {
        if (!tokens || !workspace || workspace_bytes < sdl_embedding_workspace_bytes(n, width)) return SDL_ERR_INVALID_ARG;
        if ((rc = check_view(d_out, dtype)) != SDL_OK) return rc;
        if (!aligned_to(tokens, index_size(index)) || !aligned_to(workspace, 8)) return SDL_ERR_ALIGNMENT;
        places.rows = kernel_view(d_out);
    }
    const Tokens t{tokens, index == SDL_INDEX_INT64, vocab};
    const Table table{static_cast<char*>(d_table), table_stride, vocab, width};
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* w = static_cast<char*>(workspace);
    if (dtype == SDL_DTYPE_BF16)
        return table_dtype == SDL_DTYPE_BF16 ? gradient<__bf16, __bf16>(places, t, table, scale, w, st) : gradient<__bf16, float>(places, t, table, scale, w, st);
    return table_dtype == SDL_DTYPE_BF16 ? gradient<float, __bf16>(places, t, table, scale, w, st) : gradient<float, float>(places, t, table, scale, w, st);
}

}  // extern "C"
