// Attention, forward (gfx950):  S = scale q k^T, masked;  P = softmax(S);  out = P v;  lse = log sum exp S.
//
// One pass over the keys with the running maximum m and sum l of every row.  A workgroup has 4 or 8 wavefronts of 32 rows; a tile of
// keys and values goes through shared memory.  S^T = k q^T has a row's scores in the registers of two lanes, and P^T as it stands is the
// operand of out^T = v^T P^T (sdl_attention.h), so that m, l and the rescaling of the result are a lane's own.
// Where there are too few rows to fill the chip, the keys are cut into chunks for a workgroup each, which leave normalised results and their
// log sums in the workspace, and a second kernel joins them.  Chunks have one size whatever a sequence's length, so that short sequences beside
// long ones leave no one waiting.
//
// In bf16 at width 128 the matrix units are busy for 34 to 45 % of the cycles and the vector units for 38 to 43 % (exponentials, the rounding of P), the two for the
// most part not at once: a workgroup's wavefronts do the same at the same time, and the registers hold two of them on a SIMD.  2 sequences of 4096
// tokens, 16 heads, no mask: 269 us, 1020 TFLOP/s (a library product of 8192^3: 1294); 8192 causal tokens: 275 us, 1000; 4 of 2048: 93 us, 740 (104 on another card), where a
// workgroup's start and end are a sixth of its life.  In fp32 the matrix instructions bound it: 122 to 126 of 155 TFLOP/s without a mask, 107 in 4 causal sequences of 2048.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "sdl_attention.h"

namespace {

using namespace sdl_device;

constexpr int kRowsPerWave = 32, kRows = 4 * kRowsPerWave;      // of a wavefront, of a workgroup of four
constexpr uint32_t kMaxSplits = 256;           // the join has one a thread
constexpr uint32_t kFewRows = 16, kFewLeast = 128, kFewUnits = 256;
template <typename T> constexpr uint32_t kFewTile = sizeof(T) == 2 ? 32 : 16;      // keys of a tile of the kernel for few rows

struct ForwardArgs {
    Attention p;
    float* part_out;        // [split][batch][key head][row][width], with more than one split
    float* part_lse;        // [split][batch][key head][row]
    uint32_t row_blocks, splits, chunk;         // chunk: keys of a split
    uint32_t few;                               // few rows: the splits take turns
    uint32_t pick;                              // splits of no use come last
    uint32_t slots;                             // few rows: workgroups among which all sequences' tiles are shared out, whose results lie one behind the other; or 0
};

// Splits that keys make.
__device__ __forceinline__ uint32_t splits_in_use(const ForwardArgs& a, int32_t keys) { return ((uint32_t)keys + a.chunk - 1) / a.chunk; }

template <typename T, int W, int BN, int WAVES, bool ASYNC>
__global__ void __launch_bounds__(WAVES * kWave, sizeof(T) == 2 ? 2 : 1) sdl_attention_kernel(const ForwardArgs a)
{
    constexpr int kRows = kRowsPerWave * WAVES;
    constexpr int HD = tile_width(W), kTiles = BN / 32, kSteps = W / 16, kOut = W / 32;
    typedef Tile<T, HD> Smem;
    __shared__ __attribute__((aligned(16))) char ks[2][Smem::bytes(BN)];
    __shared__ __attribute__((aligned(16))) char vs[2][Smem::bytes(BN)];
    const Attention& p = a.p;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c = lane & 31, half = lane >> 5;

    uint32_t unit, nth, split;
    if (a.pick) {
        const auto splits = [&](uint32_t u, uint32_t n) {
            return splits_in_use(a, Sequence(p, u / p.kv_heads, 0).most_seen(p, (a.row_blocks - 1 - n) * kRows, kRows));
        };
        if (!pick_item(blockIdx.x, p.batch * p.kv_heads, a.row_blocks, splits, unit, nth, split)) return;
    } else {
        const uint32_t units = p.batch * p.kv_heads, each = a.row_blocks * a.splits;
        if (workgroup() >= units * each) return;
        const Place place(workgroup(), units, each, p.spread);
        unit = place.unit;
        nth = place.within / a.splits;
        split = place.within % a.splits;
    }
    const uint32_t block = a.row_blocks - 1 - nth;          // the longest first
    const Sequence s(p, unit / p.kv_heads, unit % p.kv_heads);

    const uint32_t n_rows = p.queries * p.group.d;
    const uint32_t row = block * kRows + wave * kRowsPerWave + c;
    const uint32_t row_in = min(row, n_rows - 1);
    const int32_t t = (int32_t)div(row_in, p.group);
    const uint32_t head = s.g * p.group.d + (row_in - (uint32_t)t * p.group.d);
    const bool valid = row < n_rows && t < s.nq;

    Frag<T> q[kSteps];
    {
        const T* src = at_row<T>(p.q, s.b, (uint32_t)t, head);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) set_frag(q[k], load_eight<ASYNC>(src, k * 16 + half * 8, valid ? p.width : 0));
    }
    const int32_t sees = valid ? s.seen(p, t) : 0;
    // the workgroup's keys: [first tile, last tile) of this split
    const int32_t t_first = (int32_t)div(min(block * kRows, n_rows - 1), p.group);
    const int32_t t_last = min((int32_t)div(min(block * kRows + kRows, n_rows) - 1, p.group), s.nq - 1);
    const int32_t keys = t_last < t_first ? 0 : s.seen(p, t_last);      // no valid row: nothing to see
    const int32_t every = t_last < t_first ? 0 : s.seen(p, t_first);    // keys that all valid rows see
    const int32_t tiles = (keys + BN - 1) / BN;
    const int32_t tile0 = (int32_t)(split * (a.chunk / BN)), tile1 = min(tiles, tile0 + (int32_t)(a.chunk / BN));
    if (a.splits > 1 && tile0 >= tile1) return;      // a chunk that no row sees is not looked at by the join
    // keys that a row of the wavefront sees: from there on it helps with the copies only
    const int32_t wave_keys = s.most_seen(p, block * kRows + wave * kRowsPerWave, kRowsPerWave);
    const TileCopy<T, HD, BN, WAVES, ASYNC> copy_k(p.k, s.b, s.g, p.width), copy_v(p.v, s.b, s.g, p.width);
#pragma unroll
    for (int i = 0; i < 2; ++i) copy_k.clear(ks[i]), copy_v.clear(vs[i]);

    f32x16_t o[kOut] = {};
    float m = -__builtin_inff(), l = 0.0f;
    if (tile0 < tile1) {
        copy_k.bring(ks[0], tile0 * BN, s.nk);
        copy_v.bring(vs[0], tile0 * BN, s.nk);
    }
    for (int32_t tile = tile0, now = 0; tile < tile1; ++tile, now ^= 1) {
        const int32_t key0 = tile * BN;
        const char *k_now = ks[now], *v_now = vs[now];
        loads_done();               // this tile is there, and all are done with the one before it
        if (tile + 1 < tile1) {
            copy_k.bring(ks[now ^ 1], key0 + BN, s.nk);
            copy_v.bring(vs[now ^ 1], key0 + BN, s.nk);
        }
        if (key0 >= wave_keys) continue;
        f32x16_t sc[kTiles] = {};
        if constexpr (W > 96) __builtin_amdgcn_s_setprio(1);        // the products go ahead of the other wavefront's exponentials: 3 % at width 128
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            if (sizeof(T) == 4 && W <= 96 && k * 16 >= (int)p.width) break;        // eight instructions of 64 cycles each for nothing
#pragma unroll
            for (int n = 0; n < kTiles; ++n) mma(sc[n], Smem::along(k_now, n * 32 + c, 2 * k + half), q[k]);
        }
        if constexpr (W > 96) __builtin_amdgcn_s_setprio(0);
        if (key0 + BN > every) {
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + n * 32 + 8 * (i / 4) + 4 * half + i % 4 >= sees) sc[n][i] = -__builtin_inff();
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[n][i]);
        top = half_max(top) * p.scale_log2;
        if (__any(top > m)) {
            const float now = fmaxf(m, top), by = exp2_fast(m - (now == -__builtin_inff() ? 0.0f : now));
            m = now;
            l *= by;
#pragma unroll
            for (int n = 0; n < kOut; ++n) o[n] *= by;
        }
        const float off = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[n][i] = exp2_fast(__builtin_fmaf(sc[n][i], p.scale_log2, -off));
                l += sc[n][i];
            }
#pragma unroll
        for (int u = 0; u < BN / 16; ++u) {
            const Frag<T> pr = frag_of(sc[u / 2], u % 2, T());
#pragma unroll
            for (int n = 0; n < kOut; ++n) mma(o[n], Smem::across(v_now, u * 16, n * 32, lane), pr);
        }
    }
    l = half_sum(l);
    if (row >= n_rows) return;
    if (sees == 0) {                      // rows that see nothing, in a workgroup whose tiles need no mask for those that do
        l = 0.0f;
#pragma unroll
        for (int n = 0; n < kOut; ++n) o[n] = f32x16_t{};
    }
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    const float lse = l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
    if (a.splits == 1) {
        T* dst = at_row<T>(p.out, s.b, (uint32_t)t, head);
#pragma unroll
        for (int n = 0; n < kOut; ++n)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                store4<ASYNC>(dst, n * 32 + 2 * i + 4 * half, p.width, o[n][i] * by, o[n][i + 1] * by, o[n][i + 2] * by, o[n][i + 3] * by);
        if (p.lse && half == 0) p.lse[((uint64_t)s.b * p.kv_heads * p.group.d + head) * p.queries + t] = lse;
    } else {
        const uint64_t line = (((uint64_t)split * p.batch + s.b) * p.kv_heads + s.g) * n_rows + row;
        float* dst = a.part_out + line * p.width;
#pragma unroll
        for (int n = 0; n < kOut; ++n)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                store4<ASYNC>(dst, n * 32 + 2 * i + 4 * half, p.width, o[n][i] * by, o[n][i + 1] * by, o[n][i + 2] * by, o[n][i + 3] * by);
        if (half == 0) a.part_lse[line] = lse;
    }
}

// Few rows over caches of different lengths: chunks of one size would leave a half of the workgroups without work and compute units with one of them or three.  The lengths
// are in device memory, so every wavefront adds up the tiles for itself: the least number of tiles each with which the workgroups are enough.  16 requests of 1 to
// 8192 tokens, 4 key heads of 128: 36 us with chunks of one size and 30 so, in fp32 77 and 53, 64 requests 106 and 95; 16 of 8192 each 48 and 49.
struct Shares {
    uint32_t n[kFewUnits / kWave];          // workgroups of unit 64 j + lane

    static __device__ __forceinline__ uint32_t sum(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)lane_scan(x), kWave - 1); }
    __device__ __forceinline__ Shares(const ForwardArgs& a, uint32_t tile)
    {
        const Attention& p = a.p;
        const uint32_t lane = threadIdx.x & (kWave - 1), units = p.batch * p.kv_heads;
        uint32_t all = 0, most = 0;
#pragma unroll
        for (uint32_t j = 0; j < kFewUnits / kWave; ++j) {
            const uint32_t u = j * kWave + lane;
            n[j] = u < units ? ((uint32_t)Sequence(p, u / p.kv_heads, 0).most_seen(p, 0, kFewRows) + tile - 1) / tile : 0;
            all += n[j];
            most = max(most, n[j]);
        }
        // no unit has more than the join has threads
        uint32_t each = max(kFewLeast / tile, (sum(all) + a.slots - 1) / a.slots);
        while (__any(most > each * kMaxSplits)) each += max(1u, each / 16);
        for (;; each += max(1u, each / 16)) {            // ends where a workgroup has a whole sequence, if not before: there are as many as units
            uint32_t taken = 0;
#pragma unroll
            for (uint32_t j = 0; j < kFewUnits / kWave; ++j) taken += (n[j] + each - 1) / each;
            if (sum(taken) <= a.slots) break;
        }
#pragma unroll
        for (uint32_t j = 0; j < kFewUnits / kWave; ++j) n[j] = (n[j] + each - 1) / each;
    }
    __device__ __forceinline__ uint32_t mine(uint32_t u) const
    {
        uint32_t x = 0;
#pragma unroll
        for (uint32_t j = 0; j < kFewUnits / kWave; ++j) x |= u / kWave == j ? n[j] : 0;
        return x;
    }
    __device__ __forceinline__ uint32_t of(uint32_t unit) const
    {
        return (uint32_t)__builtin_amdgcn_readlane((int)mine(unit), (int)(unit % kWave));
    }
    __device__ __forceinline__ uint32_t before(uint32_t unit) const
    {
        const uint32_t lane = threadIdx.x & (kWave - 1);
        uint32_t x = 0;
#pragma unroll
        for (uint32_t j = 0; j < kFewUnits / kWave; ++j) x += j * kWave + lane < unit ? n[j] : 0;
        return sum(x);
    }
};

// The same for up to 16 rows, tokens that are generated one by one, where reading the keys and values is all there is to it.  A workgroup is one wavefront
// with tiles of its own, so that nothing waits for anything but its own copies, and the compute unit's other wavefronts (four at width 128) fill in. The rows
// are the columns of the 16x16 instructions.  The splits of a (batch, key head) take turns with the tiles, so that what they read at a time lies side by side.
// 64 requests of 8192 tokens, 16 heads over 4 of width 128 (1.07 GB): 166 us, 6.5 TB/s; 16 of up to 8192 (134 MB): 30 us, 4.5 TB/s, of which the join is 4.
template <typename T, int W, bool ASYNC, bool ONCE>
__global__ void __launch_bounds__(kWave) sdl_attention_few_kernel(const ForwardArgs a)
{
    constexpr int HD = tile_width(W), BN = kFewTile<T>, kTiles = BN / 16, kSteps = W / 32, kOut = W / 16;
    typedef Tile<T, HD> Smem;
    __shared__ __attribute__((aligned(16))) char ks[2][Smem::bytes(BN)];
    __shared__ __attribute__((aligned(16))) char vs[2][Smem::bytes(BN)];
    const Attention& p = a.p;
    const int lane = threadIdx.x, c = lane & 15, quarter = lane >> 4;
    uint32_t unit, nth, split, shares = 0;
    if (a.slots) {
        const Shares of(a, BN);
        if (!pick_item(blockIdx.x, p.batch * p.kv_heads, 1, [&](uint32_t u, uint32_t) { return of.mine(u); }, unit, nth, split)) return;
        shares = of.of(unit);
    } else {
        const uint32_t units = p.batch * p.kv_heads;
        if (workgroup() >= units * a.splits) return;
        const Place place(workgroup(), units, a.splits, p.spread);
        unit = place.unit;
        split = place.within;
    }
    const Sequence s(p, unit / p.kv_heads, unit % p.kv_heads);
    const int32_t keys = s.nq > 0 ? s.seen(p, s.nq - 1) : 0, splits = (int32_t)(a.slots ? shares : splits_in_use(a, keys));
    if (a.splits > 1 && (int32_t)split >= splits) return;       // not looked at by the join
    const TileCopy<T, HD, BN, 1, ASYNC, ONCE> copy_k(p.k, s.b, s.g, p.width), copy_v(p.v, s.b, s.g, p.width);
#pragma unroll
    for (int i = 0; i < 2; ++i) copy_k.clear(ks[i]), copy_v.clear(vs[i]);
    const int32_t key_begin = (int32_t)split * BN, step = splits * BN;
    if (key_begin < keys) {
        copy_k.bring(ks[0], key_begin, s.nk);
        copy_v.bring(vs[0], key_begin, s.nk);
    }

    const uint32_t n_rows = p.queries * p.group.d, row = min((uint32_t)c, n_rows - 1), t = div(row, p.group);
    const uint32_t head = s.g * p.group.d + (row - t * p.group.d);
    const bool valid = (uint32_t)c < n_rows && (int32_t)t < s.nq;
    const int32_t sees = valid ? s.seen(p, (int32_t)t) : 0;
    Frag<T> q[kSteps];
#pragma unroll
    for (int k = 0; k < kSteps; ++k) set_frag(q[k], load_eight<ASYNC>(at_row<T>(p.q, s.b, t, head), k * 32 + quarter * 8, valid ? p.width : 0));

    f32x4_t o[kOut] = {};
    float m = -__builtin_inff(), l = 0.0f;
    for (int32_t key0 = key_begin, now = 0; key0 < keys; key0 += step, now ^= 1) {
        own_loads_done();
        if (key0 + step < keys) {
            copy_k.bring(ks[now ^ 1], key0 + step, s.nk);
            copy_v.bring(vs[now ^ 1], key0 + step, s.nk);
        }
        f32x4_t sc[kTiles] = {};
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int n = 0; n < kTiles; ++n) mma16(sc[n], Smem::along(ks[now], n * 16 + c, 4 * k + quarter), q[k]);
        float top = -__builtin_inff();
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (key0 + n * 16 + 4 * quarter + i >= sees) sc[n][i] = -__builtin_inff();
                top = fmaxf(top, sc[n][i]);
            }
        top = quarter_max(top) * p.scale_log2;
        if (__any(top > m)) {
            const float up = fmaxf(m, top), by = exp2_fast(m - (up == -__builtin_inff() ? 0.0f : up));
            m = up;
            l *= by;
#pragma unroll
            for (int n = 0; n < kOut; ++n) o[n] *= by;
        }
        const float off = m == -__builtin_inff() ? 0.0f : m;
        Frag<T> pr;
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sc[n][i] = exp2_fast(__builtin_fmaf(sc[n][i], p.scale_log2, -off));
                l += sc[n][i];
            }
        if constexpr (sizeof(T) == 2) {
            pr.v = __builtin_bit_cast(bf16x8_t, u32x4{pack_bf16(sc[0][0], sc[0][1]), pack_bf16(sc[0][2], sc[0][3]),
                                                      pack_bf16(sc[kTiles - 1][0], sc[kTiles - 1][1]), pack_bf16(sc[kTiles - 1][2], sc[kTiles - 1][3])});
#pragma unroll
            for (int n = 0; n < kOut; ++n) mma16(o[n], Smem::across16(vs[now], n * 16), pr);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) pr.v[i] = sc[0][i];
#pragma unroll
            for (int n = 0; n < kOut; ++n) mma16(o[n], Smem::across16(vs[now], n * 16), pr, 4);
        }
    }
    l = quarter_sum(l);
    if ((uint32_t)c >= n_rows) return;
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    const float lse = l == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
    if (a.splits == 1) {
        T* dst = at_row<T>(p.out, s.b, t, head);
#pragma unroll
        for (int n = 0; n < kOut; ++n) store4<ASYNC>(dst, n * 16 + 4 * quarter, p.width, o[n][0] * by, o[n][1] * by, o[n][2] * by, o[n][3] * by);
        if (p.lse && quarter == 0) p.lse[((uint64_t)s.b * p.kv_heads * p.group.d + head) * p.queries + t] = lse;
    } else {
        const uint64_t line = (a.slots ? blockIdx.x : (uint64_t)split * p.batch * p.kv_heads + unit) * n_rows + row;
        float* dst = a.part_out + line * p.width;
#pragma unroll
        for (int n = 0; n < kOut; ++n) store4<ASYNC>(dst, n * 16 + 4 * quarter, p.width, o[n][0] * by, o[n][1] * by, o[n][2] * by, o[n][3] * by);
        if (quarter == 0) a.part_lse[line] = lse;
    }
}

// out = sum over splits of exp(lse_s - lse) out_s, lse = log sum exp of the lse_s.  For up to 32 splits of many rows: 32 lanes have a row, a split's weight each, and
// four elements each of the sum.
template <typename T>
__global__ void __launch_bounds__(256) sdl_attention_join_rows_kernel(const ForwardArgs a)
{
    const Attention& p = a.p;
    const uint32_t n_rows = p.queries * p.group.d, lines = p.batch * p.kv_heads * n_rows, lane = threadIdx.x % 32, d = lane * 4;
    const uint32_t line = min(blockIdx.x * 8 + threadIdx.x / 32, lines - 1);        // more than one may do the last
    const uint32_t bg = line / n_rows, row = line - bg * n_rows, t = div(row, p.group);
    const Sequence s(p, bg / p.kv_heads, bg % p.kv_heads);
    const uint32_t last = a.few ? s.nq - 1 : t;        // splits that take turns are all of use to every row
    const uint32_t n = (int32_t)t < s.nq ? splits_in_use(a, s.seen(p, (int32_t)last)) : 0;
    const float mine = lane < n ? a.part_lse[(uint64_t)lane * lines + line] : -__builtin_inff();
    float top = mine;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    const float off = top == -__builtin_inff() ? 0.0f : top, weight = exp2_fast((mine - off) * kLog2e), sum = lane_sum<32>(weight);
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
    const float* src = a.part_out + (uint64_t)line * p.width + d;
    const uint64_t step = (uint64_t)lines * p.width;
    f32x4_t x = {};
#pragma unroll 4
    for (uint32_t i = 0; i < n; ++i) {
        const float w = __shfl(weight, (int)i, 32);
        if (d + 4 <= p.width)
            x += w * *reinterpret_cast<const f32x4_elem*>(src + i * step);
        else
            for (uint32_t j = 0; j < 4; ++j) x[j] += d + j < p.width ? w * src[i * step + j] : 0.0f;
    }
    const uint32_t head = s.g * p.group.d + (row - t * p.group.d);
    if (d < p.width) store4(at_row<T>(p.out, s.b, t, head), d, p.width, x[0] * by, x[1] * by, x[2] * by, x[3] * by);
    if (p.lse && lane == 0)
        p.lse[((uint64_t)s.b * p.kv_heads * p.group.d + head) * p.queries + t] = sum == 0.0f ? -__builtin_inff() : off + __builtin_amdgcn_logf(sum) * kLn2;
}

// The same for few rows, or many splits: a workgroup has one row, its threads hold a split's weight each, then eight groups
// of 32 take turns with the splits, four elements a thread.
template <typename T>
__global__ void __launch_bounds__(256) sdl_attention_join_kernel(const ForwardArgs a)
{
    __shared__ float weights[kMaxSplits], parts[2][4];
    __shared__ f32x4_t sums[8][32];
    const Attention& p = a.p;
    const uint32_t n_rows = p.queries * p.group.d, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint32_t lines = p.batch * p.kv_heads * n_rows, line = blockIdx.x;
    const uint32_t bg = line / n_rows, row = line - bg * n_rows, t = div(row, p.group);
    const Sequence s(p, bg / p.kv_heads, bg % p.kv_heads);
    const uint32_t last = a.few ? s.nq - 1 : t;        // splits that take turns are all of use to every row
    uint32_t n = 0, first = line, next = lines;           // rows of results: the first split's, and from one split to the next
    if (a.slots) {
        const Shares of(a, kFewTile<T>);
        first = of.before(bg) * n_rows + row;
        next = n_rows;
        if ((int32_t)t < s.nq) n = of.of(bg);
    } else if ((int32_t)t < s.nq) {
        n = splits_in_use(a, s.seen(p, (int32_t)last));
    }
    const uint32_t group = threadIdx.x / 32, d = threadIdx.x % 32 * 4;
    const float* src = a.part_out + (uint64_t)first * p.width + d;
    const uint64_t step = (uint64_t)next * p.width;
    const float mine = threadIdx.x < n ? a.part_lse[(uint64_t)threadIdx.x * next + first] : -__builtin_inff();
    float top = mine;
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    if (lane == 0) parts[0][wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(parts[0][0], parts[0][1]), fmaxf(parts[0][2], parts[0][3]));
    const float off = top == -__builtin_inff() ? 0.0f : top, weight = exp2_fast((mine - off) * kLog2e);
    float sum = lane_sum<kWave>(weight);
    if (lane == 0) parts[1][wave] = sum;
    weights[threadIdx.x] = weight;
    __syncthreads();
    sum = (parts[1][0] + parts[1][1]) + (parts[1][2] + parts[1][3]);
    f32x4_t x = {};
    if (d + 4 <= p.width) {
#pragma unroll 4
        for (uint32_t i = group; i < n; i += 8) x += weights[i] * *reinterpret_cast<const f32x4_elem*>(src + i * step);
    } else {
        for (uint32_t i = group; i < n; i += 8)
            for (uint32_t j = 0; j < 4; ++j) x[j] += d + j < p.width ? weights[i] * src[i * step + j] : 0.0f;
    }
    sums[group][threadIdx.x % 32] = x;
    __syncthreads();
    const uint32_t head = s.g * p.group.d + (row - t * p.group.d);
    if (threadIdx.x < 32 && d < p.width) {
#pragma unroll
        for (int i = 1; i < 8; ++i) x += sums[i][threadIdx.x];
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        store4(at_row<T>(p.out, s.b, t, head), d, p.width, x[0] * by, x[1] * by, x[2] * by, x[3] * by);
    }
    if (p.lse && threadIdx.x == 0)
        p.lse[((uint64_t)s.b * p.kv_heads * p.group.d + head) * p.queries + t] = sum == 0.0f ? -__builtin_inff() : off + __builtin_amdgcn_logf(sum) * kLn2;
}

// Keys of a split.  A problem that has fewer workgroups than fill the chip is cut, down to what pays for a workgroup's start and its share of the join:
//   workgroups of four wavefronts   512 are two for every compute unit; cut to 1024 below that, of 256 keys at least (an fp32 tile takes the
//                                   matrix units 16 times as long: 64)
//   few rows, of one wavefront      1024 are what the shared memory holds at width 128, of 128 keys at least: 16 caches of 8192 tokens for 4 heads
//                                   56 / 49 / 50 / 54 us with 512 / 1024 / 2048 / 4096
uint32_t chunk_of(uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads, sdl_dtype_t dtype)
{
    const uint64_t rows = (uint64_t)queries * (heads / kv_heads);
    const bool few = rows <= kFewRows;
    const uint64_t groups = (rows + kRows - 1) / kRows * batch * kv_heads, fill = 1024, enough = few ? 1024 : 512;
    const uint64_t least = few ? kFewLeast : dtype == SDL_DTYPE_BF16 ? 256 : 64;
    uint64_t n = keys;
    if (groups < enough) {
        n = keys * groups / fill;
        if (n < least) n = least;
        if (n < (keys + kMaxSplits - 1) / kMaxSplits) n = (keys + kMaxSplits - 1) / kMaxSplits;
    }
    const uint64_t unit = !few && dtype == SDL_DTYPE_BF16 ? 128 : 64;         // whole tiles
    n = (n + unit - 1) / unit * unit;
    return (uint32_t)(n < unit ? unit : n);
}

// Workgroups among which the tiles of few rows' caches are shared out, where the units are few enough to be counted through by each, and their tiles no more than 32 bits
// hold.  Caches that go into 1024 chunks of the least size are all at work at once as it is.
uint32_t slots_of(uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads)
{
    const uint64_t units = (uint64_t)batch * kv_heads;
    const bool pays = (uint64_t)queries * (heads / kv_heads) <= kFewRows && units <= kFewUnits && units * ((keys + kFewLeast - 1) / kFewLeast) > 1024;
    return pays && units * keys < (1ull << 35) ? 1024u : 0u;
}

uint32_t splits_of(uint32_t chunk, uint32_t keys) { return keys <= chunk ? 1u : (keys + chunk - 1) / chunk; }

// Widths over 64 in bf16: eight wavefronts a workgroup and tiles of 128 keys, half as many waits for one another, where such workgroups are two for every compute unit, or one
// and all alike.  2 sequences of 4096 tokens, 16 heads of 128, no mask: 304 us with four wavefronts and 64 keys, 280 so (one sequence 145 and 135); 8192 causal
// tokens of 16 heads over 4: 292 and 275; 2 causal sequences of 2048, which are 256 workgroups of different lengths: 65 and 66.
bool is_tall(uint32_t batch, uint32_t queries, uint32_t heads, uint32_t kv_heads, uint32_t width, sdl_dtype_t dtype, bool causal, uint32_t splits)
{
    const uint64_t rows = (uint64_t)queries * (heads / kv_heads), groups = (rows + 2 * kRows - 1) / (2 * kRows) * batch * kv_heads;
    return dtype == SDL_DTYPE_BF16 && width > 64 && splits == 1 && rows > kFewRows && groups >= (causal ? 512 : 256);
}

template <typename T>
int join(const ForwardArgs& a, hipStream_t st)
{
    const uint64_t lines = (uint64_t)a.p.batch * a.p.kv_heads * a.p.queries * a.p.group.d;
    // 256 rows of 16 splits 4.6 us with a workgroup a row and 8.6 with 32 lanes, 12,408 rows of 9 splits 18 and 9 us
    if (!a.slots && a.splits <= 32 && lines >= 2048)
        hipLaunchKernelGGL((sdl_attention_join_rows_kernel<T>), dim3((uint32_t)((lines + 7) / 8)), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((sdl_attention_join_kernel<T>), dim3((uint32_t)lines), dim3(256), 0, st, a);
    return launched();
}

template <typename T>
int forward(const ForwardArgs& a, bool tall, hipStream_t st)
{
    const dim3 grid = grid_of(a.slots ? a.slots : a.row_blocks * a.splits * a.p.batch * a.p.kv_heads);
    // keys of a tile, of half as many at widths over 64: 64 KB of shared memory (8 sequences of 1024 tokens, 12 heads of 64: 36 us with 64 keys, 32 with 128)
    constexpr int kTileKeys = sizeof(T) == 2 ? 128 : 64;
    const bool async = async_rows(a.p.k, a.p.width, sizeof(T)) && async_rows(a.p.v, a.p.width, sizeof(T));
    // Keys and values of 128 MB and more go past the caches: two of them are more than the memory-side cache (256 MB) holds, and a decoder has one a block.  Single tokens, 16 heads over 4
    // of 128, through the caches and past them, a dozen caches in turn and the same one over and over: 34 MB 17.4 and 17.1 us, 15.0 and 17.2; 67 MB 21.3 and 20.7, 18.8 and 20.0; 134 MB
    // 35.0 and 31.9, 29.6 and 30.5; 268 MB 58 and 52, 48 and 49.  The valid lengths are in device memory, so it goes by what the caches have room for; half of it valid, 134 MB
    // 24.2 and 23.1, 20.7 and 21.2; 268 MB 35.5 and 33.1, 30.5 and 30.8.
    const bool once = 2 * (uint64_t)a.p.batch * a.p.keys * a.p.kv_heads * a.p.width * sizeof(T) >= (1u << 27);
    if (a.few) {
#define SDL_FEW(W)                                                                                                                    \
    do {                                                                                                                              \
        if (!async) hipLaunchKernelGGL((sdl_attention_few_kernel<T, W, false, false>), grid, dim3(kWave), 0, st, a);                  \
        else if (once) hipLaunchKernelGGL((sdl_attention_few_kernel<T, W, true, true>), grid, dim3(kWave), 0, st, a);                \
        else hipLaunchKernelGGL((sdl_attention_few_kernel<T, W, true, false>), grid, dim3(kWave), 0, st, a);                         \
    } while (0)
        if (a.p.width <= 32) SDL_FEW(32);
        else if (a.p.width <= 64) SDL_FEW(64);
        else if (a.p.width <= 96) SDL_FEW(96);
        else SDL_FEW(128);
#undef SDL_FEW
    } else {
#define SDL_ROWS(W, BN, WAVES)                                                                                                        \
    do {                                                                                                                              \
        if (async) hipLaunchKernelGGL((sdl_attention_kernel<T, W, BN, WAVES, true>), grid, dim3(WAVES * kWave), 0, st, a);            \
        else hipLaunchKernelGGL((sdl_attention_kernel<T, W, BN, WAVES, false>), grid, dim3(WAVES * kWave), 0, st, a);                 \
    } while (0)
        if (a.p.width <= 32) SDL_ROWS(32, kTileKeys, 4);
        else if (a.p.width <= 64) SDL_ROWS(64, kTileKeys, 4);
        else if (sizeof(T) == 2 && tall) {
            if constexpr (sizeof(T) == 2) {
                if (a.p.width <= 96) SDL_ROWS(96, 128, 8);
                else SDL_ROWS(128, 128, 8);
            }
        } else if (a.p.width <= 96) SDL_ROWS(96, kTileKeys / 2, 4);
        else SDL_ROWS(128, kTileKeys / 2, 4);
#undef SDL_ROWS
    }
    const int rc = launched();
    return rc != SDL_OK || a.splits == 1 ? rc : join<T>(a, st);
}

}  // namespace

extern "C" {

size_t sdl_attention_workspace_bytes(uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads, uint32_t width, sdl_dtype_t dtype)
{
    if (!sdl_attention_shape(batch, queries, keys, heads, kv_heads, width, dtype)) return 0;
    const uint32_t n = splits_of(chunk_of(batch, queries, keys, heads, kv_heads, dtype), keys);
    if (n == 1) return 0;
    const size_t lines = (size_t)n * batch * heads * queries, shared = (size_t)slots_of(batch, queries, keys, heads, kv_heads) * (heads / kv_heads) * queries;
    return (lines > shared ? lines : shared) * (width + 1) * sizeof(float);
}

int sdl_attention(const sdl_view_t* q, const sdl_view_t* k, const sdl_view_t* v, uint32_t batch, uint32_t queries, uint32_t keys,
                  uint32_t heads, uint32_t kv_heads, uint32_t width, sdl_dtype_t dtype, float scale, int causal, const int32_t* q_len,
                  const int32_t* k_len, const sdl_view_t* out, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    ForwardArgs a{};
    int rc = sdl_attention_problem(a.p, batch, queries, keys, heads, kv_heads, width, dtype, scale, causal, q_len, k_len);
    if (rc != SDL_OK) return rc;
    if (batch == 0 || queries == 0 || heads == 0) return SDL_OK;
    if ((rc = check_view(q, dtype)) != SDL_OK || (rc = check_output(out, dtype, batch, queries, heads)) != SDL_OK) return rc;
    if (keys && ((rc = check_view(k, dtype)) != SDL_OK || (rc = check_view(v, dtype)) != SDL_OK)) return rc;
    if (!aligned_to(lse, 4) || !aligned_to(workspace, 4)) return SDL_ERR_ALIGNMENT;
    const size_t need = sdl_attention_workspace_bytes(batch, queries, keys, heads, kv_heads, width, dtype);
    if (need && (!workspace || workspace_bytes < need)) return SDL_ERR_INVALID_ARG;
    a.p.q = kernel_view(q);
    if (keys) a.p.k = kernel_view(k), a.p.v = kernel_view(v);
    a.p.out = kernel_view(out);
    a.p.lse = lse;
    a.chunk = chunk_of(batch, queries, keys, heads, kv_heads, dtype);
    a.splits = splits_of(a.chunk, keys);
    a.part_out = static_cast<float*>(workspace);
    if (k_len && a.splits > 1) a.slots = slots_of(batch, queries, keys, heads, kv_heads);
    const uint64_t rows = (uint64_t)queries * a.p.group.d;
    a.part_lse = a.part_out + (a.slots ? a.slots * rows : (size_t)a.splits * batch * heads * queries) * width;
    const bool tall = is_tall(batch, queries, heads, kv_heads, width, dtype, a.p.causal, a.splits);
    a.row_blocks = (uint32_t)((rows + (tall ? 2 : 1) * kRows - 1) / ((tall ? 2 : 1) * kRows));
    a.few = rows <= kFewRows;
    a.pick = !a.few && pick_items(a.p, a.row_blocks, a.splits);
    const uint64_t groups = (uint64_t)a.row_blocks * a.splits * batch * kv_heads;
    if (groups > 0x7fffffffu || (a.splits > 1 && (uint64_t)batch * queries * heads > 0x7fffffffu)) return SDL_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == SDL_DTYPE_BF16 ? forward<__bf16>(a, tall, st) : forward<float>(a, tall, st);
}

}  // extern "C"
