// Attention, forward (gfx950):  S = scale q k^T, masked;  P = softmax(S);  out = P v;  lse = log sum exp S.
//
// One pass over the keys with the running maximum m and sum l of every row.  A workgroup has 4 wavefronts of 32 rows; a tile of
// keys and values goes through shared memory.  S^T = k q^T has a row's scores in the registers of two lanes, and P^T as it stands is the
// operand of out^T = v^T P^T (sdl_attention.h), so that m, l and the rescaling of the result are a lane's own.
// Where there are too few rows to fill the chip, the keys are cut into chunks for a workgroup each, which leave normalised results and their
// log sums in the workspace, and a second kernel joins them.  Chunks have one size whatever a sequence's length, so that short sequences beside
// long ones leave no one waiting.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "sdl_attention.h"

namespace {

using namespace sdl_device;

constexpr int kRowsPerWave = 32, kWaves = 4, kRows = kRowsPerWave * kWaves;
constexpr uint32_t kMaxSplits = kWave;         // the join has one a lane

struct ForwardArgs {
    Attention p;
    float* part_out;        // [split][batch][key head][row][width], with more than one split
    float* part_lse;        // [split][batch][key head][row]
    uint32_t row_blocks, splits, chunk;         // chunk: keys of a split
};

template <typename T, int HD, int BN, bool ASYNC>
__global__ void __launch_bounds__(kWaves * kWave, sizeof(T) == 2 ? 2 : 1) sdl_attention_kernel(const ForwardArgs a)
{
    constexpr int kTiles = BN / 32, kSteps = HD / 16, kOut = HD / 32;
    typedef Tile<T, HD> Smem;
    __shared__ __attribute__((aligned(16))) char ks[2][Smem::bytes(BN)];
    __shared__ __attribute__((aligned(16))) char vs[2][Smem::bytes(BN)];
    const Attention& p = a.p;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c = lane & 31, half = lane >> 5;

    const Place place(blockIdx.x, p.batch * p.kv_heads, a.row_blocks * a.splits);
    const uint32_t split = place.within % a.splits;
    const uint32_t block = a.row_blocks - 1 - place.within / a.splits;      // the longest first
    const Sequence s(p, place.unit / p.kv_heads, place.unit % p.kv_heads);

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
        for (int k = 0; k < kSteps; ++k) set_frag(q[k], load8(src, k * 16 + half * 8, valid ? p.width : 0));
    }
    const int32_t sees = valid ? s.seen(p, t) : 0;
    // the workgroup's keys: [first tile, last tile) of this split
    const int32_t t_first = (int32_t)div(min(block * kRows, n_rows - 1), p.group);
    const int32_t t_last = min((int32_t)div(min(block * kRows + kRows, n_rows) - 1, p.group), s.nq - 1);
    const int32_t keys = t_last < t_first ? 0 : s.seen(p, t_last);      // no valid row: nothing to see
    const int32_t every = t_last < t_first ? 0 : s.seen(p, t_first);    // keys that all valid rows see
    const int32_t tiles = (keys + BN - 1) / BN;
    const int32_t tile0 = (int32_t)(split * (a.chunk / BN)), tile1 = min(tiles, tile0 + (int32_t)(a.chunk / BN));
    if (split > 0 && tile0 >= tile1) return;         // a chunk that no row sees is not looked at by the join
    // whether the wavefront has a row that sees a key of the chunk: the others help with the copies only
    const bool busy = __any(sees > tile0 * BN);

    const TileCopy<T, HD, BN, kWaves, ASYNC> copy_k(p.k, s.b, s.g, p.width), copy_v(p.v, s.b, s.g, p.width);
#pragma unroll
    for (int i = 0; i < 2; ++i) copy_k.clear(ks[i]), copy_v.clear(vs[i]);

    f32x16_t o[kOut] = {};
    float m = -__builtin_inff(), l = 0.0f;
    if (tile0 < tile1) {
        copy_k.bring(ks[0], tile0 * BN, s.nk);
        copy_v.bring(vs[0], tile0 * BN, s.nk);
    }
    auto step = [&](int32_t tile, char* k_now, char* v_now, char* k_next, char* v_next) __attribute__((always_inline)) {
        const int32_t key0 = tile * BN;
        loads_done();               // this tile is there, and all are done with the one before it
        if (tile + 1 < tile1) {
            copy_k.bring(k_next, key0 + BN, s.nk);
            copy_v.bring(v_next, key0 + BN, s.nk);
        }
        if (!busy) return;
        f32x16_t sc[kTiles] = {};
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int n = 0; n < kTiles; ++n) mma(sc[n], Smem::along(k_now, n * 32 + c, 2 * k + half), q[k]);
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
            for (int n = 0; n < kOut; ++n) mma(o[n], Smem::across(v_now, u * 16, n * 32), pr);
        }
    };
    for (int32_t tile = tile0; tile < tile1; tile += 2) {
        step(tile, ks[0], vs[0], ks[1], vs[1]);
        if (tile + 1 < tile1) step(tile + 1, ks[1], vs[1], ks[0], vs[0]);
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
                store4(dst, n * 32 + 2 * i + 4 * half, p.width, o[n][i] * by, o[n][i + 1] * by, o[n][i + 2] * by, o[n][i + 3] * by);
        if (p.lse && half == 0) p.lse[((uint64_t)s.b * p.kv_heads * p.group.d + head) * p.queries + t] = lse;
    } else {
        const uint64_t line = (((uint64_t)split * p.batch + s.b) * p.kv_heads + s.g) * n_rows + row;
        float* dst = a.part_out + line * p.width;
#pragma unroll
        for (int n = 0; n < kOut; ++n)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                store4(dst, n * 32 + 2 * i + 4 * half, p.width, o[n][i] * by, o[n][i + 1] * by, o[n][i + 2] * by, o[n][i + 3] * by);
        if (half == 0) a.part_lse[line] = lse;
    }
}

// out = sum over splits of exp(lse_s - lse) out_s, lse = log sum exp of the lse_s: one wavefront a row, two elements a lane, and the weight
// of split s in lane s.
template <typename T>
__global__ void __launch_bounds__(256) sdl_attention_join_kernel(const ForwardArgs a)
{
    const Attention& p = a.p;
    const uint32_t n_rows = p.queries * p.group.d, lane = threadIdx.x & (kWave - 1);
    const uint32_t lines = p.batch * p.kv_heads * n_rows;
    const uint32_t line = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave);
    if (line >= lines) return;
    const uint32_t bg = line / n_rows, row = line - bg * n_rows, t = div(row, p.group);
    const Sequence s(p, bg / p.kv_heads, bg % p.kv_heads);
    const uint32_t head = s.g * p.group.d + (row - t * p.group.d);
    const uint32_t sees = (int32_t)t < s.nq ? (uint32_t)s.seen(p, (int32_t)t) : 0;
    const uint32_t n = (sees + a.chunk - 1) / a.chunk;
    const float mine = lane < n ? a.part_lse[(uint64_t)lane * lines + line] : -__builtin_inff();
    float top = mine;
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    const float off = top == -__builtin_inff() ? 0.0f : top;
    const float weight = exp2_fast((mine - off) * kLog2e), sum = lane_sum<kWave>(weight);
    const float scaled = sum == 0.0f ? 0.0f : weight / sum;
    float x = 0.0f, y = 0.0f;
    const uint32_t d = 2 * lane;
    const float* src = a.part_out + (uint64_t)line * p.width;
#pragma unroll 8
    for (uint32_t i = 0; i < n; ++i) {
        const float by = u2f(__builtin_amdgcn_readlane(f2u(scaled), i));
        const float* from = src + (uint64_t)i * lines * p.width;
        if (d < p.width) x = __builtin_fmaf(by, from[d], x);
        if (d + 1 < p.width) y = __builtin_fmaf(by, from[d + 1], y);
    }
    T* dst = at_row<T>(p.out, s.b, t, head);
    if (d < p.width) dst[d] = (T)x;
    if (d + 1 < p.width) dst[d + 1] = (T)y;
    if (p.lse && lane == 0)
        p.lse[((uint64_t)s.b * p.kv_heads * p.group.d + head) * p.queries + t] = sum == 0.0f ? -__builtin_inff() : off + __builtin_amdgcn_logf(sum) * kLn2;
}

// Keys of a chunk: as few as make about `kFill` workgroups of a problem that has fewer, and no fewer than pay for a workgroup's start and its
// share of the join (256; an fp32 tile takes the matrix units 16 times as long: 64).
constexpr uint32_t kFill = 1024;

uint32_t chunk_of(uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads, sdl_dtype_t dtype)
{
    const uint64_t rows = (uint64_t)queries * (heads / kv_heads);
    const uint64_t groups = (rows + kRows - 1) / kRows * batch * kv_heads, least = dtype == SDL_DTYPE_BF16 ? 256 : 64;
    uint64_t n = keys;
    if (groups < kFill / 2) {
        n = keys * groups / kFill;
        if (n < least) n = least;
        if (n < (keys + kMaxSplits - 1) / kMaxSplits) n = (keys + kMaxSplits - 1) / kMaxSplits;
    }
    n = (n + 63) / 64 * 64;           // whole tiles
    return n < 64 ? 64u : (uint32_t)n;
}

uint32_t splits_of(uint32_t chunk, uint32_t keys) { return keys <= chunk ? 1u : (keys + chunk - 1) / chunk; }

template <typename T>
int forward(const ForwardArgs& a, hipStream_t st)
{
    const dim3 grid(a.row_blocks * a.splits * a.p.batch * a.p.kv_heads), block(kWaves * kWave);
    constexpr int kNarrow = sizeof(T) == 2 ? 64 : 32;       // keys of a tile: 64 KB of shared memory at width 128
    const bool async = async_rows(a.p.k, a.p.width, sizeof(T)) && async_rows(a.p.v, a.p.width, sizeof(T));
    if (a.p.width <= 64) {
        if (async) hipLaunchKernelGGL((sdl_attention_kernel<T, 64, 64, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((sdl_attention_kernel<T, 64, 64, false>), grid, block, 0, st, a);
    } else {
        if (async) hipLaunchKernelGGL((sdl_attention_kernel<T, 128, kNarrow, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((sdl_attention_kernel<T, 128, kNarrow, false>), grid, block, 0, st, a);
    }
    int rc = launched();
    if (rc != SDL_OK || a.splits == 1) return rc;
    const uint64_t lines = (uint64_t)a.p.batch * a.p.kv_heads * a.p.queries * a.p.group.d;
    hipLaunchKernelGGL((sdl_attention_join_kernel<T>), dim3((uint32_t)((lines + 3) / 4)), dim3(256), 0, st, a);
    return launched();
}

}  // namespace

extern "C" {

size_t sdl_attention_workspace_bytes(uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads, uint32_t width, sdl_dtype_t dtype)
{
    if (!sdl_attention_shape(batch, queries, keys, heads, kv_heads, width, dtype)) return 0;
    const uint32_t n = splits_of(chunk_of(batch, queries, keys, heads, kv_heads, dtype), keys);
    return n == 1 ? 0 : (size_t)n * batch * heads * queries * (width + 1) * sizeof(float);
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
    a.part_lse = a.part_out + (size_t)a.splits * batch * heads * queries * width;
    const uint64_t rows = (uint64_t)queries * a.p.group.d;
    a.row_blocks = (uint32_t)((rows + kRows - 1) / kRows);
    const uint64_t groups = (uint64_t)a.row_blocks * a.splits * batch * kv_heads;
    if (groups > 0x7fffffffu || (a.splits > 1 && (uint64_t)batch * queries * heads > 0x7fffffffu)) return SDL_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == SDL_DTYPE_BF16 ? forward<__bf16>(a, st) : forward<float>(a, st);
}

}  // extern "C"
