// Layer norm of rows of `width` elements, forward and backward (gfx950).
//
//   mean = sum x / C      rstd = 1 / sqrt(sum (x - mean)^2 / C + eps)      h = (x - mean) rstd
//   forward    y  = h w + b
//   backward   a  = dy w,  dx = rstd (a - sum a / C - h sum (a h) / C),  dw = sum over rows of dy h,  db = sum over rows of dy
//
// Memory bounds both: the forward pass reads x and writes y, the backward pass reads x and dy and writes dx.  A row stays in the
// registers of the TPR lanes that share it (eight elements a lane and step, K steps), so that the sum of squares is taken around the
// mean itself and x is read once.  All sums are fp32.
//
// 8192 rows of 2048 in bf16: forward 13.1 us, 5.1 TB/s; backward 19.8 us, 5.1 TB/s, and 3.8 for the sums of dw; a copy of that size takes 10.3 us, 6.5 TB/s.
// 98,304 rows of 64: 8.8 and 11.6 us.  A launch that does nothing takes 3: small calls are the host's launches, 2.5 us each.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "sdl_operand.h"

namespace {

using namespace sdl_device;

struct Rows {
    Div heads, tokens;      // row -> (batch, token, head), head fastest
    uint32_t n;
    uint32_t width;
};

struct NormArgs {
    Rows rows;
    View x, y, dy;          // backward: y is dx
    const void* w;
    const void* b;
    float* mean;
    float* rstd;
    float* partial;         // backward: [workgroups][2][width]
    float eps;
    uint32_t sums;          // backward: 1 for dweight, 2 for dbias
};

template <typename T>
__device__ __forceinline__ T* row_of(const View& v, const Rows& rows, uint32_t r)
{
    const uint32_t bt = div(r, rows.heads), h = r - bt * rows.heads.d;
    const uint32_t b = div(bt, rows.tokens), t = bt - b * rows.tokens.d;
    return reinterpret_cast<T*>(v.data) + ((int64_t)b * v.batch + (int64_t)t * v.token + (int64_t)h * v.head);
}

// Sum over the TPR threads of a row; more than one wavefront goes through shared memory (`turn` alternates its two halves, so that one
// barrier a sum is enough).
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float (*part)[16], int& turn)
{
    if constexpr (TPR <= kWave) {
        return lane_sum<TPR>(x);
    } else {
        x = lane_sum<kWave>(x);
        if ((threadIdx.x & (kWave - 1)) == 0) part[turn][threadIdx.x / kWave] = x;
        __syncthreads();
        const uint32_t first = threadIdx.x / TPR * (TPR / kWave);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / kWave; ++i) s += part[turn][first + i];
        turn ^= 1;
        return s;
    }
}

// Eight parameters a step, as they lie in memory: bf16 takes half the registers.
struct Params {
    u32x4 lo, hi;
    __device__ __forceinline__ float get(bool bf16, int j) const
    {
        const uint32_t half = lo[j / 2], whole = j < 4 ? lo[j & 3] : hi[j & 3];
        return u2f(!bf16 ? whole : (j & 1) ? (half & 0xffff0000u) : (half << 16));
    }
};
__device__ __forceinline__ Params load_raw(const void* p, bool bf16, uint32_t at, uint32_t n)
{
    if (bf16) return Params{load8(static_cast<const __bf16*>(p), at, n).w, u32x4{}};
    const Eight<float> x = load8(static_cast<const float*>(p), at, n);
    return Params{x.lo, x.hi};
}

// A workgroup takes the rows of its number, + gridDim, ...: the parameters stay in registers, and the next row is on its way while one is worked on.
template <typename T, bool PB, int BLOCK, int TPR, int K>
__global__ void __launch_bounds__(BLOCK) sdl_norm_kernel(const NormArgs a)
{
    constexpr uint32_t kRows = BLOCK / TPR;
    __shared__ float part[2][16];
    int turn = 0;
    const uint32_t C = a.rows.width, lane = threadIdx.x % TPR;
    uint32_t r0 = blockIdx.x * kRows;
    const uint32_t mine = threadIdx.x / TPR;
    Eight<T> next[K];
    const T* x = row_of<T>(a.x, a.rows, min(r0 + mine, a.rows.n - 1));
#pragma unroll
    for (int k = 0; k < K; ++k) next[k] = load8(x, (k * TPR + lane) * 8, C);
    Params w[K], b[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (a.w) w[k] = load_raw(a.w, PB, (k * TPR + lane) * 8, C);
        if (a.b) b[k] = load_raw(a.b, PB, (k * TPR + lane) * 8, C);
    }
    for (; r0 < a.rows.n; r0 += gridDim.x * kRows) {
        const uint32_t r = r0 + mine;
        float v[K][8], s = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = next[k].get(j);
        if (r0 + gridDim.x * kRows < a.rows.n) {
            x = row_of<T>(a.x, a.rows, min(r + gridDim.x * kRows, a.rows.n - 1));
#pragma unroll
            for (int k = 0; k < K; ++k) next[k] = load8(x, (k * TPR + lane) * 8, C);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[k][j];
        const float n = (float)C, mean = row_sum<TPR>(s, part, turn) / n;
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[k][j] -= mean;
                if ((k * TPR + lane) * 8 + j >= C) v[k][j] = 0.0f;
                s = __builtin_fmaf(v[k][j], v[k][j], s);
            }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(s, part, turn) / n + a.eps);
        if (r >= a.rows.n) continue;
        T* y = row_of<T>(a.y, a.rows, r);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t at = (k * TPR + lane) * 8;
            float out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) out[j] = __builtin_fmaf(v[k][j] * rstd, a.w ? w[k].get(PB, j) : 1.0f, a.b ? b[k].get(PB, j) : 0.0f);
            if (at < C) store8(y, at, C, out);
        }
        if (lane == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

// The rows as above; a thread keeps the sums of dy h and dy of its columns in registers, the workgroup adds them up over its wavefronts in a fixed
// order and writes one line of partial sums.
template <typename T, bool PB, int BLOCK, int TPR, int K>
__global__ void __launch_bounds__(BLOCK) sdl_norm_backward_kernel(const NormArgs a)
{
    constexpr uint32_t kRows = BLOCK / TPR;          // rows a workgroup has at a time
    constexpr bool kAhead = K * sizeof(T) <= 8;      // whether the registers hold the next row as well
    constexpr int kLines = TPR < kWave ? BLOCK / kWave : (int)kRows;
    __shared__ float part[2][16];
    __shared__ float sums[kLines > 1 ? kLines * TPR * 8 : 1];
    int turn = 0;
    const uint32_t C = a.rows.width, lane = threadIdx.x % TPR, mine = threadIdx.x / TPR;
    uint32_t r0 = blockIdx.x * kRows;
    Eight<T> next_x[K], next_d[K];
    float next_mean, next_rstd;
    auto load = [&](uint32_t r) __attribute__((always_inline)) {
        const uint32_t row = min(r, a.rows.n - 1);
        const T* x = row_of<T>(a.x, a.rows, row);
        const T* dy = row_of<T>(a.dy, a.rows, row);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            next_x[k] = load8(x, (k * TPR + lane) * 8, C);
            next_d[k] = load8(dy, (k * TPR + lane) * 8, C);
        }
        next_mean = a.mean[row];
        next_rstd = a.rstd[row];
    };
    if constexpr (kAhead) load(r0 + mine);
    Params w[K];
    float dw[K][8], db[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (a.w) w[k] = load_raw(a.w, PB, (k * TPR + lane) * 8, C);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[k][j] = 0.0f, db[k][j] = 0.0f;
    }
    const float n = (float)C;
    for (; r0 < a.rows.n; r0 += gridDim.x * kRows) {
        const uint32_t r = r0 + mine;
        if constexpr (!kAhead) load(r);
        Eight<T> vx[K], vd[K];
#pragma unroll
        for (int k = 0; k < K; ++k) vx[k] = next_x[k], vd[k] = next_d[k];
        const float mean = next_mean, rstd = next_rstd;
        if constexpr (kAhead) {
            if (r0 + gridDim.x * kRows < a.rows.n) load(r + gridDim.x * kRows);
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float g = vd[k].get(j) * (a.w ? w[k].get(PB, j) : 1.0f), h = (vx[k].get(j) - mean) * rstd;
                s1 += g;                                  // elements past the row: dy is 0 there
                s2 = __builtin_fmaf(g, h, s2);
            }
        s1 = row_sum<TPR>(s1, part, turn) / n;
        s2 = row_sum<TPR>(s2, part, turn) / n;
        if (r >= a.rows.n) continue;
        T* dx = row_of<T>(a.y, a.rows, r);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t at = (k * TPR + lane) * 8;
            float out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = vd[k].get(j), h = (vx[k].get(j) - mean) * rstd;
                out[j] = rstd * (d * (a.w ? w[k].get(PB, j) : 1.0f) - s1 - h * s2);
                dw[k][j] = __builtin_fmaf(d, h, dw[k][j]);
                db[k][j] += d;
            }
            if (at < C) store8(dx, at, C, out);
        }
    }
    float* line = a.partial + (uint64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if (!(a.sums & (1u << q))) continue;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = q ? db[k][j] : dw[k][j];
            if constexpr (kLines == 1) {
                store8(line + q * C, (k * TPR + lane) * 8, C, s);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int m = TPR; m < kWave; m *= 2) s[j] += __shfl_xor(s[j], m);
                __syncthreads();
                if ((threadIdx.x & (kWave - 1)) < TPR)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sums[(threadIdx.x / (TPR < kWave ? kWave : TPR) * TPR + lane) * 8 + j] = s[j];
                __syncthreads();
                for (uint32_t c = threadIdx.x; c < TPR * 8; c += BLOCK) {
                    float t = 0.0f;
#pragma unroll
                    for (int l = 0; l < kLines; ++l) t += sums[l * TPR * 8 + c];
                    if (k * TPR * 8 + c < C) line[q * C + k * TPR * 8 + c] = t;
                }
            }
        }
    }
}

struct SumArgs {
    const float* partial;
    void* dw;
    void* db;
    uint32_t lines, width, params_bf16, first, columns;       // columns [first, first + columns) of a line
};

// Column sums of the workgroups' lines: 32 columns and 32 shares of the lines a workgroup, each share added up in order, then the shares.
__global__ void __launch_bounds__(1024) sdl_norm_sum_kernel(const SumArgs a)
{
    __shared__ float sums[32][33];
    const uint32_t col = threadIdx.x % 32, share = threadIdx.x / 32, i = blockIdx.x * 32 + col, c = a.first + i;
    float s = 0.0f;
    if (i < a.columns) {
        const float* p = a.partial + (uint64_t)share * 2 * a.width + c;
#pragma unroll 8
        for (uint32_t l = share; l < a.lines; l += 32, p += 64 * (uint64_t)a.width) s += *p;
    }
    sums[share][col] = s;
    __syncthreads();
    if (share != 0 || i >= a.columns) return;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += sums[k][col];
    void* out = c < a.width ? a.dw : a.db;
    const uint32_t at = c < a.width ? c : c - a.width;
    if (a.params_bf16)
        static_cast<__bf16*>(out)[at] = (__bf16)s;
    else
        static_cast<float*>(out)[at] = s;
}

// Workgroups of a backward launch, at most: one for every compute unit, as each leaves a line of sums; two for rows that are little to wait for and still keep most of a
// wavefront's lanes.  With the column sums, in us, 256 / 512 / 768 of them: 16,384 rows in bf16 of 128 6.7 / 7.1 / 7.1, of 192 10.6 / 9.6 / 11.8, of 300 19.9 / 16.1 / 18.6 (fp32 20.2 /
// 16.9 / 18.6), of 512 13.9 / 13.6 / 13.9, of 520 21.1 / 22.9 / 24.8; 98,304 of 64 11.2 / 11.0 / 11.5; 8192 of 768 13.9 / 15.8 / 17.9.
constexpr uint32_t most_lines(uint32_t width) { return width > 128 && width <= 512 ? 512 : 256; }
// Of a forward launch: four for every compute unit, and eight of those with two rows at a time.  Two wavefronts a row at widths over 1024, 8192 rows of 2048 in bf16
// 14.3 us with one and 13.1 with two, 16,384 of 1500 29 and 26; 8192 rows of 768, of one wavefront, 8.8 us with 1024 workgroups and 9.8 with 2048.
constexpr uint32_t kForward = 1024;

template <typename T, bool PB>
int forward(const NormArgs& a, hipStream_t st)
{
    const uint32_t C = a.rows.width, n = a.rows.n;
#define SDL_LAUNCH(BLOCK, TPR, K)                                                                                          \
    do {                                                                                                                   \
        const uint32_t groups = (n + (BLOCK / TPR) - 1) / (BLOCK / TPR);                                                   \
        const uint32_t most = TPR == 128 ? 2 * kForward : kForward;                                                       \
        hipLaunchKernelGGL((sdl_norm_kernel<T, PB, BLOCK, TPR, K>), dim3(groups < most ? groups : most), dim3(BLOCK), 0, st, a); \
    } while (0)
    if (C <= 64) SDL_LAUNCH(256, 8, 1);
    else if (C <= 128) SDL_LAUNCH(256, 16, 1);
    else if (C <= 256) SDL_LAUNCH(256, 32, 1);
    else if (C <= 512) SDL_LAUNCH(256, 64, 1);
    else if (C <= 1024) SDL_LAUNCH(256, 64, 2);
    else if (C <= 2048) SDL_LAUNCH(256, 128, 2);
    else if (C <= 4096) SDL_LAUNCH(512, 512, 1);
    else if (C <= 8192) SDL_LAUNCH(512, 512, 2);
    else SDL_LAUNCH(1024, 1024, 2);
#undef SDL_LAUNCH
    return launched();
}

template <typename T, bool PB>
int backward(const NormArgs& a, uint32_t* lines, hipStream_t st)
{
    const uint32_t C = a.rows.width, n = a.rows.n;
#define SDL_LAUNCH(BLOCK, TPR, K)                                                                                          \
    do {                                                                                                                   \
        const uint32_t groups = (n + (BLOCK / TPR) - 1) / (BLOCK / TPR);                                                   \
        *lines = groups < most_lines(C) ? groups : most_lines(C);                                                                  \
        hipLaunchKernelGGL((sdl_norm_backward_kernel<T, PB, BLOCK, TPR, K>), dim3(*lines), dim3(BLOCK), 0, st, a);         \
    } while (0)
    if (C <= 64) SDL_LAUNCH(512, 8, 1);
    else if (C <= 128) SDL_LAUNCH(512, 16, 1);
    else if (C <= 256) SDL_LAUNCH(512, 32, 1);
    else if (C <= 512) SDL_LAUNCH(512, 64, 1);
    else if (C <= 1024) SDL_LAUNCH(512, 64, 2);
    else if (C <= 2048 && sizeof(T) == 2) SDL_LAUNCH(512, 64, 4);
    else if (C <= 2048) SDL_LAUNCH(512, 256, 1);
    else if (C <= 4096) SDL_LAUNCH(512, 512, 1);
    else if (C <= 8192) SDL_LAUNCH(512, 512, 2);
    else SDL_LAUNCH(512, 512, 4);
#undef SDL_LAUNCH
    return launched();
}

int check_shape(uint32_t batch, uint32_t tokens, uint32_t heads, uint32_t width, sdl_dtype_t dtype, sdl_dtype_t param_dtype)
{
    if (!known(dtype) || !known(param_dtype) || width == 0) return SDL_ERR_INVALID_ARG;
    if (width > SDL_NORM_MAX_WIDTH) return SDL_ERR_UNSUPPORTED;
    const uint64_t bt = (uint64_t)batch * tokens;
    if (bt > 0x7fffffffu || bt * heads > 0x7fffffffu) return SDL_ERR_UNSUPPORTED;
    return SDL_OK;
}

Rows make_rows(uint32_t batch, uint32_t tokens, uint32_t heads, uint32_t width)
{
    return Rows{make_div(heads), make_div(tokens), batch * tokens * heads, width};
}

}  // namespace

extern "C" {

int sdl_layer_norm(const sdl_view_t* x, uint32_t batch, uint32_t tokens, uint32_t heads, uint32_t width, sdl_dtype_t dtype,
                   const void* weight, const void* bias, sdl_dtype_t param_dtype, float eps, const sdl_view_t* y, float* mean,
                   float* rstd, void* stream)
{
    int rc = check_shape(batch, tokens, heads, width, dtype, param_dtype);
    if (rc != SDL_OK) return rc;
    if (!(eps >= 0.0f) || eps > 3.4028235e38f) return SDL_ERR_INVALID_ARG;
    if (batch == 0 || tokens == 0 || heads == 0) return SDL_OK;
    if ((rc = check_view(x, dtype)) != SDL_OK) return rc;
    if ((rc = check_output(y, dtype, batch, tokens, heads)) != SDL_OK) return rc;
    if (!aligned_to(weight, dtype_size(param_dtype)) || !aligned_to(bias, dtype_size(param_dtype)) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return SDL_ERR_ALIGNMENT;
    NormArgs a{};
    a.rows = make_rows(batch, tokens, heads, width);
    a.x = kernel_view(x);
    a.y = kernel_view(y);
    a.w = weight;
    a.b = bias;
    a.mean = mean;
    a.rstd = rstd;
    a.eps = eps;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (param_dtype == SDL_DTYPE_BF16) return dtype == SDL_DTYPE_BF16 ? forward<__bf16, true>(a, st) : forward<float, true>(a, st);
    return dtype == SDL_DTYPE_BF16 ? forward<__bf16, false>(a, st) : forward<float, false>(a, st);
}

size_t sdl_layer_norm_workspace_bytes(uint32_t width)
{
    return width > SDL_NORM_MAX_WIDTH ? 0 : (size_t)most_lines(width) * 2 * width * sizeof(float);
}

int sdl_layer_norm_backward(const sdl_view_t* dy, const sdl_view_t* x, uint32_t batch, uint32_t tokens, uint32_t heads, uint32_t width,
                            sdl_dtype_t dtype, const void* weight, sdl_dtype_t param_dtype, const float* mean, const float* rstd,
                            const sdl_view_t* dx, void* dweight, void* dbias, void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = check_shape(batch, tokens, heads, width, dtype, param_dtype);
    if (rc != SDL_OK) return rc;
    const bool sums = dweight || dbias, empty = batch == 0 || tokens == 0 || heads == 0;
    const size_t p = dtype_size(param_dtype);
    if (!aligned_to(weight, p) || !aligned_to(dweight, p) || !aligned_to(dbias, p)) return SDL_ERR_ALIGNMENT;
    NormArgs a{};
    hipStream_t st = static_cast<hipStream_t>(stream);
    uint32_t lines = 0;
    if (!empty) {
        if ((rc = check_view(dy, dtype)) != SDL_OK || (rc = check_view(x, dtype)) != SDL_OK) return rc;
        if ((rc = check_output(dx, dtype, batch, tokens, heads)) != SDL_OK) return rc;
        if (!mean || !rstd) return SDL_ERR_INVALID_ARG;
        if (!aligned_to(mean, 4) || !aligned_to(rstd, 4) || !aligned_to(workspace, 4)) return SDL_ERR_ALIGNMENT;
        if (sums && (!workspace || workspace_bytes < sdl_layer_norm_workspace_bytes(width))) return SDL_ERR_INVALID_ARG;
        a.rows = make_rows(batch, tokens, heads, width);
        a.x = kernel_view(x);
        a.dy = kernel_view(dy);
        a.y = kernel_view(dx);
        a.w = weight;
        a.mean = const_cast<float*>(mean);
        a.rstd = const_cast<float*>(rstd);
        a.partial = static_cast<float*>(workspace);
        a.sums = (dweight ? 1u : 0u) | (dbias ? 2u : 0u);
        if (param_dtype == SDL_DTYPE_BF16)
            rc = dtype == SDL_DTYPE_BF16 ? backward<__bf16, true>(a, &lines, st) : backward<float, true>(a, &lines, st);
        else
            rc = dtype == SDL_DTYPE_BF16 ? backward<__bf16, false>(a, &lines, st) : backward<float, false>(a, &lines, st);
        if (rc != SDL_OK) return rc;
    }
    if (!sums) return SDL_OK;
    const uint32_t first = dweight ? 0 : width, columns = dweight && dbias ? 2 * width : width;
    const SumArgs s{static_cast<const float*>(workspace), dweight, dbias, lines, width, param_dtype == SDL_DTYPE_BF16, first, columns};
    hipLaunchKernelGGL(sdl_norm_sum_kernel, dim3((columns + 31) / 32), dim3(1024), 0, st, s);
    return launched();
}

}  // extern "C"
