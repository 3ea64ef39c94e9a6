// Layer norm of rows of `width` elements, forward and backward (gfx950).
//
//   mean = sum x / C      rstd = 1 / sqrt(sum (x - mean)^2 / C + eps)      h = (x - mean) rstd
//   forward    y  = h w + b
//   backward   a  = dy w,  dx = rstd (a - sum a / C - h sum (a h) / C),  dw = sum over rows of dy h,  db = sum over rows of dy
//
// Memory bounds both: the forward pass reads x and writes y, the backward pass reads x and dy and writes dx.  A row stays in the
// registers of the TPR lanes that share it (eight elements a lane and step, K steps), so that the sum of squares is taken around the
// mean itself and x is read once.  All sums are fp32.
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
    uint32_t params_bf16;
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
__device__ __forceinline__ float row_sum(float x, float (*part)[8], int& turn)
{
    if constexpr (TPR <= kWave) {
        return lane_sum<TPR>(x);
    } else {
        x = lane_sum<kWave>(x);
        if ((threadIdx.x & (kWave - 1)) == 0) part[turn][threadIdx.x / kWave] = x;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / kWave; ++i) s += part[turn][i];
        turn ^= 1;
        return s;
    }
}

template <typename T, int BLOCK, int TPR, int K>
__global__ void __launch_bounds__(BLOCK) sdl_norm_kernel(const NormArgs a)
{
    __shared__ float part[2][8];
    int turn = 0;
    const uint32_t C = a.rows.width, lane = threadIdx.x % TPR;
    const uint32_t r = blockIdx.x * (BLOCK / TPR) + threadIdx.x / TPR;
    const bool in = r < a.rows.n;
    const uint32_t row = in ? r : a.rows.n - 1;
    const T* x = row_of<T>(a.x, a.rows, row);
    Eight<T> v[K];
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = load8(x, (k * TPR + lane) * 8, C);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[k].get(j);
    const float n = (float)C, mean = row_sum<TPR>(s, part, turn) / n;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = (k * TPR + lane) * 8 + j < C ? v[k].get(j) - mean : 0.0f;
            s = __builtin_fmaf(d, d, s);
        }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(s, part, turn) / n + a.eps);
    if (!in) return;
    T* y = row_of<T>(a.y, a.rows, row);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint32_t at = (k * TPR + lane) * 8;
        if (at >= C) break;
        float w[8], b[8], out[8];
        if (a.w) load_params(a.w, a.params_bf16, at, C, w);
        if (a.b) load_params(a.b, a.params_bf16, at, C, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float h = (v[k].get(j) - mean) * rstd;
            out[j] = __builtin_fmaf(h, a.w ? w[j] : 1.0f, a.b ? b[j] : 0.0f);
        }
        store8(y, at, C, out);
    }
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
}

// Every workgroup takes the rows r = its number, + gridDim, ...; a thread keeps the sums of dy h and dy of its columns in registers, the
// workgroup adds them up over its wavefronts in a fixed order and writes one line of partial sums.
template <typename T, int BLOCK, int TPR, int K>
__global__ void __launch_bounds__(BLOCK) sdl_norm_backward_kernel(const NormArgs a)
{
    constexpr int kRows = BLOCK / TPR;          // rows a workgroup has at a time
    constexpr int kLines = TPR < kWave ? BLOCK / kWave : kRows;
    __shared__ float part[2][8];
    __shared__ float sums[kLines > 1 ? kLines * (TPR < kWave ? TPR : TPR) * 8 : 1];
    int turn = 0;
    const uint32_t C = a.rows.width, lane = threadIdx.x % TPR;
    float w[K][8], dw[K][8], db[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[k][j] = 1.0f, dw[k][j] = 0.0f, db[k][j] = 0.0f;
        if (a.w) load_params(a.w, a.params_bf16, (k * TPR + lane) * 8, C, w[k]);
    }
    const float n = (float)C;
    for (uint32_t r0 = blockIdx.x * kRows; r0 < a.rows.n; r0 += gridDim.x * kRows) {
        const uint32_t r = r0 + threadIdx.x / TPR;
        const bool in = r < a.rows.n;
        const uint32_t row = in ? r : a.rows.n - 1;
        const T* x = row_of<T>(a.x, a.rows, row);
        const T* dy = row_of<T>(a.dy, a.rows, row);
        Eight<T> vx[K], vd[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            vx[k] = load8(x, (k * TPR + lane) * 8, C);
            vd[k] = load8(dy, (k * TPR + lane) * 8, C);
        }
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float g = vd[k].get(j) * w[k][j], h = (vx[k].get(j) - mean) * rstd;
                s1 += g;                                  // elements past the row: dy is 0 there
                s2 = __builtin_fmaf(g, h, s2);
            }
        s1 = row_sum<TPR>(s1, part, turn) / n;
        s2 = row_sum<TPR>(s2, part, turn) / n;
        if (in) {
            T* dx = row_of<T>(a.y, a.rows, row);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const uint32_t at = (k * TPR + lane) * 8;
                float out[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = vd[k].get(j), h = (vx[k].get(j) - mean) * rstd;
                    out[j] = rstd * (d * w[k][j] - s1 - h * s2);
                    dw[k][j] = __builtin_fmaf(d, h, dw[k][j]);
                    db[k][j] += d;
                }
                if (at < C) store8(dx, at, C, out);
            }
        }
    }
    if (!a.partial) return;
    float* line = a.partial + (uint64_t)blockIdx.x * 2 * C;
    if constexpr (kLines == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            store8(line, (k * TPR + lane) * 8, C, dw[k]);
            store8(line + C, (k * TPR + lane) * 8, C, db[k]);
        }
    } else {
        const uint32_t wave = threadIdx.x / kWave;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float s[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    s[j] = q ? db[k][j] : dw[k][j];
#pragma unroll
                    for (int m = TPR; m < kWave; m *= 2) s[j] += __shfl_xor(s[j], m);
                }
                __syncthreads();
                if ((threadIdx.x & (kWave - 1)) < TPR)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sums[(wave * TPR + lane) * 8 + j] = s[j];
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

struct SumArgs {
    const float* partial;
    void* dw;
    void* db;
    uint32_t lines, width, params_bf16;
};

// Column sums of the workgroups' lines: 64 columns and 16 shares of the lines a workgroup, each share added up in order, then the shares.
__global__ void __launch_bounds__(1024) sdl_norm_sum_kernel(const SumArgs a)
{
    __shared__ float sums[16][kWave];
    const uint32_t c = blockIdx.x * kWave + threadIdx.x % kWave, share = threadIdx.x / kWave, C2 = 2 * a.width;
    float s = 0.0f;
    if (c < C2)
        for (uint32_t l = share; l < a.lines; l += 16) s += a.partial[(uint64_t)l * C2 + c];
    sums[share][threadIdx.x % kWave] = s;
    __syncthreads();
    if (share != 0 || c >= C2) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += sums[i][threadIdx.x];
    void* out = c < a.width ? a.dw : a.db;
    const uint32_t at = c < a.width ? c : c - a.width;
    if (!out) return;
    if (a.params_bf16)
        static_cast<__bf16*>(out)[at] = (__bf16)s;
    else
        static_cast<float*>(out)[at] = s;
}

constexpr uint32_t kMaxLines = 256;     // workgroups of a backward launch, at most

template <typename T>
int forward(const NormArgs& a, hipStream_t st)
{
    const uint32_t C = a.rows.width, n = a.rows.n;
#define SDL_LAUNCH(BLOCK, TPR, K) hipLaunchKernelGGL((sdl_norm_kernel<T, BLOCK, TPR, K>), dim3((n + (BLOCK / TPR) - 1) / (BLOCK / TPR)), dim3(BLOCK), 0, st, a)
    if (C <= 64) SDL_LAUNCH(256, 8, 1);
    else if (C <= 128) SDL_LAUNCH(256, 16, 1);
    else if (C <= 256) SDL_LAUNCH(256, 32, 1);
    else if (C <= 512) SDL_LAUNCH(256, 64, 1);
    else if (C <= 1024) SDL_LAUNCH(256, 64, 2);
    else if (C <= 2048) SDL_LAUNCH(256, 64, 4);
    else if (C <= 4096) SDL_LAUNCH(512, 512, 1);
    else if (C <= 8192) SDL_LAUNCH(512, 512, 2);
    else SDL_LAUNCH(512, 512, 4);
#undef SDL_LAUNCH
    return launched();
}

template <typename T>
int backward(const NormArgs& a, uint32_t* lines, hipStream_t st)
{
    const uint32_t C = a.rows.width, n = a.rows.n;
#define SDL_LAUNCH(TPR, K)                                                                                                 \
    do {                                                                                                                   \
        const uint32_t groups = (n + (512 / TPR) - 1) / (512 / TPR);                                                       \
        *lines = groups < kMaxLines ? groups : kMaxLines;                                                                  \
        hipLaunchKernelGGL((sdl_norm_backward_kernel<T, 512, TPR, K>), dim3(*lines), dim3(512), 0, st, a);                 \
    } while (0)
    if (C <= 64) SDL_LAUNCH(8, 1);
    else if (C <= 128) SDL_LAUNCH(16, 1);
    else if (C <= 256) SDL_LAUNCH(32, 1);
    else if (C <= 512) SDL_LAUNCH(64, 1);
    else if (C <= 1024) SDL_LAUNCH(64, 2);
    else if (C <= 2048) SDL_LAUNCH(64, 4);
    else if (C <= 4096) SDL_LAUNCH(512, 1);
    else if (C <= 8192) SDL_LAUNCH(512, 2);
    else SDL_LAUNCH(512, 4);
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
    a.params_bf16 = param_dtype == SDL_DTYPE_BF16;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == SDL_DTYPE_BF16 ? forward<__bf16>(a, st) : forward<float>(a, st);
}

size_t sdl_layer_norm_workspace_bytes(uint32_t width)
{
    return width > SDL_NORM_MAX_WIDTH ? 0 : (size_t)kMaxLines * 2 * width * sizeof(float);
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
        a.partial = sums ? static_cast<float*>(workspace) : nullptr;
        a.params_bf16 = param_dtype == SDL_DTYPE_BF16;
        rc = dtype == SDL_DTYPE_BF16 ? backward<__bf16>(a, &lines, st) : backward<float>(a, &lines, st);
        if (rc != SDL_OK) return rc;
    }
    if (!sums) return SDL_OK;
    const SumArgs s{static_cast<const float*>(workspace), dweight, dbias, lines, width, param_dtype == SDL_DTYPE_BF16};
    hipLaunchKernelGGL(sdl_norm_sum_kernel, dim3((2 * width + kWave - 1) / kWave), dim3(1024), 0, st, s);
    return launched();
}

}  // extern "C"
