// Cross entropy of logits with targets, and its gradient (gfx950).
//
// A row of logits is read once and stays in the registers of 64 to 1024 threads, its gradient is written once: both passes in one call move
// what one pass has to, and that is what bounds them.  Every thread takes the maximum m of its elements and the sum s of exp(x - m) over them; two such pairs
// are one with M = max(m1, m2), s = s1 exp(m1 - M) + s2 exp(m2 - M), so that a row costs one exchange between its threads.  With M and s of the row,
//     lse = M + log s,   p = exp(x - M) / s
// and the loss is formed from M - x[target] and log s, which loses nothing where the target is nearly certain and lse and x[target] are nearly equal.
#include "sdl_operand.h"

namespace {

using namespace sdl_device;

constexpr float kLog2e = 1.44269504088896340736f;

struct LossArgs {
    View x, d;
    const void* targets;
    const float* d_loss;
    float *loss, *lse;
    Div tokens;
    uint32_t rows, vocab, wide;     // targets of 64 bits
    float smoothing, hit, share, z; // hit = 1 - smoothing, share = smoothing / vocab
};

// The row's target, or a negative number where it has none.
__device__ __forceinline__ int32_t target_of(const LossArgs& a, uint32_t row)
{
    const int64_t t = a.wide ? static_cast<const int64_t*>(a.targets)[row] : (int64_t) static_cast<const int32_t*>(a.targets)[row];
    return t >= 0 && t < (int64_t)a.vocab ? (int32_t)t : -1;
}

template <typename T>
__device__ __forceinline__ T* row_of(const LossArgs& a, const View& v, uint32_t row)
{
    const uint32_t b = div(row, a.tokens), t = row - b * a.tokens.d;
    return reinterpret_cast<T*>(v.data) + ((int64_t)b * v.batch + (int64_t)t * v.token);
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// exp(x - m) where m is at least x
__device__ __forceinline__ float exp_under(float x, float m) { return exp2_of((x - m) * kLog2e); }

// Maximum, sum of exp(x - maximum), sum of x, and the target's logit (0 in the lanes that do not have it).
struct Part {
    float m, s, sum, hit;
};

// exp(from - to) for the joining of two parts; a part of nothing but -infinity has s = 0.
__device__ __forceinline__ Part join(const Part& a, const Part& b)
{
    const float m = fmaxf(a.m, b.m);
    const float base = m == -__builtin_inff() ? 0.0f : m;
    return Part{m, a.s * exp_under(a.m, base) + b.s * exp_under(b.m, base), a.sum + b.sum, a.hit + b.hit};
}

__device__ __forceinline__ Part wave_join(Part p)
{
#pragma unroll
    for (int k = 32; k; k /= 2) {
        const Part q{__shfl_xor(p.m, k), __shfl_xor(p.s, k), __shfl_xor(p.sum, k), __shfl_xor(p.hit, k)};
        p = join(p, q);         // the same bits in both lanes: sums of two do not go by their order
    }
    return p;
}

// Elements [at, at + 8) of a row of n; what is behind the row is -infinity.
__device__ __forceinline__ Eight<__bf16> load_logits(const __bf16* row, uint32_t at, uint32_t n)
{
    if (at + 8 <= n) return load8(row, at, n);
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
    uint32_t h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = at + j < n ? p[at + j] : 0xff80u;
    return Eight<__bf16>{u32x4{h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16)}};
}
__device__ __forceinline__ Eight<float> load_logits(const float* row, uint32_t at, uint32_t n)
{
    if (at + 8 <= n) return load8(row, at, n);
    const uint32_t* p = reinterpret_cast<const uint32_t*>(row);
    Eight<float> r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        r.lo[j] = at + j < n ? p[at + j] : 0xff800000u;
        r.hi[j] = at + 4 + j < n ? p[at + 4 + j] : 0xff800000u;
    }
    return r;
}

// What K groups of eight elements, TPR groups apart, are as a part of their row.
template <typename T, int K, int TPR>
__device__ __forceinline__ Part part_of(const Eight<T> (&e)[K], uint32_t first, uint32_t n, int32_t target, bool smooth)
{
    float m[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        m[k] = e[k].get(0);
#pragma unroll
        for (int j = 1; j < 8; ++j) m[k] = fmaxf(m[k], e[k].get(j));
    }
    Part p{m[0], 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 1; k < K; ++k) p.m = fmaxf(p.m, m[k]);
    const float base = p.m == -__builtin_inff() ? 0.0f : p.m;
    float s[4] = {};
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j % 4] += exp_under(e[k].get(j), base);
        const uint32_t at = first + k * TPR * 8;
        if (smooth && at < n) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += at + j < n ? e[k].get(j) : 0.0f;
            p.sum += sum;
        }
        if (at == ((uint32_t)target & ~7u)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) p.hit = j == (target & 7) ? e[k].get(j) : p.hit;
        }
    }
    p.s = (s[0] + s[1]) + (s[2] + s[3]);
    return p;
}

// The row's loss and lse, from its whole part.
__device__ __forceinline__ void write_loss(const LossArgs& a, uint32_t row, const Part& p)
{
    const float log_s = logf(p.s);
    const float lse = p.m + log_s;
    float loss = log_s + a.hit * (p.m - p.hit);
    if (a.smoothing > 0.0f) loss += a.smoothing * (p.m - p.sum / (float)a.vocab);
    if (a.z != 0.0f) loss += a.z * lse * lse;
    if (a.loss) a.loss[row] = loss;
    if (a.lse) a.lse[row] = lse;
}

// Gradient of eight elements: factor exp(x - m) - even, and `hit` less at the target.
template <typename T>
__device__ __forceinline__ void write_gradient(T* row, uint32_t at, uint32_t n, const Eight<T>& e, float m, float factor, float even, float hit, int32_t target)
{
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = factor * exp_under(e.get(j), m) - even;
    if (at == ((uint32_t)target & ~7u)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] -= j == (target & 7) ? hit : 0.0f;
    }
    store8(row, at, n, v);
}

template <typename T, int TPR>
__device__ __forceinline__ void write_zeros(T* row, uint32_t first, uint32_t n)
{
    const float zero[8] = {};
    for (uint32_t at = first; at < n; at += TPR * 8) store8(row, at, n, zero);
}

// TPR threads a row, K groups of eight elements each; FIT: a row is that long at most and stays in the registers, else it is read again for its gradient.
template <typename T, int BLOCK, int TPR, int K, bool FIT>
__global__ void __launch_bounds__(BLOCK) sdl_cross_entropy_kernel(const LossArgs a)
{
    constexpr int kWaves = TPR / kWave;
    static_assert(TPR == kWave || TPR == BLOCK, "a row is a wavefront's or a workgroup's");
    const uint32_t row = workgroup() * (BLOCK / TPR) + threadIdx.x / TPR, n = a.vocab, first = threadIdx.x % TPR * 8;
    if (row >= a.rows) return;
    const int32_t target = target_of(a, row);
    T* d = a.d.data ? row_of<T>(a, a.d, row) : nullptr;
    if (target < 0) {
        if (threadIdx.x % TPR == 0) {
            if (a.loss) a.loss[row] = 0.0f;
            if (a.lse) a.lse[row] = 0.0f;
        }
        if (d) write_zeros<T, TPR>(d, first, n);
        return;
    }
    const T* x = row_of<const T>(a, a.x, row);
    const bool smooth = a.smoothing > 0.0f;
    Eight<T> e[K];
    Part p{-__builtin_inff(), 0.0f, 0.0f, 0.0f};
    if constexpr (FIT) {
#pragma unroll
        for (int k = 0; k < K; ++k) e[k] = load_logits(x, first + k * TPR * 8, n);
        p = part_of<T, K, TPR>(e, first, n, target, smooth);
    } else {
        for (uint32_t at = first; at < n; at += TPR * 8 * K) {
#pragma unroll
            for (int k = 0; k < K; ++k) e[k] = load_logits(x, at + k * TPR * 8, n);
            p = join(p, part_of<T, K, TPR>(e, at, n, target, smooth));
        }
    }
    p = wave_join(p);
    if constexpr (kWaves > 1) {
        __shared__ Part parts[kWaves];
        if (threadIdx.x % kWave == 0) parts[threadIdx.x / kWave] = p;
        __syncthreads();
        p = parts[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) p = join(p, parts[w]);
    }
    if (threadIdx.x % TPR == 0) write_loss(a, row, p);
    if (!d) return;
    const float g = a.d_loss ? a.d_loss[row] : 1.0f;
    const float factor = g * (1.0f + 2.0f * a.z * (p.m + logf(p.s))) / p.s, even = g * a.share, hit = g * a.hit;
    if constexpr (FIT) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t at = first + k * TPR * 8;
            if (at < n) write_gradient(d, at, n, e[k], p.m, factor, even, hit, target);
        }
    } else {
        for (uint32_t at = first; at < n; at += TPR * 8 * K) {
#pragma unroll
            for (int k = 0; k < K; ++k) e[k] = load_logits(x, at + k * TPR * 8, n);
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (at + k * TPR * 8 < n) write_gradient(d, at + k * TPR * 8, n, e[k], p.m, factor, even, hit, target);
        }
    }
}

// The gradient alone, from the forward pass' lse.
template <typename T, int BLOCK, int TPR, int K>
__global__ void __launch_bounds__(BLOCK) sdl_cross_entropy_backward_kernel(const LossArgs a)
{
    const uint32_t row = workgroup() * (BLOCK / TPR) + threadIdx.x / TPR, n = a.vocab, first = threadIdx.x % TPR * 8;
    if (row >= a.rows) return;
    const int32_t target = target_of(a, row);
    T* d = row_of<T>(a, a.d, row);
    if (target < 0) {
        write_zeros<T, TPR>(d, first, n);
        return;
    }
    const T* x = row_of<const T>(a, a.x, row);
    const float lse = a.lse[row], g = a.d_loss ? a.d_loss[row] : 1.0f;
    const float factor = g * (1.0f + 2.0f * a.z * lse), even = g * a.share, hit = g * a.hit;
    for (uint32_t at = first; at < n; at += TPR * 8 * K) {
        Eight<T> e[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            e[k] = Eight<T>{};
            if (at + k * TPR * 8 < n) e[k] = load8(x, at + k * TPR * 8, n);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (at + k * TPR * 8 < n) write_gradient(d, at + k * TPR * 8, n, e[k], lse, factor, even, hit, target);
    }
}

template <typename T>
int loss(const LossArgs& a, hipStream_t st)
{
    const uint32_t V = a.vocab;
#define SDL_LAUNCH(BLOCK, TPR, K, FIT) \
    hipLaunchKernelGGL((sdl_cross_entropy_kernel<T, BLOCK, TPR, K, FIT>), grid_of((a.rows - 1) / (BLOCK / TPR) + 1), dim3(BLOCK), 0, st, a)
    if (V <= 512) SDL_LAUNCH(256, 64, 1, true);
    else if (V <= 1024) SDL_LAUNCH(256, 64, 2, true);
    else if (V <= 2048) SDL_LAUNCH(256, 64, 4, true);
    else if (V <= 4096) SDL_LAUNCH(256, 256, 2, true);
    else if (V <= 8192) SDL_LAUNCH(256, 256, 4, true);
    else if (V <= 16384) SDL_LAUNCH(512, 512, 4, true);
    else if (V <= 32768) SDL_LAUNCH(512, 512, 8, true);
    else if (V <= 65536) SDL_LAUNCH(1024, 1024, 8, true);
    else if (V <= 131072 && sizeof(T) == 2) SDL_LAUNCH(1024, 1024, 16, true);
    else SDL_LAUNCH(1024, 1024, 4, false);
#undef SDL_LAUNCH
    return launched();
}

template <typename T>
int gradient(const LossArgs& a, hipStream_t st)
{
    if (a.vocab <= 2048)
        hipLaunchKernelGGL((sdl_cross_entropy_backward_kernel<T, 256, 64, 4>), grid_of((a.rows - 1) / 4 + 1), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((sdl_cross_entropy_backward_kernel<T, 256, 256, 4>), grid_of(a.rows), dim3(256), 0, st, a);
    return launched();
}

int check(const sdl_view_t* logits, uint32_t batch, uint32_t tokens, uint32_t vocab, sdl_dtype_t dtype, const void* targets, sdl_index_t index, float smoothing,
          float z)
{
    if (!known(dtype) || (index != SDL_INDEX_INT32 && index != SDL_INDEX_INT64) || vocab == 0) return SDL_ERR_INVALID_ARG;
    if (!(smoothing >= 0.0f && smoothing <= 1.0f) || !(z >= 0.0f && z - z == 0.0f)) return SDL_ERR_INVALID_ARG;
    if (vocab > SDL_CROSS_ENTROPY_MAX_VOCAB || (uint64_t)batch * tokens > 0x7fffffffu) return SDL_ERR_UNSUPPORTED;
    if (batch == 0 || tokens == 0) return SDL_OK;
    const int rc = check_view(logits, dtype);
    if (rc != SDL_OK) return rc;
    if (!targets) return SDL_ERR_INVALID_ARG;
    return aligned_to(targets, index == SDL_INDEX_INT64 ? 8 : 4) ? SDL_OK : SDL_ERR_ALIGNMENT;
}

// The gradient may lie in the logits' place, with their strides.
int check_gradient(const sdl_view_t* d, const sdl_view_t* x, sdl_dtype_t dtype, uint32_t batch, uint32_t tokens)
{
    const int rc = check_output(d, dtype, batch, tokens, 1);
    if (rc != SDL_OK) return rc;
    return d->data == x->data && ((batch > 1 && d->stride_batch != x->stride_batch) || (tokens > 1 && d->stride_token != x->stride_token)) ? SDL_ERR_INVALID_ARG
                                                                                                                                        : SDL_OK;
}

LossArgs arguments(const sdl_view_t* logits, const sdl_view_t* d_logits, uint32_t batch, uint32_t tokens, uint32_t vocab, const void* targets, sdl_index_t index,
                   float smoothing, float z, const float* d_loss)
{
    return LossArgs{kernel_view(logits), d_logits ? kernel_view(d_logits) : View{}, targets, d_loss, nullptr, nullptr, make_div(tokens), batch * tokens, vocab,
                    index == SDL_INDEX_INT64, smoothing, 1.0f - smoothing, smoothing / (float)vocab, z};
}

}  // namespace

extern "C" {

int sdl_cross_entropy(const sdl_view_t* logits, uint32_t batch, uint32_t tokens, uint32_t vocab, sdl_dtype_t dtype, const void* targets, sdl_index_t index,
                      float smoothing, float z, float* loss_out, float* lse, const float* d_loss, const sdl_view_t* d_logits, void* stream)
{
    int rc = check(logits, batch, tokens, vocab, dtype, targets, index, smoothing, z);
    if (rc != SDL_OK || batch == 0 || tokens == 0) return rc;
    if (!loss_out && !lse && !d_logits) return SDL_ERR_INVALID_ARG;
    if (d_logits && (rc = check_gradient(d_logits, logits, dtype, batch, tokens)) != SDL_OK) return rc;
    if (!aligned_to(loss_out, 4) || !aligned_to(lse, 4) || !aligned_to(d_loss, 4)) return SDL_ERR_ALIGNMENT;
    LossArgs a = arguments(logits, d_logits, batch, tokens, vocab, targets, index, smoothing, z, d_loss);
    a.loss = loss_out;
    a.lse = lse;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == SDL_DTYPE_BF16 ? loss<__bf16>(a, st) : loss<float>(a, st);
}

int sdl_cross_entropy_backward(const sdl_view_t* logits, uint32_t batch, uint32_t tokens, uint32_t vocab, sdl_dtype_t dtype, const void* targets, sdl_index_t index,
                               float smoothing, float z, const float* lse, const float* d_loss, const sdl_view_t* d_logits, void* stream)
{
    int rc = check(logits, batch, tokens, vocab, dtype, targets, index, smoothing, z);
    if (rc != SDL_OK || batch == 0 || tokens == 0) return rc;
    if (!lse) return SDL_ERR_INVALID_ARG;
    if ((rc = check_gradient(d_logits, logits, dtype, batch, tokens)) != SDL_OK) return rc;
    if (!aligned_to(lse, 4) || !aligned_to(d_loss, 4)) return SDL_ERR_ALIGNMENT;
    LossArgs a = arguments(logits, d_logits, batch, tokens, vocab, targets, index, smoothing, z, d_loss);
    a.lse = const_cast<float*>(lse);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == SDL_DTYPE_BF16 ? gradient<__bf16>(a, st) : gradient<float>(a, st);
}

}  // extern "C"
