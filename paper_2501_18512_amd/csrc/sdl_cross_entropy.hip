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

// Maximum, sum of exp(x - maximum), and sum of x of some of a row's elements.
struct Part {
    float m, s, sum;
};

// A part of nothing but -infinity has s = 0.
__device__ __forceinline__ Part join(const Part& a, const Part& b)
{
    const float m = fmaxf(a.m, b.m);
    const float base = m == -__builtin_inff() ? 0.0f : m;
    return Part{m, a.s * exp_under(a.m, base) + b.s * exp_under(b.m, base), a.sum + b.sum};
}

__device__ __forceinline__ float wave_max(float x)
{
    x = fmaxf(x, dpp<0xb1>(x));
    x = fmaxf(x, dpp<0x4e>(x));
    x = fmaxf(x, dpp<0x141>(x));
    x = fmaxf(x, dpp<0x140>(x));
    u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(f2u(x), f2u(x), false, false));
    x = fmaxf(u2f(p[0]), u2f(p[1]));
    p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(f2u(x), f2u(x), false, false));
    return fmaxf(u2f(p[0]), u2f(p[1]));
}

// The lanes' parts as one, in all of them.
__device__ __forceinline__ Part wave_join(const Part& p, bool smooth)
{
    const float m = wave_max(p.m), base = m == -__builtin_inff() ? 0.0f : m;
    return Part{m, lane_sum<kWave>(p.s * exp_under(p.m, base)), smooth ? lane_sum<kWave>(p.sum) : 0.0f};
}

// The same bits, for the compiler others, that it has when `now` is worked out: else it would keep eight numbers instead of the four words that they come in, for all that
// a thread holds (104 registers instead of 70 for eight groups, and memory for sixteen).
__device__ __forceinline__ void forget(Eight<__bf16>& e, float& now) { asm volatile("" : "+v"(e.w), "+v"(now)); }
__device__ __forceinline__ void forget(Eight<float>&, float&) {}

// A row of n elements in groups of eight that start on 16 bytes: group g stands for [8 g - lead, 8 g - lead + 8).  The first and the last, which may stick out, are the eight
// elements at the row's end instead, so that others' are among them too: those are not counted, and what two threads write to one place is the same.  All of a thread's accesses are
// whole ones that wait for nothing.  Rows of 32001 in bf16 instead of 32000: 219 us with groups that start with the row, 179 so.  (TINY rows, which may have less than eight
// elements, go element by element.)
template <bool TINY>
struct Groups {
    uint32_t n;
    int32_t lead;

    template <typename T>
    __device__ __forceinline__ Groups(uint32_t n_, const T* row) : n(n_), lead(TINY ? 0 : (int32_t)((uintptr_t)row % 16 / sizeof(T))) {}
    __device__ __forceinline__ bool there(uint32_t first) const { return first < n + lead; }      // first = 8 g
    __device__ __forceinline__ uint32_t from(uint32_t first) const
    {
        return TINY ? first : (uint32_t)min(max((int32_t)first - lead, 0), (int32_t)n - 8);
    }
    // whether the j-th element from from(first) on is the group's
    __device__ __forceinline__ bool has(uint32_t first, int j) const
    {
        return TINY ? first + j < n : from(first) + j + lead - first < 8;
    }
    // whether a group that this thread, whose first one is 8 g, has of every TPR touches the element
    template <int TPR>
    __device__ __forceinline__ bool touches(uint32_t first, uint32_t element) const
    {
        const uint32_t own = first / 8;
        if (TINY) return element / 8 % TPR == own;
        return (element + lead) / 8 % TPR == own || (element < 8 && own == 0) || (element >= n - 8 && (n - 1 + lead) / 8 % TPR == own);
    }
    template <typename T>
    __device__ __forceinline__ Eight<T> load(const T* row, uint32_t first) const;
    template <typename T>
    __device__ __forceinline__ void store(T* row, uint32_t first, const float* v) const;
};

// In bf16, where an access of a wavefront's is whole cache lines, rows go past the caches: 8192 of 32000 with their gradient 195 us with cached accesses, 179 so; 256 of them 10.4
// and 9.0.  In fp32 it is two halves of every 32 bytes: 4096 rows 203 us and 216, 1551 of 5003 13.0 and 16.1.
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));

template <bool TINY>
template <typename T>
__device__ __forceinline__ Eight<T> Groups<TINY>::load(const T* row, uint32_t first) const
{
    if constexpr (TINY) {
        const T low = (T)-__builtin_inff();
        T v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = first + j < n ? row[first + j] : low;
        return __builtin_bit_cast(Eight<T>, v);
    } else if constexpr (sizeof(T) == 2) {
        const u32x4_at2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_at2*>(row + from(first)));
        return Eight<T>{u32x4{w.x, w.y, w.z, w.w}};
    } else {
        return load8(row, from(first), ~0u);
    }
}

template <bool TINY>
template <typename T>
__device__ __forceinline__ void Groups<TINY>::store(T* row, uint32_t first, const float* v) const
{
    if constexpr (TINY) {
        store8(row, first, n, v);
    } else if constexpr (sizeof(T) == 2) {
        const u32x4_at2 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4_at2*>(row + from(first)));
    } else {
        store8(row, from(first), ~0u, v);
    }
}

// What K groups of eight elements, TPR groups apart, are as a part of their row.  No branch goes by an element: a thread's groups stay in the words they came in.
template <bool TINY, typename T, int K, int TPR>
__device__ __forceinline__ Part part_of(Eight<T> (&e)[K], uint32_t first, const Groups<TINY>& groups, bool smooth)
{
    Part p{-__builtin_inff(), 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float m = e[k].get(0);
#pragma unroll
        for (int j = 1; j < 8; ++j) m = fmaxf(m, e[k].get(j));
        p.m = fmaxf(p.m, m);
        forget(e[k], p.m);
    }
    const float base = p.m == -__builtin_inff() ? 0.0f : p.m;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = groups.has(first + k * TPR * 8, j) ? exp_under(e[k].get(j), base) : 0.0f;
        p.s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        forget(e[k], p.s);
    }
    if (smooth) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += groups.has(first + k * TPR * 8, j) ? e[k].get(j) : 0.0f;
            p.sum += sum;
            forget(e[k], p.sum);
        }
    }
    return p;
}

// What a row's gradient is made of: factor exp(x - m) - even, and `hit` less at the target.
struct Slope {
    float m, factor, even, hit;
};

template <bool TINY, typename T, int K, int TPR>
__device__ __forceinline__ void write_gradient(T* row, uint32_t first, const Groups<TINY>& groups, Eight<T> (&e)[K], const Slope& g)
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = g.factor * exp_under(e[k].get(j), g.m) - g.even;
        if (groups.there(first + k * TPR * 8)) groups.store(row, first + k * TPR * 8, v);
    }
}

// The target's element, once more by every thread that has written it: a wavefront's stores to one place keep their order.
template <bool TINY, typename T, int TPR>
__device__ __forceinline__ void write_target(T* row, uint32_t first, const Groups<TINY>& groups, int32_t target, float x, const Slope& g)
{
    if (groups.template touches<TPR>(first, (uint32_t)target)) row[target] = (T)(g.factor * exp_under(x, g.m) - g.even - g.hit);
}

template <bool TINY, typename T, int TPR>
__device__ __forceinline__ void write_zeros(T* row, uint32_t first, const Groups<TINY>& groups)
{
    const float zero[8] = {};
    for (uint32_t at = first; groups.there(at); at += TPR * 8) groups.store(row, at, zero);
}

// TPR threads a row, K groups of eight elements each; FIT: a row is that long at most and stays in the registers, else it is read again for its gradient.
template <typename T, int BLOCK, int TPR, int K, bool FIT, bool TINY = false>
__global__ void __launch_bounds__(BLOCK) sdl_cross_entropy_kernel(const LossArgs a)
{
    constexpr int kWaves = TPR / kWave;
    static_assert(TPR == kWave || TPR == BLOCK, "a row is a wavefront's or a workgroup's");
    const uint32_t row = TPR == BLOCK ? workgroup() : workgroup() * (BLOCK / TPR) + threadIdx.x / TPR, n = a.vocab;
    uint32_t first = threadIdx.x % TPR * 8;
    if (row >= a.rows) return;
    const int32_t target = target_of(a, row);
    T* d = a.d.data ? row_of<T>(a, a.d, row) : nullptr;
    if (target < 0) {
        if (threadIdx.x % TPR == 0) {
            if (a.loss) a.loss[row] = 0.0f;
            if (a.lse) a.lse[row] = 0.0f;
        }
        if (d) write_zeros<TINY, T, TPR>(d, first, Groups<TINY>(n, d));
        return;
    }
    const T* x = row_of<const T>(a, a.x, row);
    const bool smooth = a.smoothing > 0.0f;
    const float at_target = (float)x[target], g = d && a.d_loss ? a.d_loss[row] : 1.0f;
    const Groups<TINY> groups(n, d ? d : x);
    Eight<T> e[K];
    Part p{-__builtin_inff(), 0.0f, 0.0f};
    if constexpr (FIT) {
#pragma unroll
        for (int k = 0; k < K; ++k) e[k] = groups.load(x, first + k * TPR * 8);
        p = part_of<TINY, T, K, TPR>(e, first, groups, smooth);
    } else {
        for (uint32_t at = first; groups.there(at); at += TPR * 8 * K) {
#pragma unroll
            for (int k = 0; k < K; ++k) e[k] = groups.load(x, at + k * TPR * 8);
            p = join(p, part_of<TINY, T, K, TPR>(e, at, groups, smooth));
        }
    }
    p = wave_join(p, smooth);
    // all of the row is read before any of it is written, which may be in its place
    asm volatile("" : : "v"(at_target) : "memory");
    if constexpr (kWaves > 1) {
        __shared__ Part parts[kWaves];
        if (threadIdx.x % kWave == 0) parts[threadIdx.x / kWave] = p;
        __syncthreads();
        p = parts[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) p = join(p, parts[w]);
    }
    const float log_s = logf(p.s), lse = p.m + log_s;
    if (threadIdx.x % TPR == 0) {
        float loss = log_s + a.hit * (p.m - at_target);
        if (smooth) loss += a.smoothing * (p.m - p.sum / (float)n);
        if (a.z != 0.0f) loss += a.z * lse * lse;
        if (a.loss) a.loss[row] = loss;
        if (a.lse) a.lse[row] = lse;
    }
    if (!d) return;
    const Slope slope{p.m, g * (1.0f + 2.0f * a.z * lse) / p.s, g * a.share, g * a.hit};
    asm volatile("" : "+v"(first));         // places are worked out again, and not kept
    if constexpr (FIT) {
        write_gradient<TINY, T, K, TPR>(d, first, groups, e, slope);
    } else {
        for (uint32_t at = first; groups.there(at); at += TPR * 8 * K) {
#pragma unroll
            for (int k = 0; k < K; ++k) e[k] = groups.load(x, at + k * TPR * 8);
            write_gradient<TINY, T, K, TPR>(d, at, groups, e, slope);
        }
    }
    write_target<TINY, T, TPR>(d, first, groups, target, at_target, slope);
}

// The gradient alone, from the forward pass' lse.
template <typename T, int BLOCK, int TPR, int K, bool TINY>
__global__ void __launch_bounds__(BLOCK) sdl_cross_entropy_backward_kernel(const LossArgs a)
{
    const uint32_t row = TPR == BLOCK ? workgroup() : workgroup() * (BLOCK / TPR) + threadIdx.x / TPR, n = a.vocab;
    uint32_t first = threadIdx.x % TPR * 8;
    if (row >= a.rows) return;
    const int32_t target = target_of(a, row);
    T* d = row_of<T>(a, a.d, row);
    if (target < 0) {
        write_zeros<TINY, T, TPR>(d, first, Groups<TINY>(n, d));
        return;
    }
    const T* x = row_of<const T>(a, a.x, row);
    const float at_target = (float)x[target], lse = a.lse[row], g = a.d_loss ? a.d_loss[row] : 1.0f;
    const Groups<TINY> groups(n, d);
    const Slope slope{lse, g * (1.0f + 2.0f * a.z * lse), g * a.share, g * a.hit};
    for (uint32_t at = first; groups.there(at); at += TPR * 8 * K) {
        Eight<T> e[K];
#pragma unroll
        for (int k = 0; k < K; ++k) e[k] = groups.load(x, at + k * TPR * 8);
        write_gradient<TINY, T, K, TPR>(d, at, groups, e, slope);
    }
    write_target<TINY, T, TPR>(d, first, groups, target, at_target, slope);
}

template <typename T>
int loss(const LossArgs& a, hipStream_t st)
{
    const uint32_t V = a.vocab;
#define SDL_LAUNCH(BLOCK, TPR, K, ...) \
    hipLaunchKernelGGL((sdl_cross_entropy_kernel<T, BLOCK, TPR, K, __VA_ARGS__>), grid_of((a.rows - 1) / (BLOCK / TPR) + 1), dim3(BLOCK), 0, st, a)
    const View& rows = a.d.data ? a.d : a.x;
    const bool even = aligned_to(rows.data, 16) && rows.batch * (int64_t)sizeof(T) % 16 == 0 && rows.token * (int64_t)sizeof(T) % 16 == 0;
    const uint32_t room = even ? V : V + 7;         // a row's groups are one more where it does not start on 16 bytes
    if (V <= 512) SDL_LAUNCH(256, 64, 1, true, true);
    else if (room <= 1024) SDL_LAUNCH(256, 64, 2, true);
    else if (room <= 2048) SDL_LAUNCH(256, 64, 4, true);
    else if (room <= 4096) SDL_LAUNCH(256, 256, 2, true);
    else if (room <= 8192) SDL_LAUNCH(256, 256, 4, true);
    else if (room <= 16384) SDL_LAUNCH(512, 512, 4, true);
    // without a gradient, fewer threads a row and more rows at a time: 8192 of 32000, half of them without a target, 51.7 us with 512 and 47.1 with 256; with one 179 and 185
    else if (room <= 32768 && !a.d.data) SDL_LAUNCH(256, 256, 16, true);
    else if (room <= 32768) SDL_LAUNCH(512, 512, 8, true);
    else if (room <= 65536) SDL_LAUNCH(512, 512, 16, true);
    else {
        if constexpr (sizeof(T) == 2) {
            if (room <= 131072) {
                SDL_LAUNCH(1024, 1024, 16, true);
                return launched();
            }
        }
        SDL_LAUNCH(1024, 1024, 4, false);
    }
#undef SDL_LAUNCH
    return launched();
}

template <typename T>
int gradient(const LossArgs& a, hipStream_t st)
{
#define SDL_LAUNCH(TPR, K, TINY) \
    hipLaunchKernelGGL((sdl_cross_entropy_backward_kernel<T, 256, TPR, K, TINY>), grid_of((a.rows - 1) / (256 / TPR) + 1), dim3(256), 0, st, a)
    if (a.vocab <= 512) SDL_LAUNCH(64, 1, true);
    else if (a.vocab <= 2048) SDL_LAUNCH(64, 2, false);
    else SDL_LAUNCH(256, 4, false);
#undef SDL_LAUNCH
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
