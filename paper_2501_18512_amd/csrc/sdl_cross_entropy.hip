// Cross entropy of logits with targets, and its gradient (gfx950).
//
// A row of logits is read once and stays in the registers of 64 to 1024 threads, its gradient is written once: both passes in one call move
// what one pass has to, and that is what bounds them: 8192 rows of 32000 in bf16 177 us, 5.9 TB/s, the loss alone 6.2.  An element costs one fused multiply-add and one exponential
// in each pass.  Every thread takes the maximum m of its elements and the sum s of exp(x - m) over them; two such pairs
// are one with M = max(m1, m2), s = s1 exp(m1 - M) + s2 exp(m2 - M), so that a row costs one exchange between its threads.  With M and s of the row,
//     lse = M + log s,   p = exp(x - M) / s
// and the loss is formed from M - x[target] and log s, which loses nothing where the target is nearly certain and lse and x[target] are nearly equal.
#include <cmath>

#include "sdl_operand.h"

namespace {

using namespace sdl_device;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct LossArgs {
    View x, d;
    const void* targets;
    const float* d_loss;
    float *loss, *lse;
    Div tokens;
    uint32_t rows, vocab, line;     // groups are counted from multiples of so many bytes
    bool wide;                      // targets of 64 bits
    float smoothing, hit, share, z; // hit = 1 - smoothing, share = smoothing / vocab
    float each;                     // a power of two, at most 1 / (2 vocab)
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

// What logits are taken as powers of two around m with: exp(x - m) = 2^(x log2(e) - from), one fused multiply-add and one exponential an element, and from = m log2(e) as it is rounded.
// That rounding has to be small, and m up to 2^21; around any other number nothing is lost but zeros (numbers so far down have none but those beside a number
// of 2^20, and rows of larger ones go another way, below).
struct Base {
    float from;
    bool near;
    __device__ __forceinline__ explicit Base(float m) : from(fabsf(m) <= 0x1p21f ? m * kLog2e : 0.0f), near(fabsf(m) <= 0x1p21f) {}
    __device__ __forceinline__ float exp(float x) const { return exp2_of(fmaf(x, kLog2e, -from)); }
    // what a sum of exp() around this is to be multiplied with for one around another, larger one
    __device__ __forceinline__ float into(const Base& to) const { return near && to.near ? exp2_of(from - to.from) : 1.0f; }
};

// Maximum, sum of exp() around it, and sum of x of some of a row's elements, of which each counts as x times a power of two: exact, and no sum of up to `vocab` of them
// leaves fp32 (logits that are masked with the lowest number).  A part of nothing but -infinity has s = 0.
struct Part {
    float m, s, sum;
};

__device__ __forceinline__ Part join(const Part& a, const Part& b)
{
    const float m = fmaxf(a.m, b.m);
    const Base to(m);
    return Part{m, a.s * Base(a.m).into(to) + b.s * Base(b.m).into(to), a.sum + b.sum};
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
    const float m = wave_max(p.m);
    const Base to(m);
    return Part{m, lane_sum<kWave>(p.s * Base(p.m).into(to)), smooth ? lane_sum<kWave>(p.sum) : 0.0f};
}

constexpr int kLine = 128;      // bytes of a cache's line

// 16 bytes from any element on
typedef uint32_t At __attribute__((ext_vector_type(4), aligned(2)));

// As many elements of a row as are 16 bytes: what one access of a thread's moves.
template <typename T>
struct Group {
    static constexpr int W = 16 / sizeof(T);
    u32x4 w;
    __device__ __forceinline__ float get(int j) const
    {
        if constexpr (sizeof(T) == 4) return u2f(w[j]);
        else return u2f(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
    }
    static __device__ __forceinline__ Group of(const float* v)
    {
        if constexpr (sizeof(T) == 4) return Group{u32x4{f2u(v[0]), f2u(v[1]), f2u(v[2]), f2u(v[3])}};
        else return Group{u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}};
    }
};

// The same bits, for the compiler others, that it has when `now` is worked out: else it would keep eight numbers instead of the four words that they come in, for all that
// a thread holds (104 registers instead of 70 for eight groups, and memory for sixteen); fp32 too is worked on in fewer registers so.
template <typename T>
__device__ __forceinline__ void forget(Group<T>& e, float& now)
{
    asm volatile("" : "+v"(e.w), "+v"(now));
}

// A row of n elements in groups of W that are counted from the cache line that it starts in, `lead` elements before it: group g stands for [W g - lead, W g - lead + W).  Those that
// stick out at either end are the W elements at that end instead, so that others' are among them too: those are not counted, and what two threads write to one place is the same.  All
// of a thread's accesses are whole ones that wait for nothing, and all of a wavefront's are whole lines.  8192 rows of 32001 in bf16: 219 us with groups that start with the row,
// 189 with groups on 16 bytes, 176 so, as long as rows of 32000.  (TINY rows, which may have less than W elements, go element by element.)
template <typename T, bool TINY>
struct Groups {
    static constexpr int W = Group<T>::W;
    uint32_t n;
    int32_t lead;

    __device__ __forceinline__ Groups(const LossArgs& a, const T* row) : n(a.vocab), lead(TINY ? 0 : (int32_t)(((uint32_t)(uintptr_t)row & (a.line - 1)) / sizeof(T))) {}
    __device__ __forceinline__ bool below(uint32_t first) const { return first < n + lead; }      // first = W g
    __device__ __forceinline__ bool there(uint32_t first) const { return below(first) && (TINY || first + W > (uint32_t)lead); }
    __device__ __forceinline__ uint32_t from(uint32_t first) const
    {
        return TINY ? first : (uint32_t)min(max((int32_t)first - lead, 0), (int32_t)n - W);
    }
    // whether a group is there as a whole and in its place
    __device__ __forceinline__ bool whole(uint32_t first) const { return !TINY && first >= (uint32_t)lead && first + W <= n + lead; }
    // whether the j-th element from from(first) on is the group's
    __device__ __forceinline__ bool has(uint32_t first, int j) const
    {
        return TINY ? first + j < n : from(first) + j + lead - first < W;
    }
    // whether a group that this thread, whose first one is W g, has of every TPR touches the element
    template <int TPR>
    __device__ __forceinline__ bool touches(uint32_t first, uint32_t element) const
    {
        const uint32_t own = first / W;
        if (TINY) return element / W % TPR == own;
        return (element + lead) / W % TPR == own || (element < W && own == (uint32_t)lead / W) || (element >= n - W && (n - 1 + lead) / W % TPR == own);
    }
    // Rows go past the caches: 8192 of 32000 in bf16 with their gradient 195 us with cached accesses, 179 so; 4096 in fp32 194 and 180.  (1551 of 5003 in fp32, which the
    // last cache holds: 11.8 and 13.0.)
    __device__ __forceinline__ Group<T> load(const T* row, uint32_t first) const
    {
        if constexpr (TINY) {
            const T low = (T)-__builtin_inff();
            T v[W];
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = first + j < n ? row[first + j] : low;
            return __builtin_bit_cast(Group<T>, v);
        } else {
            const At at = __builtin_nontemporal_load(reinterpret_cast<const At*>(row + from(first)));
            return Group<T>{u32x4{at.x, at.y, at.z, at.w}};
        }
    }
    __device__ __forceinline__ void store(T* row, uint32_t first, const float* v) const
    {
        if constexpr (TINY) {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (first + j < n) row[first + j] = (T)v[j];
        } else {
            const u32x4 w = Group<T>::of(v).w;
            __builtin_nontemporal_store(At{w.x, w.y, w.z, w.w}, reinterpret_cast<At*>(row + from(first)));
        }
    }
    // The same for no element but the group's, in their places.
    __device__ __forceinline__ Group<T> load_own(const T* row, uint32_t first) const
    {
        if (whole(first)) return load(row, first);
        T v[W];
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = first + j - lead < n ? row[first + j - lead] : (T)0.0f;
        return __builtin_bit_cast(Group<T>, v);
    }
    __device__ __forceinline__ void store_own(T* row, uint32_t first, const float* v) const
    {
        if (whole(first)) return store(row, first, v);
#pragma unroll
        for (int j = 0; j < W; ++j)
            if (first + j - lead < n) row[first + j - lead] = (T)v[j];
    }

};

template <int W>
__device__ __forceinline__ float sum_of(const float* v)
{
    float s = (v[0] + v[1]) + (v[2] + v[3]);
    if constexpr (W == 8) s += (v[4] + v[5]) + (v[6] + v[7]);
    return s;
}

// The same of v times a power of two.
template <int W>
__device__ __forceinline__ float sum_of(const float* v, float each)
{
    float s = fmaf(v[0], each, v[1] * each) + fmaf(v[2], each, v[3] * each);
    if constexpr (W == 8) s += fmaf(v[4], each, v[5] * each) + fmaf(v[6], each, v[7] * each);
    return s;
}

// What K groups of elements, TPR groups apart, are as a part of their row.  No branch goes by an element: a thread's groups stay in the words they came in.
template <bool FIT, bool TINY, typename T, int K, int TPR>
__device__ __forceinline__ Part part_of(Group<T> (&e)[K], uint32_t first, const Groups<T, TINY>& groups, bool smooth, float each)
{
    constexpr int W = Group<T>::W;
    Part p{-__builtin_inff(), 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float m = e[k].get(0);
#pragma unroll
        for (int j = 1; j < W; ++j) m = fmaxf(m, e[k].get(j));
        p.m = fmaxf(p.m, m);
        forget(e[k], p.m);
    }
    const Base base(p.m);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float v[W];
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = base.exp(e[k].get(j));
        // (a row that stays in the registers has half of the groups that its kernel has room for, but for seven elements)
        if ((!FIT || k == 0 || k + 1 >= K / 2) && !__all(groups.whole(first + k * TPR * W)))
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = groups.has(first + k * TPR * W, j) ? v[j] : 0.0f;
        p.s += sum_of<W>(v);
        forget(e[k], p.s);
    }
    if (smooth) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float v[W];
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = e[k].get(j);
            if ((!FIT || k == 0 || k + 1 >= K / 2) && !__all(groups.whole(first + k * TPR * W)))
#pragma unroll
                for (int j = 0; j < W; ++j) v[j] = groups.has(first + k * TPR * W, j) ? v[j] : 0.0f;
            p.sum += sum_of<W>(v, each);
            forget(e[k], p.sum);
        }
    }
    return p;
}

// What a row's gradient is made of: factor exp(x - m) - even, and `hit` less at the target.
struct Slope {
    float m, factor, even, hit;
};

// NEAR: the factor is one of exp() around the base.
template <bool NEAR>
__device__ __forceinline__ float slope_at(const Slope& g, const Base& base, float x)
{
    return fmaf(g.factor, NEAR ? base.exp(x) : exp_under(x, g.m), -g.even);
}

template <bool TINY, typename T, int K, int TPR>
__device__ __forceinline__ void write_gradient(T* row, uint32_t first, const Groups<T, TINY>& groups, Group<T> (&e)[K], const Slope& g)
{
    constexpr int W = Group<T>::W;
    const Base base(g.m);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float v[W];
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = slope_at<true>(g, base, e[k].get(j));
        if (groups.there(first + k * TPR * W)) groups.store(row, first + k * TPR * W, v);
    }
}

// The gradient of a row that is read for it, and may be written in its place: a group that sticks out reads and writes no one else's elements.
template <bool NEAR, bool TINY, typename T, int K, int TPR>
__device__ __forceinline__ void read_and_write_gradient(const T* x, T* d, uint32_t first, const Groups<T, TINY>& groups, int32_t target, const Slope& g)
{
    constexpr int W = Group<T>::W;
    const Base base(g.m);
    for (uint32_t at = first; groups.below(at); at += TPR * W * K) {
        Group<T> e[K];
#pragma unroll
        for (int k = 0; k < K; ++k) e[k] = groups.load_own(x, at + k * TPR * W);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t one = at + k * TPR * W;
            float v[W];
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = slope_at<NEAR>(g, base, e[k].get(j));
            if (((uint32_t)target + groups.lead) / W == one / W)
#pragma unroll
                for (int j = 0; j < W; ++j) v[j] -= (uint32_t)target + groups.lead == one + j ? g.hit : 0.0f;
            groups.store_own(d, one, v);
        }
    }
}

// The target's element, once more by every thread that has written it: a wavefront's stores to one place keep their order.
template <bool TINY, typename T, int TPR>
__device__ __forceinline__ void write_target(T* row, uint32_t first, const Groups<T, TINY>& groups, int32_t target, float x, const Slope& g)
{
    if (groups.template touches<TPR>(first, (uint32_t)target)) row[target] = (T)(slope_at<true>(g, Base(g.m), x) - g.hit);
}

template <bool TINY, typename T, int TPR>
__device__ __forceinline__ void write_zeros(T* row, uint32_t first, const Groups<T, TINY>& groups)
{
    constexpr int W = Group<T>::W;
    const float zero[W] = {};
    for (uint32_t at = first; groups.below(at); at += TPR * W)
        if (groups.there(at)) groups.store(row, at, zero);
}

// TPR threads a row, K groups of eight elements each; FIT: a row is that long at most and stays in the registers, else it is read again for its gradient.
template <typename T, int BLOCK, int TPR, int K, bool FIT, bool TINY = false>
__global__ void __launch_bounds__(BLOCK) sdl_cross_entropy_kernel(const LossArgs a)
{
    constexpr int kWaves = TPR / kWave, W = Group<T>::W;
    static_assert(TPR == kWave || TPR == BLOCK, "a row is a wavefront's or a workgroup's");
    const uint32_t row = TPR == BLOCK ? workgroup() : workgroup() * (BLOCK / TPR) + threadIdx.x / TPR, n = a.vocab;
    uint32_t first = threadIdx.x % TPR * W;
    if (row >= a.rows) return;
    const int32_t target = target_of(a, row);
    T* d = a.d.data ? row_of<T>(a, a.d, row) : nullptr;
    if (target < 0) {
        if (threadIdx.x % TPR == 0) {
            if (a.loss) a.loss[row] = 0.0f;
            if (a.lse) a.lse[row] = 0.0f;
        }
        if (d) write_zeros<TINY, T, TPR>(d, first, Groups<T, TINY>(a, d));
        return;
    }
    const T* x = row_of<const T>(a, a.x, row);
    const bool smooth = a.smoothing > 0.0f;
    const float at_target = (float)x[target], g = d && a.d_loss ? a.d_loss[row] : 1.0f;
    const Groups<T, TINY> groups(a, d ? d : x);
    Group<T> e[K];
    Part p{-__builtin_inff(), 0.0f, 0.0f};
    if constexpr (FIT) {
#pragma unroll
        for (int k = 0; k < K; ++k) e[k] = groups.load(x, first + k * TPR * W);
        p = part_of<FIT, TINY, T, K, TPR>(e, first, groups, smooth, a.each);
    } else {
        for (uint32_t at = first; groups.below(at); at += TPR * W * K) {
#pragma unroll
            for (int k = 0; k < K; ++k) e[k] = groups.load(x, at + k * TPR * W);
            p = join(p, part_of<FIT, TINY, T, K, TPR>(e, at, groups, smooth, a.each));
        }
    }
    p = wave_join(p, smooth);
    // all of the row is read before any of it is written, which may be in its place
    asm volatile("" : : "v"(at_target) : "memory");
    __shared__ Part parts[kWaves];
    if constexpr (kWaves > 1) {
        if (threadIdx.x % kWave == 0) parts[threadIdx.x / kWave] = p;
        __syncthreads();
        const uint32_t lane = threadIdx.x % kWave;
        p = wave_join(lane < kWaves ? parts[lane] : Part{-__builtin_inff(), 0.0f, 0.0f}, smooth);
    }
    // a row whose maximum is no number that the sums could be taken around: once more, by differences from it
    const bool far = fabsf(p.m) > 0x1p20f && fabsf(p.m) < __builtin_inff();
    if (far) {
        float s = 0.0f;
        for (uint32_t at = first; groups.below(at); at += TPR * W) {
            const Group<T> x8 = groups.load(x, at);
#pragma unroll
            for (int j = 0; j < W; ++j) s += groups.has(at, j) ? exp_under(x8.get(j), p.m) : 0.0f;
        }
        p.s = lane_sum<kWave>(s);
        if constexpr (kWaves > 1) {
            __syncthreads();
            if (threadIdx.x % kWave == 0) parts[threadIdx.x / kWave].s = p.s;
            __syncthreads();
            p.s = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) p.s += parts[w].s;
        }
    }
    const Base base(p.m);
    // log of the sum of exp(x - m): that of the sum around the base, less what the base's rounding has made of it
    const float log_s = logf(p.s) - (!far && base.near ? fmaf(p.m, kLog2e, -base.from) * kLn2 : 0.0f);
    const float lse = p.m == __builtin_inff() ? __builtin_nanf("") : p.m + log_s;
    if (threadIdx.x % TPR == 0) {
        // (an infinite logit counts as the mean's, if it counts as nothing else; differences by half, which have room for any two numbers)
        float loss = log_s + (a.hit > 0.0f ? 2.0f * (a.hit * (0.5f * p.m - 0.5f * at_target)) : 0.0f);
        if (smooth) loss += 2.0f * (a.smoothing * (0.5f * p.m - 0.5f * (p.sum / ((float)n * a.each))));
        if (a.z != 0.0f) loss += a.z * lse * lse;
        if (a.loss) a.loss[row] = p.m == __builtin_inff() ? lse : loss;
        if (a.lse) a.lse[row] = lse;
    }
    if (!d) return;
    const Slope slope{p.m, p.m == __builtin_inff() ? lse : g * (1.0f + 2.0f * a.z * lse) / p.s, g * a.share, g * a.hit};
    asm volatile("" : "+v"(first));         // places are worked out again, and not kept
    if (far) {
        read_and_write_gradient<false, TINY, T, 1, TPR>(x, d, first, groups, target, slope);
    } else if constexpr (FIT) {
        write_gradient<TINY, T, K, TPR>(d, first, groups, e, slope);
        write_target<TINY, T, TPR>(d, first, groups, target, at_target, slope);
    } else {
        read_and_write_gradient<true, TINY, T, K, TPR>(x, d, first, groups, target, slope);
    }
}

// The gradient alone, from the forward pass' lse: a row is read and written once, in rounds of which each waits for its loads, 8192 rows of 32000 in bf16 197 us, 5.3 TB/s.
template <typename T, int BLOCK, int TPR, int K, bool TINY>
__global__ void __launch_bounds__(BLOCK) sdl_cross_entropy_backward_kernel(const LossArgs a)
{
    constexpr int W = Group<T>::W;
    const uint32_t row = TPR == BLOCK ? workgroup() : workgroup() * (BLOCK / TPR) + threadIdx.x / TPR;
    uint32_t first = threadIdx.x % TPR * W;
    if (row >= a.rows) return;
    const int32_t target = target_of(a, row);
    T* d = row_of<T>(a, a.d, row);
    if (target < 0) {
        write_zeros<TINY, T, TPR>(d, first, Groups<T, TINY>(a, d));
        return;
    }
    const T* x = row_of<const T>(a, a.x, row);
    const float lse = a.lse[row], g = a.d_loss ? a.d_loss[row] : 1.0f;
    const Groups<T, TINY> groups(a, d);
    // around lse, with what its rounding makes of the base taken back; an infinite or far lse by differences
    if (fabsf(lse) <= 0x1p20f) {
        const Slope slope{lse, g * (1.0f + 2.0f * a.z * lse) * exp2_of(-fmaf(lse, kLog2e, -Base(lse).from)), g * a.share, g * a.hit};
        read_and_write_gradient<true, TINY, T, K, TPR>(x, d, first, groups, target, slope);
    } else {
        const Slope slope{lse, g * (1.0f + 2.0f * a.z * lse), g * a.share, g * a.hit};
        read_and_write_gradient<false, TINY, T, 1, TPR>(x, d, first, groups, target, slope);
    }
}

template <typename T>
int loss(LossArgs a, hipStream_t st)
{
    const View& rows = a.d.data ? a.d : a.x;
    const auto lie_on = [&](uint32_t line) {
        return aligned_to(rows.data, line) && rows.batch * (int64_t)sizeof(T) % line == 0 && rows.token * (int64_t)sizeof(T) % line == 0;
    };
    // the elements that a row's groups have room for, from a line on, or where that would take a longer kernel from 16 bytes on
    const uint32_t V = a.vocab, room = V + (lie_on(16) ? 0 : 16 / sizeof(T) - 1), room_line = V + (lie_on(kLine) ? 0 : kLine / sizeof(T) - 1);
#define SDL_LAUNCH(LIMIT, BLOCK, TPR, K, ...) \
    do { \
        a.line = room_line <= (LIMIT) ? kLine : 16; \
        hipLaunchKernelGGL((sdl_cross_entropy_kernel<T, BLOCK, TPR, (K) * (8 / Group<T>::W), __VA_ARGS__>), grid_of((a.rows - 1) / (BLOCK / TPR) + 1), dim3(BLOCK), 0, st, \
                           a); \
        return launched(); \
    } while (0)
#define SDL_FIT(LIMIT, BLOCK, TPR, K) \
    if (room <= (LIMIT)) SDL_LAUNCH(LIMIT, BLOCK, TPR, K, true)
    // Rows in as many threads as keep them in registers, and no more.  A wavefront: 65536 rows of 1000 in bf16 47 us, 256 threads 109; 32768 of 2000 45 and 60.  256 threads: 16384 of 4000
    // 43, a wavefront 45, 512 threads 57; of 8000 84 and 85.  512 threads: 8192 of 16000 86, 256 91, 1024 88; of 32000 178, 184 and 169, but the loss alone, half the rows without a
    // target, 42 and with 1024 threads 52; 6000 of 40000 166 and 163, 91 and 97.  1024 threads: 2048 of 131072 204, read a second time instead 272.
    constexpr uint32_t kLongest = sizeof(T) == 2 ? 512 : 1024;
    if (V <= 512) SDL_LAUNCH(512, 256, 64, 1, true, true);
    SDL_FIT(1024, 256, 64, 2);
    SDL_FIT(2048, 256, 64, 4);
    SDL_FIT(4096, 256, 256, 2);
    SDL_FIT(8192, 256, 256, 4);
    SDL_FIT(16384, 512, 512, 4);
    SDL_FIT(32768, 512, 512, 8);
    SDL_FIT(65536, kLongest, kLongest, 16 * 512 / kLongest);
    if constexpr (sizeof(T) == 2) SDL_FIT(131072, 1024, 1024, 16);
    SDL_LAUNCH(~0u, 1024, 1024, 4, false);
#undef SDL_FIT
#undef SDL_LAUNCH
}

template <typename T>
int gradient(LossArgs a, hipStream_t st)
{
    a.line = kLine;
#define SDL_LAUNCH(TPR, K, TINY) \
    hipLaunchKernelGGL((sdl_cross_entropy_backward_kernel<T, 256, TPR, (K) * (8 / Group<T>::W), TINY>), grid_of((a.rows - 1) / (256 / TPR) + 1), dim3(256), 0, st, a)
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
    return LossArgs{kernel_view(logits), d_logits ? kernel_view(d_logits) : View{}, targets, d_loss, nullptr, nullptr, make_div(tokens), batch * tokens, vocab, 16,
                    index == SDL_INDEX_INT64, smoothing, 1.0f - smoothing, smoothing / (float)vocab, z, std::ldexp(0.5f, -(int)make_div(vocab).l)};
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
