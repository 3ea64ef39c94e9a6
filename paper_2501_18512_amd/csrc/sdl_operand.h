// What the operators of the inner step share (gfx950): element types, strided views, loads and stores of
// eight elements at any alignment, sums over the lanes that hold one row, division by a fixed number.
// Internal to csrc/; nothing here is part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "sdl.h"
#include "sdl_device.h"

namespace sdl_device {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// A view as a kernel takes it: element strides of a [batch][token][head][width] array, unit stride within a row.
struct View {
    char* data;
    int64_t batch, token, head;
};

// n / d for n < 2^31 by one multiplication (T. Granlund, P. L. Montgomery, Division by invariant integers using multiplication, 1994): with 2^l the least power of two >= d, n/d = (floor(m n / 2^32) + n) >> l
// for m = floor(2^32 (2^l - d) / d) + 1.
struct Div {
    uint32_t m, l, d;
};

inline Div make_div(uint32_t d)
{
    uint32_t l = 0;
    while (l < 32 && ((uint64_t)1 << l) < d) ++l;
    return Div{(uint32_t)((((((uint64_t)1 << l) - d) << 32) / d) + 1), l, d};
}

__device__ __forceinline__ uint32_t div(uint32_t n, const Div& d) { return (__umulhi(d.m, n) + n) >> d.l; }

template <typename T> __device__ __forceinline__ float to_f32(T x) { return (float)x; }

// Eight consecutive elements as they lie in memory.
template <typename T> struct Eight;
template <> struct Eight<__bf16> {
    u32x4 w;
    __device__ __forceinline__ float get(int j) const { return u2f((j & 1) ? (w[j / 2] & 0xffff0000u) : (w[j / 2] << 16)); }
};
template <> struct Eight<float> {
    u32x4 lo, hi;
    __device__ __forceinline__ float get(int j) const { return u2f(j < 4 ? lo[j & 3] : hi[j & 3]); }
};

// Elements [at, at + 8) of a row of n: those from n on are zero and are not read.  Whole groups go through 128-bit
// accesses of element alignment.
__device__ __forceinline__ Eight<__bf16> load8(const __bf16* row, uint32_t at, uint32_t n)
{
    Eight<__bf16> r;
    if (at + 8 <= n) {
        const u32x4_bf16elem x = *reinterpret_cast<const u32x4_bf16elem*>(row + at);
        r.w = u32x4{x.x, x.y, x.z, x.w};
        return r;
    }
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
    uint32_t h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = at + j < n ? p[at + j] : 0u;
    r.w = u32x4{h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16)};
    return r;
}

__device__ __forceinline__ Eight<float> load8(const float* row, uint32_t at, uint32_t n)
{
    Eight<float> r;
    if (at + 8 <= n) {
        const u32x4_f32elem* p = reinterpret_cast<const u32x4_f32elem*>(row + at);
        const u32x4_f32elem a = p[0], b = p[1];
        r.lo = u32x4{a.x, a.y, a.z, a.w};
        r.hi = u32x4{b.x, b.y, b.z, b.w};
        return r;
    }
    const uint32_t* p = reinterpret_cast<const uint32_t*>(row);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        r.lo[j] = at + j < n ? p[at + j] : 0u;
        r.hi[j] = at + 4 + j < n ? p[at + 4 + j] : 0u;
    }
    return r;
}

// The same for rows of eight elements and more, whose last ones come in one access that ends with the row and are moved into place: attention at widths
// that are no multiple of eight, 4 causal sequences of 1024 tokens, 16 heads of 100 in bf16, forward 136 -> 87 us and backward 260 -> 189.  In fp32 an element is an
// access of its own width.
__device__ __forceinline__ Eight<__bf16> load8_ends(const __bf16* row, uint32_t at, uint32_t n)
{
    if (n < 8) return load8(row, at, n);
    const uint32_t from = at + 8 <= n ? at : n - 8, by = at - from;         // elements to be dropped; all of them from eight on
    const u32x4_bf16elem x = *reinterpret_cast<const u32x4_bf16elem*>(row + from);
    u32x4 w = u32x4{x.x, x.y, x.z, x.w};
    if (by) {
        if (by & 1) w = u32x4{(w.x >> 16) | (w.y << 16), (w.y >> 16) | (w.z << 16), (w.z >> 16) | (w.w << 16), w.w >> 16};
        if (by & 2) w = u32x4{w.y, w.z, w.w, 0};
        if (by & 4) w = u32x4{w.z, w.w, 0, 0};
        if (by >= 8) w = u32x4{0, 0, 0, 0};
    }
    return Eight<__bf16>{w};
}
__device__ __forceinline__ Eight<float> load8_ends(const float* row, uint32_t at, uint32_t n) { return load8(row, at, n); }

// The same where n is a multiple of eight: far less code, which a kernel that runs for a few microseconds has to fetch.
template <bool WHOLE, typename T>
__device__ __forceinline__ Eight<T> load_eight(const T* row, uint32_t at, uint32_t n)
{
    if constexpr (WHOLE) {
        if (at >= n) return Eight<T>{};
        n = at + 8;
    }
    return load8(row, at, n);
}

// two fp32 -> two bf16 (round to nearest even) in one word, first value in the low half
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

__device__ __forceinline__ void store8(__bf16* row, uint32_t at, uint32_t n, const float* v)
{
    const uint32_t w[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    if (at + 8 <= n) {
        *reinterpret_cast<u32x4_bf16elem*>(row + at) = u32x4_bf16elem{w[0], w[1], w[2], w[3]};
        return;
    }
    uint16_t* p = reinterpret_cast<uint16_t*>(row);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (at + j < n) p[at + j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
}

__device__ __forceinline__ void store8(float* row, uint32_t at, uint32_t n, const float* v)
{
    if (at + 8 <= n) {
        u32x4_f32elem* p = reinterpret_cast<u32x4_f32elem*>(row + at);
        p[0] = u32x4_f32elem{f2u(v[0]), f2u(v[1]), f2u(v[2]), f2u(v[3])};
        p[1] = u32x4_f32elem{f2u(v[4]), f2u(v[5]), f2u(v[6]), f2u(v[7])};
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (at + j < n) row[at + j] = v[j];
}

// A launch takes less than 2^32 threads along x.  Workgroups are numbered through rows of kGridX of them (a multiple of the dies, and 2^31 threads at 1024 each); those of the last
// row that are too many have nothing to do.
constexpr uint32_t kGridX = 1u << 21;
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * kGridX + blockIdx.x; }
inline dim3 grid_of(uint64_t groups) { return groups <= kGridX ? dim3((uint32_t)groups) : dim3(kGridX, (uint32_t)((groups + kGridX - 1) / kGridX)); }

template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return u2f((uint32_t)__builtin_amdgcn_update_dpp(0, (int)f2u(x), CTRL, 0xf, 0xf, true));
}

// Sum over the N neighbouring lanes that hold one row (N a power of two from 8 to 64); every one of them gets it.
template <int N>
__device__ __forceinline__ float lane_sum(float x)
{
    x += dpp<0xb1>(x);                                  // lane ^ 1
    x += dpp<0x4e>(x);                                  // lane ^ 2
    x += dpp<0x141>(x);                                 // the other four of eight
    if constexpr (N >= 16) x += dpp<0x140>(x);          // the other eight of sixteen
    if constexpr (N >= 32) {
        const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(f2u(x), f2u(x), false, false));
        const uint32_t a = p.x, b = p.y;
        x = u2f(a) + u2f(b);
    }
    if constexpr (N >= 64) {
        const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(f2u(x), f2u(x), false, false));
        const uint32_t a = p.x, b = p.y;
        x = u2f(a) + u2f(b);
    }
    return x;
}

// The sum of the lanes up to and including this one, over a whole wavefront.
__device__ __forceinline__ uint32_t lane_scan(uint32_t x)
{
#define SDL_SCAN(CTRL, ROWS) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false)
    SDL_SCAN(0x111, 0xf);       // from one lane down in a row of 16, then 2, 4, 8
    SDL_SCAN(0x112, 0xf);
    SDL_SCAN(0x114, 0xf);
    SDL_SCAN(0x118, 0xf);
    SDL_SCAN(0x142, 0xa);       // the last of rows 0 and 2 to rows 1 and 3
    SDL_SCAN(0x143, 0xc);       // the last of row 1 to rows 2 and 3
#undef SDL_SCAN
    return x;
}

// ------------------------------------------------------------------------------------------------- host side

inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline size_t dtype_size(sdl_dtype_t t) { return t == SDL_DTYPE_BF16 ? 2 : 4; }
inline bool known(sdl_dtype_t t) { return t == SDL_DTYPE_FP32 || t == SDL_DTYPE_BF16; }

inline int check_view(const sdl_view_t* v, sdl_dtype_t t)
{
    if (!v || !v->data) return SDL_ERR_INVALID_ARG;
    return aligned_to(v->data, dtype_size(t)) ? SDL_OK : SDL_ERR_ALIGNMENT;
}

// An array that a call writes: no two rows of it may be one.
inline int check_output(const sdl_view_t* v, sdl_dtype_t t, uint64_t batch, uint64_t tokens, uint64_t heads)
{
    const int rc = check_view(v, t);
    if (rc != SDL_OK) return rc;
    if ((batch > 1 && v->stride_batch == 0) || (tokens > 1 && v->stride_token == 0) || (heads > 1 && v->stride_head == 0)) return SDL_ERR_INVALID_ARG;
    return SDL_OK;
}

inline View kernel_view(const sdl_view_t* v)
{
    return View{static_cast<char*>(v->data), v->stride_batch, v->stride_token, v->stride_head};
}

inline int launched() { return hipGetLastError() == hipSuccess ? SDL_OK : SDL_ERR_DEVICE; }

}  // namespace sdl_device
