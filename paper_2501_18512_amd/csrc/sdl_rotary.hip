// Rotary positions (gfx950): the pairs of the first R elements of every head are turned by position times frequency.
//
//   (a, b) -> s (a cos(p f_i) - b sin(p f_i), a sin(p f_i) + b cos(p f_i)),  i < R/2;  inverse: the angle's sign changes
//
// Memory bounds it: every element is read and written once.  A thread has eight pairs (i .. i+7) of one token and walks over heads, so that the
// angles, the dear part, are worked out once for them all.  An angle is held in turns in 64 bits until its whole turns are off: at position
// 10^5 an fp32 angle would be good to three digits.  What is left is a pair of fp32 numbers, so that the sines and cosines next to whole quarter turns keep their digits as well:
// error in fp32 (root mean square, 2048 positions, width 128) 5.6e-8 with the first of the two only and 4.5e-8 so, for 1 % of the time, 3 % in small fp32 calls.
//
// 8192 tokens of 32 heads of 128 in bf16 (134 MB): 24 us, 5.5 TB/s.  16 tokens of 20 heads: 4.2 us, of which the launch is 3 and the angles are the rest.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "sdl_operand.h"

namespace {

using namespace sdl_device;

struct RotaryArgs {
    View x, out;
    const int32_t* positions;       // [batch][tokens], or NULL: first + token
    const double* f;                // [R / 2] radians a position
    Div chunks, parts, tokens;      // thread -> (batch, token, share of the heads, eight pairs), the last fastest
    uint64_t n;
    uint32_t heads, heads_each, width, half;
    int32_t first;                  // counted on from in 64 bits
    float scale, sign;
};

template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(256) sdl_rotary_kernel(const RotaryArgs a)
{
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= a.n) return;
    uint32_t rest = div((uint32_t)id, a.chunks);
    const uint32_t chunk = (uint32_t)id - rest * a.chunks.d;
    uint32_t q = div(rest, a.parts);
    const uint32_t part = rest - q * a.parts.d;
    const uint32_t b = div(q, a.tokens), t = q - b * a.tokens.d;
    const uint32_t h0 = part * a.heads_each, h1 = h0 + a.heads_each < a.heads ? h0 + a.heads_each : a.heads;
    const T* x = reinterpret_cast<const T*>(a.x.data) + ((int64_t)b * a.x.batch + (int64_t)t * a.x.token);
    T* out = reinterpret_cast<T*>(a.out.data) + ((int64_t)b * a.out.batch + (int64_t)t * a.out.token);
    const uint32_t i0 = chunk * 8, R = 2 * a.half;
    if (i0 >= a.half) {             // behind the pairs: elements that stay
        const uint32_t at = R + (chunk - (a.half + 7) / 8) * 8;
        for (uint32_t h = h0; h < h1; ++h) {
            const Eight<T> v = load8(x + (int64_t)h * a.x.head, at, a.width);
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = v.get(j);
            store8(out + (int64_t)h * a.out.head, at, a.width, w);
        }
        return;
    }
    const double pos = a.positions ? (double)a.positions[(uint64_t)b * a.tokens.d + t] : (double)a.first + (double)t;
    float c[8], s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const double turns = pos * (i0 + j < a.half ? a.f[i0 + j] * 0.15915494309189535 : 0.0);
        const double rest = 2.0 * (turns - rint(turns));            // half turns, in [-1, 1]
        const float near = (float)rest, off = (float)(rest - (double)near) * 3.14159265f;
        float sj, cj;
        sincospif(near, &sj, &cj);
        // what the rounding of the angle to fp32 left out, at most 2^-25 of a half turn: the next terms are under 2^-47
        c[j] = __builtin_fmaf(-sj, off, cj) * a.scale;
        s[j] = __builtin_fmaf(cj, off, sj) * a.scale * a.sign;
    }
    for (uint32_t h = h0; h < h1; ++h) {
        const T* xr = x + (int64_t)h * a.x.head;
        T* yr = out + (int64_t)h * a.out.head;
        float u[8], v[8];
        if constexpr (INTERLEAVED) {
            const Eight<T> lo = load8(xr, 2 * i0, R), hi = load8(xr, 2 * i0 + 8, R);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = j < 4 ? lo.get(2 * j) : hi.get(2 * j - 8), r = j < 4 ? lo.get(2 * j + 1) : hi.get(2 * j - 7);
                float* to = j < 4 ? u + 2 * j : v + 2 * j - 8;
                to[0] = p * c[j] - r * s[j];
                to[1] = p * s[j] + r * c[j];
            }
            store8(yr, 2 * i0, R, u);
            store8(yr, 2 * i0 + 8, R, v);
        } else {
            const Eight<T> lo = load8(xr, i0, a.half), hi = load8(xr + a.half, i0, a.half);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = lo.get(j), r = hi.get(j);
                u[j] = p * c[j] - r * s[j];
                v[j] = p * s[j] + r * c[j];
            }
            store8(yr, i0, a.half, u);
            store8(yr + a.half, i0, a.half, v);
        }
    }
}

}  // namespace

extern "C" {

int sdl_rotary_frequencies(uint32_t rot, double base, sdl_rotary_scaling_t scaling, double factor, double low, double high,
                           uint32_t trained_length, double* out)
{
    if (!out || rot == 0 || (rot & 1u) || rot > SDL_ROTARY_MAX_WIDTH || !std::isfinite(base) || base <= 0.0) return SDL_ERR_INVALID_ARG;
    if (scaling != SDL_ROTARY_PLAIN && scaling != SDL_ROTARY_LINEAR && scaling != SDL_ROTARY_PARTS) return SDL_ERR_INVALID_ARG;
    if (scaling != SDL_ROTARY_PLAIN && (!std::isfinite(factor) || factor <= 0.0)) return SDL_ERR_INVALID_ARG;
    if (scaling == SDL_ROTARY_PARTS && (!std::isfinite(low) || !std::isfinite(high) || low < 0.0 || high <= low || trained_length == 0))
        return SDL_ERR_INVALID_ARG;
    for (uint32_t i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot);
        if (scaling == SDL_ROTARY_LINEAR) {
            f /= factor;
        } else if (scaling == SDL_ROTARY_PARTS) {
            const double turns = trained_length * f / 6.283185307179586;
            double keep = (turns - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f *= keep + (1.0 - keep) / factor;
        }
        out[i] = f;
    }
    return SDL_OK;
}

int sdl_rotary(const sdl_view_t* x, uint32_t batch, uint32_t tokens, uint32_t heads, uint32_t width, sdl_dtype_t dtype, uint32_t rot,
               sdl_rotary_layout_t layout, const int32_t* positions, int32_t first_position, const double* frequencies, float scale,
               int inverse, const sdl_view_t* out, void* stream)
{
    if (!known(dtype) || (layout != SDL_ROTARY_HALF && layout != SDL_ROTARY_INTERLEAVED)) return SDL_ERR_INVALID_ARG;
    if (width == 0 || (rot & 1u) || rot > width || !std::isfinite(scale)) return SDL_ERR_INVALID_ARG;
    if (width > SDL_ROTARY_MAX_WIDTH) return SDL_ERR_UNSUPPORTED;
    if (batch == 0 || tokens == 0 || heads == 0) return SDL_OK;
    int rc = check_view(x, dtype);
    if (rc != SDL_OK || (rc = check_output(out, dtype, batch, tokens, heads)) != SDL_OK) return rc;
    if (rot && !frequencies) return SDL_ERR_INVALID_ARG;
    if (!aligned_to(positions, 4) || !aligned_to(frequencies, 8)) return SDL_ERR_ALIGNMENT;
    const bool in_place = x->data == out->data;
    if (in_place && ((batch > 1 && x->stride_batch != out->stride_batch) || (tokens > 1 && x->stride_token != out->stride_token) ||
                     (heads > 1 && x->stride_head != out->stride_head)))
        return SDL_ERR_INVALID_ARG;
    RotaryArgs a{};
    a.half = rot / 2;
    // in place, the elements behind the pairs stay where they are
    const uint32_t chunks = (a.half + 7) / 8 + (in_place ? 0u : (width - rot + 7) / 8);
    if (chunks == 0) return SDL_OK;
    const uint64_t bt = (uint64_t)batch * tokens;
    // step by step: a product of all four may be a multiple of 2^64
    if (bt > 0x7fffffffu || bt * chunks > 0x7fffffffu || bt * chunks * heads > 0x7fffffffu) return SDL_ERR_UNSUPPORTED;
    // Heads a thread walks over: as many as leave 131,072 threads, a wavefront and more for every SIMD, and no more than eight of them up to four times as many: 4096
    // tokens of 8 heads of 128, two heads a thread 6.0 us and one 7.4 (the angles); 32,768 of 16, eight a thread 49 us and sixteen 53.
    uint64_t parts = (131072 + bt * chunks - 1) / (bt * chunks);
    while (heads > 8 * parts && bt * chunks * parts < 524288) parts *= 2;
    if (parts > heads) parts = heads;
    a.heads_each = (uint32_t)((heads + parts - 1) / parts);
    parts = (heads + a.heads_each - 1) / a.heads_each;
    a.x = kernel_view(x);
    a.out = kernel_view(out);
    a.positions = positions;
    a.f = frequencies;
    a.chunks = make_div(chunks);
    a.parts = make_div((uint32_t)parts);
    a.tokens = make_div(tokens);
    a.n = bt * chunks * parts;
    a.heads = heads;
    a.width = width;
    a.first = first_position;
    a.scale = scale;
    a.sign = inverse ? -1.0f : 1.0f;
    const dim3 grid((uint32_t)((a.n + 255) / 256)), block(256);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool half = layout == SDL_ROTARY_HALF;
    if (dtype == SDL_DTYPE_BF16) {
        if (half) hipLaunchKernelGGL((sdl_rotary_kernel<__bf16, false>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((sdl_rotary_kernel<__bf16, true>), grid, block, 0, st, a);
    } else {
        if (half) hipLaunchKernelGGL((sdl_rotary_kernel<float, false>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((sdl_rotary_kernel<float, true>), grid, block, 0, st, a);
    }
    return launched();
}

}  // extern "C"
