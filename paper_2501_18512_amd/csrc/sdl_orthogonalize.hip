// Orthogonalising matrices by Newton-Schulz steps (gfx950).
//
//     X = x / (norm(x) + eps),  then for every (a, b, c):  A = X X^T,  X = a X + (b A + c A^2) X
//
// works on X = U S V^T as U p(S) V^T with p(s) = a s + b s^3 + c s^5: no product moves the singular vectors.  Three products a step, of
// which A and A^2 are symmetric and only half is formed; they bound it.  A tall matrix is worked on as its transpose.
//
// The products run on fp16 matrix instructions with fp32 sums.  X lies within the unit ball (the coefficients are checked on the host), so a power of
// two keeps its elements in the middle of fp16's range: X 2^14, A 2^12, and b A + c A^2 by what its bound allows.
//   - X itself is kept in fp32 beside its fp16 image, and a X is taken from there.  What the images lose is then a factor near 1 on what a
//     direction already is: an error of X itself would be lifted with the small singular values, 3.4 times a step.
//   - results in bf16: one image, 11 bits.  An error of 2^-12 an element, 0.0003 to 0.0005 of the result after five steps, under the 0.0017 of its own rounding.
//   - results in fp32: two images, x 2^14 = hi + lo, 22 bits, and three products hi hi + hi lo + lo hi.  What is left out is 2^-24.
// An operand's rows are cut into pieces of 128 bytes, one step of a product's loop each: 64 elements, or 32 of hi and the same 32 of lo.
#include <algorithm>
#include <cmath>
#include <utility>

#include "sdl_operand.h"

namespace {

using namespace sdl_device;

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kScaleX = 16384.0f, kScaleA = 4096.0f;

// One matrix in the workspace, of which the next lies `each` bytes further.  Both sides are filled up with zeros to whole tiles.
struct Work {
    char* base;
    size_t each;
    size_t x32, x16, xt16, xt16_other, a16, b16;     // offsets
    uint32_t n, m;                                    // n <= m, filled up
    uint32_t split;
    __host__ __device__ uint32_t pitch(uint32_t k) const { return k * (split ? 4u : 2u); }     // bytes of a row of k elements of an image
};

// Image of v at element k of a row.
template <bool SPLIT>
__device__ __forceinline__ void put(char* row, uint32_t k, float v)
{
    const _Float16 hi = (_Float16)v;
    if constexpr (SPLIT) {
        char* at = row + (k / 32) * 128 + (k % 32) * 2;
        *reinterpret_cast<_Float16*>(at) = hi;
        *reinterpret_cast<_Float16*>(at + 64) = (_Float16)(v - (float)hi);
    } else {
        *reinterpret_cast<_Float16*>(row + k * 2) = hi;
    }
}
// N elements from k on, a multiple of N
template <bool SPLIT, int N>
__device__ __forceinline__ void put_many(char* row, uint32_t k, const float* v)
{
    typedef _Float16 vec __attribute__((ext_vector_type(N)));
    vec hi, lo;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        hi[i] = (_Float16)v[i];
        lo[i] = (_Float16)(v[i] - (float)hi[i]);
    }
    if constexpr (SPLIT) {
        char* at = row + (k / 32) * 128 + (k % 32) * 2;
        *reinterpret_cast<vec*>(at) = hi;
        *reinterpret_cast<vec*>(at + 64) = lo;
    } else {
        *reinterpret_cast<vec*>(row + k * 2) = hi;
    }
}
template <bool SPLIT>
__device__ __forceinline__ float take(const char* row, uint32_t k)
{
    if constexpr (SPLIT) {
        const char* at = row + (k / 32) * 128 + (k % 32) * 2;
        return (float)*reinterpret_cast<const _Float16*>(at) + (float)*reinterpret_cast<const _Float16*>(at + 64);
    } else {
        return (float)*reinterpret_cast<const _Float16*>(row + k * 2);
    }
}

// ------------------------------------------------------------------------------------------- norm, first images

struct FirstArgs {
    View x;                     // rows along `token`
    uint32_t rows, cols, tall, parts;
    double* squares;            // [matrix][parts]
    double eps;
    Work w;
};

// Sum of squares of a matrix' rows part, part + parts, ...: in 64 bits, in which no square of a 32-bit number is out of range.
template <typename T>
__global__ void __launch_bounds__(256) sdl_orthogonalize_norm_kernel(const FirstArgs a)
{
    __shared__ double sums[4];
    const uint32_t part = blockIdx.x, matrix = blockIdx.y;
    const T* x = reinterpret_cast<const T*>(a.x.data) + (int64_t)matrix * a.x.batch;
    const uint32_t groups = (a.cols + 7) / 8;
    // threads beyond a row's groups take further rows
    const uint32_t across = min(groups, 256u), down = 256 / across, r0 = threadIdx.x / across, g0 = threadIdx.x % across;
    double s = 0.0;
    if (r0 < down)
        for (uint32_t r = part * down + r0; r < a.rows; r += a.parts * down)
            for (uint32_t g = g0; g < groups; g += across) {
                const Eight<T> e = load8(x + (int64_t)r * a.x.token, g * 8, a.cols);
#pragma unroll
                for (int j = 0; j < 8; ++j) s += (double)e.get(j) * (double)e.get(j);
            }
#pragma unroll
    for (int k = 32; k; k /= 2) s += __shfl_xor(s, k);
    if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.squares[(size_t)matrix * a.parts + part] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// x over its norm, in fp32 and as images of both orders, in tiles of 64 by 64 of what the workspace holds.
template <typename T, bool SPLIT>
__global__ void __launch_bounds__(256) sdl_orthogonalize_first_kernel(const FirstArgs a)
{
    __shared__ float tile[64][65];
    __shared__ double inverse;
    const uint32_t matrix = blockIdx.z, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;      // of the n by m matrix
    if (threadIdx.x < kWave) {
        double s = 0.0;
        for (uint32_t p = threadIdx.x; p < a.parts; p += kWave) s += a.squares[(size_t)matrix * a.parts + p];
#pragma unroll
        for (int k = 32; k; k /= 2) s += __shfl_xor(s, k);
        const double norm = sqrt(s) + a.eps;
        if (threadIdx.x == 0) inverse = norm == 0.0 ? 0.0 : 1.0 / norm;
    }
    __syncthreads();
    const T* x = reinterpret_cast<const T*>(a.x.data) + (int64_t)matrix * a.x.batch;
    const uint32_t r0 = a.tall ? j0 : i0, c0 = a.tall ? i0 : j0;
    for (uint32_t i = threadIdx.x; i < 512; i += 256) {
        const uint32_t r = i / 8, c = i % 8 * 8;
        Eight<T> e{};
        if (r0 + r < a.rows && c0 + c < a.cols) e = load8(x + (int64_t)(r0 + r) * a.x.token, c0 + c, a.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = (float)((double)e.get(j) * inverse);
            if (a.tall) tile[c + j][r] = v;
            else tile[r][c + j] = v;
        }
    }
    __syncthreads();
    char* base = a.w.base + matrix * a.w.each;
    for (uint32_t i = threadIdx.x; i < 512; i += 256) {
        const uint32_t r = i / 8, c = i % 8 * 8;
        float v[8], s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = tile[r][c + j], s[j] = v[j] * kScaleX;
        store8(reinterpret_cast<float*>(base + a.w.x32) + (size_t)(i0 + r) * a.w.m + j0, c, c + 8, v);
        put_many<SPLIT, 8>(base + a.w.x16 + (size_t)(i0 + r) * a.w.pitch(a.w.m), j0 + c, s);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = tile[c + j][r] * kScaleX;
        put_many<SPLIT, 8>(base + a.w.xt16 + (size_t)(j0 + r) * a.w.pitch(a.w.n), i0 + c, s);
    }
}

// ----------------------------------------------------------------------------------------------------- products

enum { GRAM, POLY, UPDATE };

struct ProductArgs {
    Work w;
    size_t p, q, t;             // offsets of the two operands' images, and of what is written: images (UPDATE: of the transpose)
    uint32_t pitch_p, pitch_q, steps;
    Div tiles, across;          // of a matrix; UPDATE: along m
    float on_sum, on_old, image;    // result = on_old * old + on_sum * product; factor of its image
    // the last update: where to
    View out;
    uint32_t last, tall, rows, cols;
    float scale;
};

// 64 pieces of 16 bytes into shared memory, past the registers: they land one behind the other.  Five wait states between a vector instruction that writes a
// scalar register and the load that reads it, of which the write of m0 is one.
__device__ __forceinline__ void copy_pieces(const char* base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(to) : "memory");
}
__device__ __forceinline__ uint32_t lds_offset(const void* p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// TILE by TILE of C = P Q^T, both operands with k along their rows, by W by W wavefronts.  In shared memory a row's step is 128 bytes, its eight
// pieces swapped around by an xor with bits 1 to 3 of the row's number: neither the copies nor the reads (16 rows, one piece) meet in a bank.
// Two steps' tiles in turn: the next one's copies are under way while one is multiplied.
//
// Layouts of the 32x32x16 instruction, lane l, half = l / 32, c = l % 32:  A row c, k = 8 half + j;  B column c, k = 8 half + j;
// D column c, rows 8 (i / 4) + 4 half + i % 4.
template <int TILE, int W, bool SPLIT, int MODE, typename O>
__global__ void __launch_bounds__(W * W * kWave) sdl_orthogonalize_product_kernel(const ProductArgs a)
{
    constexpr int kBytes = TILE * 128, kSide = TILE / W, kParts = kSide / 32, kCopies = TILE / 8 / (W * W);
    static_assert(kParts * 32 == kSide && kCopies * 8 * W * W == TILE, "whole instructions");
    __shared__ __attribute__((aligned(128))) char lds[2][2][kBytes];
    const uint32_t lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), half = lane / 32, c = lane % 32;
    const uint32_t matrix = div(blockIdx.x, a.tiles), t = blockIdx.x - matrix * a.tiles.d;
    uint32_t ti, tj;
    if constexpr (MODE == UPDATE) {
        ti = div(t, a.across);
        tj = t - ti * a.across.d;
    } else {            // tiles on and under the diagonal, row by row
        ti = (uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while (ti * (ti + 1) / 2 > t) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
        ti = __builtin_amdgcn_readfirstlane(ti);
        tj = t - ti * (ti + 1) / 2;
    }
    char* base = a.w.base + matrix * a.w.each;
    const char* from_p = base + a.p + (size_t)(ti * TILE + wave * kCopies * 8) * a.pitch_p;
    const char* from_q = base + a.q + (size_t)(tj * TILE + wave * kCopies * 8) * a.pitch_q;
    // the piece that comes to lie where the lane's 16 bytes land, in the even instructions; 4 further, by xor, in the odd ones
    const uint32_t piece = ((lane % 8) ^ (lane / 16)) * 16;
    const uint32_t off_p = lane / 8 * a.pitch_p + piece, off_q = lane / 8 * a.pitch_q + piece;
    const auto bring = [&](uint32_t step) {
        const uint32_t to = lds_offset(lds[step % 2][0]) + wave * kCopies * 1024;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            // an instruction's parity is its number's: kCopies is even, or there is one wavefront's parity to count
            const uint32_t odd = ((wave * kCopies + i) & 1) * 64;
            copy_pieces(from_p + (size_t)i * 8 * a.pitch_p + step * 128, off_p ^ odd, to + i * 1024);
            copy_pieces(from_q + (size_t)i * 8 * a.pitch_q + step * 128, off_q ^ odd, to + kBytes + i * 1024);
        }
    };
    f32x16_t acc[kParts][kParts] = {};
    const uint32_t i0 = wave / W * kSide, j0 = wave % W * kSide, mix = (c >> 1) & 7;
    bring(0);
    for (uint32_t step = 0; step < a.steps; ++step) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
        if (step + 1 < a.steps) bring(step + 1);
        const char *rows_p = lds[step % 2][0] + (i0 + c) * 128, *rows_q = lds[step % 2][1] + (j0 + c) * 128;
        const auto frag = [&](const char* rows, int part, uint32_t p) {
            return *reinterpret_cast<const f16x8_t*>(rows + part * 4096 + ((p ^ mix) * 16));
        };
#pragma unroll
        for (int k = 0; k < (SPLIT ? 2 : 4); ++k) {
            f16x8_t p[kParts], q[kParts];
#pragma unroll
            for (int i = 0; i < kParts; ++i) p[i] = frag(rows_p, i, 2 * k + half), q[i] = frag(rows_q, i, 2 * k + half);
#pragma unroll
            for (int i = 0; i < kParts; ++i)
#pragma unroll
                for (int j = 0; j < kParts; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[i], q[j], acc[i][j], 0, 0, 0);
            if constexpr (SPLIT) {
                f16x8_t low[kParts];
#pragma unroll
                for (int j = 0; j < kParts; ++j) low[j] = frag(rows_q, j, 4 + 2 * k + half);
#pragma unroll
                for (int i = 0; i < kParts; ++i)
#pragma unroll
                    for (int j = 0; j < kParts; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[i], low[j], acc[i][j], 0, 0, 0);
#pragma unroll
                for (int i = 0; i < kParts; ++i) low[i] = frag(rows_p, i, 4 + 2 * k + half);
#pragma unroll
                for (int i = 0; i < kParts; ++i)
#pragma unroll
                    for (int j = 0; j < kParts; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(low[i], q[j], acc[i][j], 0, 0, 0);
            }
        }
    }
    const uint32_t n = a.w.n, m = a.w.m;
#pragma unroll
    for (int pi = 0; pi < kParts; ++pi)
#pragma unroll
        for (int pj = 0; pj < kParts; ++pj) {
            const uint32_t j = tj * TILE + j0 + pj * 32 + c;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t i = ti * TILE + i0 + pi * 32 + 8 * u + 4 * half;
                float v[4];
                if constexpr (MODE == GRAM) {
                    char* out = base + a.t;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        v[r] = acc[pi][pj][4 * u + r] * a.on_sum;
                        put<SPLIT>(out + (size_t)(i + r) * a.w.pitch(n), j, v[r]);
                    }
                    if (ti != tj) put_many<SPLIT, 4>(out + (size_t)j * a.w.pitch(n), i, v);
                } else if constexpr (MODE == POLY) {
                    char* out = base + a.t;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float old = take<SPLIT>(base + a.w.a16 + (size_t)(i + r) * a.w.pitch(n), j);
                        v[r] = (a.on_old * old + acc[pi][pj][4 * u + r] * a.on_sum) * a.image;
                        put<SPLIT>(out + (size_t)(i + r) * a.w.pitch(n), j, v[r]);
                    }
                    if (ti != tj) put_many<SPLIT, 4>(out + (size_t)j * a.w.pitch(n), i, v);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float* x = reinterpret_cast<float*>(base + a.w.x32) + (size_t)(i + r) * m + j;
                        v[r] = a.on_old * *x + acc[pi][pj][4 * u + r] * a.on_sum;
                        if (!a.last) *x = v[r];
                    }
                    if (!a.last) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) put<SPLIT>(base + a.w.x16 + (size_t)(i + r) * a.w.pitch(m), j, v[r] *= kScaleX);
                        put_many<SPLIT, 4>(base + a.t + (size_t)j * a.w.pitch(n), i, v);
                    } else {
                        O* out = reinterpret_cast<O*>(a.out.data) + (int64_t)matrix * a.out.batch;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint32_t row = a.tall ? j : i + r, col = a.tall ? i + r : j;
                            if (row < a.rows && col < a.cols) out[(int64_t)row * a.out.token + col] = (O)(v[r] * a.scale);
                        }
                    }
                }
            }
        }
}

// -------------------------------------------------------------------------------------------------------- host

// Side of a product's tiles.
uint32_t tile_of(uint32_t batch, uint32_t n, uint32_t m)
{
    const uint64_t tiles = (uint64_t)batch * ((n + 127) / 128) * ((m + 127) / 128);
    return tiles >= 128 ? 128 : 64;
}

constexpr uint32_t kParts = 64;     // sums of squares of a matrix

struct Layout {
    Work w;
    uint32_t tile;
    size_t squares, bytes;
};

Layout layout_of(uint32_t batch, uint32_t rows, uint32_t cols, bool split)
{
    Layout l{};
    const uint32_t n = rows < cols ? rows : cols, m = rows < cols ? cols : rows;
    l.tile = tile_of(batch, n, m);
    Work& w = l.w;
    w.split = split;
    w.n = (n + l.tile - 1) / l.tile * l.tile;
    w.m = (m + l.tile - 1) / l.tile * l.tile;
    size_t at = 0;
    const auto place = [&at](size_t bytes) {
        const size_t here = at;
        at += (bytes + 127) / 128 * 128;
        return here;
    };
    w.x32 = place((size_t)w.n * w.m * 4);
    w.x16 = place((size_t)w.n * w.pitch(w.m));
    w.xt16 = place((size_t)w.m * w.pitch(w.n));
    w.xt16_other = place((size_t)w.m * w.pitch(w.n));
    w.a16 = place((size_t)w.n * w.pitch(w.n));
    w.b16 = place((size_t)w.n * w.pitch(w.n));
    w.each = at;
    l.squares = (size_t)batch * w.each;
    l.bytes = l.squares + (size_t)batch * kParts * sizeof(double);
    return l;
}

// The largest |a s + b s^3 + c s^5| for 0 <= s <= h.
double reach(double a, double b, double c, double h)
{
    const auto p = [&](double u) { return std::fabs(std::sqrt(u) * (a + u * (b + u * c))); };
    double most = p(h * h);
    const auto look = [&](double u) {
        if (u > 0.0 && u < h * h && p(u) > most) most = p(u);
    };
    // zeros of the derivative a + 3 b u + 5 c u^2
    if (c == 0.0) {
        if (b != 0.0) look(-a / (3.0 * b));
    } else {
        const double d = 9.0 * b * b - 20.0 * a * c;
        if (d >= 0.0) {
            look((-3.0 * b + std::sqrt(d)) / (10.0 * c));
            look((-3.0 * b - std::sqrt(d)) / (10.0 * c));
        }
    }
    return most;
}

template <int TILE, int W, bool SPLIT, int MODE, typename O>
int product(const ProductArgs& a, uint32_t batch, hipStream_t st)
{
    hipLaunchKernelGGL((sdl_orthogonalize_product_kernel<TILE, W, SPLIT, MODE, O>), dim3(batch * a.tiles.d), dim3(W * W * kWave), 0, st, a);
    return launched();
}

template <int TILE, int W, bool SPLIT, typename O>
int steps_of(const Layout& l, uint32_t batch, uint32_t rows, uint32_t cols, const float* coefficients, uint32_t steps, float scale, const sdl_view_t* out,
             hipStream_t st)
{
    const Work& w = l.w;
    const uint32_t per = SPLIT ? 32 : 64, n = w.n / TILE, m = w.m / TILE;
    size_t xt = w.xt16, other = w.xt16_other;
    double h = 1.0;
    for (uint32_t s = 0; s < steps; ++s) {
        const double ca = coefficients[3 * s], cb = coefficients[3 * s + 1], cc = coefficients[3 * s + 2];
        // what the polynomial's matrix can be decides its image's scale
        const double bound = std::fabs(cb) * h * h + std::fabs(cc) * h * h * h * h;
        const float scale_b = (float)std::exp2(std::min(14.0, std::floor(std::log2(32768.0 / std::max(bound, 1e-30)))));
        h = reach(ca, cb, cc, h);
        ProductArgs a{};
        a.w = w;
        a.p = a.q = w.x16;
        a.t = w.a16;
        a.pitch_p = a.pitch_q = w.pitch(w.m);
        a.steps = w.m / per;
        a.tiles = make_div(n * (n + 1) / 2);
        a.on_sum = kScaleA / (kScaleX * kScaleX);
        if (product<TILE, W, SPLIT, GRAM, O>(a, batch, st) != SDL_OK) return SDL_ERR_DEVICE;
        a.p = a.q = w.a16;
        a.t = w.b16;
        a.pitch_p = a.pitch_q = w.pitch(w.n);
        a.steps = w.n / per;
        a.on_old = (float)(cb / kScaleA);
        a.on_sum = (float)(cc / ((double)kScaleA * kScaleA));
        a.image = scale_b;
        if (product<TILE, W, SPLIT, POLY, O>(a, batch, st) != SDL_OK) return SDL_ERR_DEVICE;
        a.p = w.b16;
        a.q = xt;
        a.t = other;
        a.tiles = make_div(n * m);
        a.across = make_div(m);
        a.on_old = (float)ca;
        a.on_sum = 1.0f / (scale_b * kScaleX);
        a.last = s + 1 == steps;
        a.out = kernel_view(out);
        a.tall = rows > cols;
        a.rows = rows;
        a.cols = cols;
        a.scale = scale;
        if (product<TILE, W, SPLIT, UPDATE, O>(a, batch, st) != SDL_OK) return SDL_ERR_DEVICE;
        std::swap(xt, other);
    }
    return SDL_OK;
}

template <typename T, bool SPLIT>
int first(const FirstArgs& a, uint32_t batch, hipStream_t st)
{
    hipLaunchKernelGGL((sdl_orthogonalize_norm_kernel<T>), dim3(a.parts, batch), dim3(256), 0, st, a);
    if (launched() != SDL_OK) return SDL_ERR_DEVICE;
    hipLaunchKernelGGL((sdl_orthogonalize_first_kernel<T, SPLIT>), dim3(a.w.m / 64, a.w.n / 64, batch), dim3(256), 0, st, a);
    return launched();
}

int check_shape(uint32_t batch, uint32_t rows, uint32_t cols)
{
    if (batch > 65535 || rows > SDL_ORTHOGONALIZE_MAX_SIDE || cols > SDL_ORTHOGONALIZE_MAX_SIDE) return SDL_ERR_UNSUPPORTED;
    return (uint64_t)batch * ((rows + 63) / 64) * ((cols + 63) / 64) > (1u << 22) ? SDL_ERR_UNSUPPORTED : SDL_OK;
}

}  // namespace

extern "C" {

size_t sdl_orthogonalize_workspace_bytes(uint32_t batch, uint32_t rows, uint32_t cols, sdl_dtype_t out_dtype)
{
    if (batch == 0 || rows == 0 || cols == 0 || !known(out_dtype) || check_shape(batch, rows, cols) != SDL_OK) return 0;
    return layout_of(batch, rows, cols, out_dtype == SDL_DTYPE_FP32).bytes;
}

int sdl_orthogonalize(const sdl_view_t* x, uint32_t batch, uint32_t rows, uint32_t cols, sdl_dtype_t dtype, const float* coefficients, uint32_t steps, float eps,
                      float scale, const sdl_view_t* out, sdl_dtype_t out_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!known(dtype) || !known(out_dtype) || steps == 0 || !coefficients) return SDL_ERR_INVALID_ARG;
    if (!(eps >= 0.0f && eps - eps == 0.0f) || !(scale - scale == 0.0f)) return SDL_ERR_INVALID_ARG;
    double h = 1.0;
    for (uint32_t s = 0; s < steps; ++s) {
        h = reach(coefficients[3 * s], coefficients[3 * s + 1], coefficients[3 * s + 2], h);
        if (!(h <= 2.0)) return SDL_ERR_INVALID_ARG;
    }
    int rc = check_shape(batch, rows, cols);
    if (rc != SDL_OK || batch == 0 || rows == 0 || cols == 0) return rc;
    if ((rc = check_view(x, dtype)) != SDL_OK || (rc = check_output(out, out_dtype, batch, rows, 1)) != SDL_OK) return rc;
    const bool split = out_dtype == SDL_DTYPE_FP32;
    const Layout l0 = layout_of(batch, rows, cols, split);
    if (!workspace || workspace_bytes < l0.bytes) return SDL_ERR_INVALID_ARG;
    if (!aligned_to(workspace, 16)) return SDL_ERR_ALIGNMENT;
    Layout l = l0;
    l.w.base = static_cast<char*>(workspace);
    FirstArgs a{};
    a.x = kernel_view(x);
    a.rows = rows;
    a.cols = cols;
    a.tall = rows > cols;
    a.parts = kParts;
    a.squares = reinterpret_cast<double*>(l.w.base + l.squares);
    a.eps = (double)eps;
    a.w = l.w;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == SDL_DTYPE_BF16) rc = split ? first<__bf16, true>(a, batch, st) : first<__bf16, false>(a, batch, st);
    else rc = split ? first<float, true>(a, batch, st) : first<float, false>(a, batch, st);
    if (rc != SDL_OK) return rc;
#define SDL_STEPS(TILE, W)                                                                                             \
    (split ? steps_of<TILE, W, true, float>(l, batch, rows, cols, coefficients, steps, scale, out, st)                 \
           : steps_of<TILE, W, false, __bf16>(l, batch, rows, cols, coefficients, steps, scale, out, st))
    return l.tile == 128 ? SDL_STEPS(128, 2) : SDL_STEPS(64, 2);
#undef SDL_STEPS
}

}  // extern "C"
