// Orthogonalising matrices by Newton-Schulz steps (gfx950).
//
//     X = x / (norm(x) + eps),  then for every (a, b, c):  A = X X^T,  X = a X + (b A + c A^2) X
//
// works on X = U S V^T as U p(S) V^T with p(s) = a s + b s^3 + c s^5: no product moves the singular vectors.  Three products a step, of
// which A and A^2 are symmetric and only half is formed; they bound it.  A tall matrix is worked on as its transpose.
//
// The products run on fp16 matrix instructions with fp32 sums.  X lies within the unit ball (the coefficients are checked on the host), so a power of
// two keeps its elements in the middle of fp16's range: X 2^14, A 2^12, and b A + c A^2 by what its bound allows.
//   - X itself is kept with more digits than its image has, and a X is taken from there.  What the images lose is then a factor near 1 on what a
//     direction already is: an error of X itself would be lifted with the small singular values, 3.4 times a step.
//   - Near its end A is nearly diagonal, and an image's error on the diagonal would go into a whole row of X: so the diagonals of A and of b A + c A^2 are kept apart in fp32, and are
//     zero in the images.
//   - results in bf16, more than 256 rows: one image, 11 bits.  Five steps are off by 0.0003 to 0.0005 of the result beside the 0.0017 of its own rounding, of rank one by 0.42 / rows.  X is its
//     image and what that leaves, as fp16 too: together the digits of fp32, down to 2^-50 of the norm, in the same four bytes.  (With what is left in bf16, 20 bits, results of rank one
//     were off by up to 1.4 times as much: what X's rounding puts into the directions that are not there is lifted with them.  The write of X is what an update waits for: in fp32 beside
//     its image it was half as much again.)
//   - results in fp32, and matrices of fewer rows: two images, x 2^14 = hi + lo, 22 bits, and three products hi hi + hi lo + lo hi.  What is left out is 2^-24.  X in fp32.  All sizes are off
//     by 0.4 to 1.7e-6, of rank one by up to 9e-5.
// An operand's rows are cut into pieces of 128 bytes, one step of a product's loop each: 64 elements, or 32 of hi and the same 32 of lo.
#include <algorithm>
#include <cmath>
#include <iterator>
#include <type_traits>
#include <utility>

#include "sdl_operand.h"

namespace {

using namespace sdl_device;

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));

constexpr float kScaleX = 16384.0f, kScaleA = 4096.0f;
constexpr float kScaleRest = 2048.0f;       // of what one image leaves of X: a part of 2^12 at most, so that it lies where the image did
constexpr uint32_t kDies = 8;
constexpr uint32_t kMostSmallSteps = 32, kMostParts = 1024;

// One matrix in the workspace, of which the next lies `each` bytes further.  Both sides are filled up with zeros to whole tiles.
struct Work {
    char* base;
    size_t each;
    size_t rest, x16, x16_other, a16, b16;           // offsets; rest: X in fp32, or in fp16 what its one image leaves
    size_t a_diagonal, b_diagonal;                    // in fp32, as large as the images
    uint32_t n, m;                                    // n <= m, filled up
    uint32_t split;
    __host__ __device__ uint32_t pitch(uint32_t k) const { return k * (split ? 4u : 2u); }     // bytes of a row of k elements of an image
};

// Eight elements of an image, from element k of its row on, a multiple of eight.
struct Parts {
    f16x8_t hi, lo;
};
__device__ __forceinline__ Parts parts_of(const float* v)
{
    typedef float f32x8_t __attribute__((ext_vector_type(8)));
    f32x8_t x, rest;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i];
    Parts p;
    p.hi = __builtin_convertvector(x, f16x8_t);
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = v[i] - (float)p.hi[i];
    p.lo = __builtin_convertvector(rest, f16x8_t);
    return p;
}
template <bool SPLIT>
__device__ __forceinline__ f16x8_t* piece(char* row, uint32_t k)
{
    return reinterpret_cast<f16x8_t*>(row + (SPLIT ? (k / 32) * 128 + (k % 32) * 2 : k * 2));
}
template <bool SPLIT>
__device__ __forceinline__ void put(char* row, uint32_t k, const Parts& p)
{
    f16x8_t* at = piece<SPLIT>(row, k);
    at[0] = p.hi;
    if constexpr (SPLIT) at[4] = p.lo;
}

// Eight elements of X, as its image (at x16) and what is kept beside it.
template <bool SPLIT>
__device__ __forceinline__ void put_x(char* base, const Work& w, size_t x16, uint32_t i, uint32_t j, const float* v)
{
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = v[e] * kScaleX;
    const Parts image = parts_of(s);
    put<SPLIT>(base + x16 + (size_t)i * w.pitch(w.m), j, image);
    if constexpr (SPLIT) {
        store8(reinterpret_cast<float*>(base + w.rest) + (size_t)i * w.m, j, j + 8, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = (s[e] - (float)image.hi[e]) * kScaleRest;
        *reinterpret_cast<f16x8_t*>(base + w.rest + ((size_t)i * w.m + j) * 2) = parts_of(s).hi;
    }
}

// ------------------------------------------------------------------------------------------- norm, first image

struct FirstArgs {
    View x;                     // rows along `token`
    uint32_t rows, cols, tall, parts;
    Div groups;                 // of eight, of a row
    double* squares;            // [matrix][parts]
    double eps;
    Work w;
};

// Sum of squares of a part of a matrix: in 64 bits, in which no square of a 32-bit number is out of range.
template <typename T>
__global__ void __launch_bounds__(256) sdl_orthogonalize_norm_kernel(const FirstArgs a)
{
    __shared__ double sums[4];
    const uint32_t part = blockIdx.x, matrix = blockIdx.y;
    const T* x = reinterpret_cast<const T*>(a.x.data) + (int64_t)matrix * a.x.batch;
    const uint32_t n = a.rows * a.groups.d;         // groups of eight of all rows
    double s = 0.0;
    for (uint32_t i0 = part * 256 + threadIdx.x; i0 < n; i0 += 4 * a.parts * 256) {
        // four loads wait together; those behind the end are the last group, and not counted
        Eight<T> e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t i = min(i0 + k * a.parts * 256, n - 1), r = div(i, a.groups);
            e[k] = load8(x + (int64_t)r * a.x.token, (i - r * a.groups.d) * 8, a.cols);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i0 + k * a.parts * 256 >= n) break;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += (double)e[k].get(j) * (double)e[k].get(j);
        }
    }
#pragma unroll
    for (int k = 32; k; k /= 2) s += __shfl_xor(s, k);
    if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.squares[(size_t)matrix * a.parts + part] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// x over its norm, or its transpose, in tiles of 64 by 64 of what the workspace holds.
template <typename T, bool SPLIT>
__global__ void __launch_bounds__(256) sdl_orthogonalize_first_kernel(const FirstArgs a)
{
    __shared__ float tile[64][65];
    __shared__ double sums[4];
    const uint32_t matrix = blockIdx.z, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;      // of the n by m matrix
    const T* x = reinterpret_cast<const T*>(a.x.data) + (int64_t)matrix * a.x.batch;
    const uint32_t r0 = a.tall ? j0 : i0, c0 = a.tall ? i0 : j0, c = threadIdx.x % 8 * 8;
    Eight<T> e[2];
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t row = r0 + threadIdx.x / 8 + 32 * k;
        e[k] = Eight<T>{};
        if (row < a.rows && c0 + c < a.cols) e[k] = load8(x + (int64_t)row * a.x.token, c0 + c, a.cols);
    }
    double s = 0.0;
#pragma unroll
    for (uint32_t k = 0; k < kMostParts / 256; ++k) {
        const uint32_t p = k * 256 + threadIdx.x;
        if (p < a.parts) s += a.squares[(size_t)matrix * a.parts + p];
    }
#pragma unroll
    for (int k = 32; k; k /= 2) s += __shfl_xor(s, k);
    if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave] = s;
    __syncthreads();
    const double norm = sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + a.eps, inverse = norm == 0.0 ? 0.0 : 1.0 / norm;
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t row = threadIdx.x / 8 + 32 * k;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = (float)((double)e[k].get(j) * inverse);
            if (a.tall) tile[c + j][row] = v;
            else tile[row][c + j] = v;
        }
    }
    __syncthreads();
    char* base = a.w.base + matrix * a.w.each;
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        const uint32_t row = threadIdx.x / 8 + 32 * k;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = tile[row][c + j];
        put_x<SPLIT>(base, a.w, a.w.x16, i0 + row, j0 + c, v);
    }
}

// ----------------------------------------------------------------------------------------------------- products

enum { GRAM, POLY, UPDATE };

// Between what lanes of a wavefront write to shared memory and what others of it read there, either way.  A wavefront's accesses keep the order they are issued in; this keeps the
// compiler from issuing them in another one, and is no instruction.
__device__ __forceinline__ void lanes_meet()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A symmetric product has few tiles, and with one long matrix few compute units are at work: then every tile's sum is cut into slices, whose partial sums go
// through memory (PART), and are added up in order by a launch that goes on as the other way does (JOIN).
enum { WHOLE, PART, JOIN };

struct ProductArgs {
    Work w;
    size_t p, q, t;             // offsets of the two operands' images, and of the one that is written
    uint32_t pitch_p, pitch_q, steps;
    Div slice_of;               // slices of a sum, and the partial sums of each:
    f32x4_t* partial;           // [workgroup][slice][4 registers][thread]
    Div tiles, across;          // of a matrix; UPDATE: along m
    float on_sum, on_old;       // result = on_old * old + on_sum * product
    // the last update: where to
    View out;
    uint32_t last, tall, rows, cols;
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

// TILE by TILE of C = P Q^T (UPDATE: P Q), by 2 by 2 wavefronts.  An operand with k along its rows: in shared memory a row's step is 128 bytes, its eight
// pieces swapped around by an xor with bits 1 to 3 of the row's number; neither the copies nor the reads (16 rows, one piece) meet in a bank.  Q of an update, X with k down its columns: a
// step is 64 (of two images 32) rows of the tile's columns, read by transposing reads of four rows at a time, whose pieces are moved apart by an xor of bits 2 and 3 with the row's number.
// Two steps' tiles in turn.  A step is G groups of products; a group's operands are read while the one before is multiplied, and the wait for the next step's tile
// comes in front of the last group, whose operands are in registers by then: its products run while the next step's first operands are read and the copies of the one after
// that are started.
//
// Layouts of the 32x32x16 instruction, lane l, half = l / 32, c = l % 32:  A row c, k = 8 half + j;  B column c, k = 8 half + j;
// D column c, rows 8 (i / 4) + 4 half + i % 4.
//
// The columns of D are the rows of C, of which a lane so has four neighbours at a time.  Results go through shared memory in blocks of a wavefront's own, so that they are written (and
// what they are added to is read) in pieces of 16 bytes, and the images of what is symmetric once more: transposing reads give its other half.
template <int TILE, bool SPLIT, int MODE, int HOW, typename O>
__global__ void __launch_bounds__(256) sdl_orthogonalize_product_kernel(const ProductArgs a)
{
    constexpr int kBytes = TILE * 128, kSide = TILE / 2, kParts = kSide / 32, kCopies = TILE / 32, kGroups = SPLIT ? 2 : 4;
    // Of a block, bytes from row to row of fp32 and of an image: a row's pieces are four banks further than those of the row before.
    constexpr int kBlock = kSide < 64 ? kSide : 64, kPitch = kBlock * 4 + 16, kImagePitch = kBlock * 2 + 16;
    constexpr int kOwn = kBlock * (kPitch > 2 * kImagePitch ? kPitch : 2 * kImagePitch);      // of a wavefront: a block, or both of its images
    constexpr int kLds = 4 * (kBytes > kOwn ? kBytes : kOwn);
    __shared__ __attribute__((aligned(128))) char lds[kLds];
    const uint32_t lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), half = lane / 32, c = lane % 32;
    // consecutive workgroups go to different dies: each die takes tiles that follow each other, which share rows in its cache
    const uint32_t die = blockIdx.x % kDies, each = gridDim.x / kDies, more = gridDim.x % kDies;
    const uint32_t number = die * each + min(die, more) + blockIdx.x / kDies;
    const uint32_t at = HOW == PART ? div(number, a.slice_of) : number, matrix = div(at, a.tiles), t = at - matrix * a.tiles.d;
    const uint32_t slice = HOW == PART ? number - at * a.slice_of.d : 0;
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
    const uint32_t first = HOW == PART ? slice * a.steps / a.slice_of.d : 0, steps = (HOW == PART ? (slice + 1) * a.steps / a.slice_of.d : a.steps) - first;
    const char* from_p = base + a.p + (size_t)(ti * TILE + wave * kCopies * 8) * a.pitch_p + (size_t)first * 128;
    constexpr int kRow = MODE == UPDATE ? TILE * (SPLIT ? 4 : 2) : 128, kRowPieces = kRow / 16, kRowsOfCopy = 1024 / kRow, kStepRows = SPLIT ? 32 : 64;      // of Q in shared memory
    const char* from_q = base + a.q + (MODE == UPDATE ? (size_t)tj * kRow : (size_t)(tj * TILE + wave * kCopies * 8) * a.pitch_q + (size_t)first * 128);
    const size_t step_q = MODE == UPDATE ? (size_t)kStepRows * a.pitch_q : 128;
    const auto apart = [](uint32_t row) { return kRowPieces >= 16 ? (row & 3) << 2 : (row & 2) << 1; };
    // the piece that comes to lie where the lane's 16 bytes land, in the even instructions; 4 further, by xor, in the odd ones
    const uint32_t piece_at = ((lane % 8) ^ (lane / 16)) * 16;
    const uint32_t off_p = lane / 8 * a.pitch_p + piece_at, off_q = lane / 8 * a.pitch_q + piece_at;
    static_assert(kCopies % 2 == 0, "an instruction's parity is its number's within the wavefront's");
    uint32_t offs_p[kCopies], offs_q[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        offs_p[i] = (off_p ^ (i % 2 * 64)) + i * 8 * a.pitch_p;
        if constexpr (MODE == UPDATE) {
            const uint32_t row = (wave * kCopies + i) * kRowsOfCopy + lane / kRowPieces;
            offs_q[i] = row * a.pitch_q + ((lane % kRowPieces) ^ apart(row)) * 16;
        } else {
            offs_q[i] = (off_q ^ (i % 2 * 64)) + i * 8 * a.pitch_q;
        }
    }
    // the i-th of a wavefront's copies of a step's tiles
    const auto copy = [&](uint32_t step, int i) {
        const uint32_t to = lds_offset(lds) + (step % 2) * (2 * kBytes) + wave * kCopies * 1024;
        if (i % 2 == 0) copy_pieces(from_p + step * 128, offs_p[i / 2], to + i / 2 * 1024);
        else copy_pieces(from_q + step * step_q, offs_q[i / 2], to + kBytes + i / 2 * 1024);
    };
    const uint32_t i0 = wave / 2 * kSide, j0 = wave % 2 * kSide, mix = (c >> 1) & 7;
    constexpr int kImages = SPLIT ? 2 : 1, kReads = 2 * kParts * kImages, kProducts = kParts * kParts * (SPLIT ? 3 : 1);     // of a group
    f16x8_t p[2][kImages][kParts], q[2][kImages][kParts];
    // The transposing read of two times four rows: lane 4 r + q of 16 names the q-th quarter of row r of 4, and gets the four rows of its column of 16.
    const auto across = [](const char* at, int four) {
        typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
        const i16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + four));
        return __builtin_bit_cast(f16x8_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // where this lane's reads of an update's Q start: row 8 half + its number of four, the piece of the columns of its half of 32
    uint32_t read_q[kImages][kParts];
    if constexpr (MODE == UPDATE) {
        const uint32_t row = 8 * half + lane % 16 / 4;
#pragma unroll
        for (int image = 0; image < kImages; ++image)
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                const uint32_t piece = (SPLIT ? (j0 / 32 + i) * 8 + image * 4 : (j0 / 32 + i) * 4) + lane % 32 / 16 * 2 + lane % 4 / 2;
                read_q[image][i] = kBytes + row * kRow + (piece ^ apart(row)) * 16 + lane % 2 * 8;
            }
    }
    // the r-th of the reads of a group's operands
    const auto read = [&](uint32_t step, int g, int to, int r) {
        const char* rows = lds + (step % 2) * (2 * kBytes) + c * 128;
        const int image = r / (2 * kParts), i = r % (2 * kParts) / 2;
        const uint32_t at = ((4 * image + 2 * g + half) ^ mix) * 16;
        if (r % 2 == 0) p[to][image][i] = *reinterpret_cast<const f16x8_t*>(rows + (i0 + i * 32) * 128 + at);
        else if constexpr (MODE == UPDATE) q[to][image][i] = across(lds + (step % 2) * (2 * kBytes) + read_q[image][i] + g * 16 * kRow, 4 * kRow);
        else q[to][image][i] = *reinterpret_cast<const f16x8_t*>(rows + kBytes + (j0 + i * 32) * 128 + at);
    };
    f32x16_t acc[kParts][kParts] = {};
    // the m-th of a group's products: hi hi of all, hi lo of all, lo hi of all
    const auto multiply = [&](int from, int m) {
        const int way = m / (kParts * kParts), i = m / kParts % kParts, j = m % kParts;
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(q[from][way == 1][j], p[from][way == 2][i], acc[i][j], 0, 0, 0);
    };
    const auto arrived = [&]() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
    };
    // The order of the instructions is the one that is written: between two products one read or copy or two.  The last two steps have nothing to copy.
    const auto multiply_step = [&](uint32_t step, auto copies) {
#pragma unroll
        for (int g = 0; g < kGroups - 1; ++g) {
#pragma unroll
            for (int m = 0; m < kProducts; ++m) {
                multiply(g % 2, m);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = kReads * m / kProducts; r < kReads * (m + 1) / kProducts; ++r) read(step, g + 1, (g + 1) % 2, r);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        arrived();
        constexpr int kAll = kReads + decltype(copies)::value * 2 * kCopies;
#pragma unroll
        for (int m = 0; m < kProducts; ++m) {
            multiply((kGroups - 1) % 2, m);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int r = kAll * m / kProducts; r < kAll * (m + 1) / kProducts; ++r) {
                if (r < kReads) read(step + 1, 0, 0, r);        // behind the last step what lies there, for nothing
                else copy(step + 2, r - kReads);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // the partial sums of a slice, a register of four at a time
    const auto partial_of = [&](uint32_t which) { return a.partial + ((size_t)at * a.slice_of.d + which) * (kParts * kParts * 4 * 256) + threadIdx.x; };
    if constexpr (HOW != JOIN) {
#pragma unroll
        for (int i = 0; i < 2 * kCopies; ++i) copy(0, i);
        arrived();
        if (steps > 1) {
#pragma unroll
            for (int i = 0; i < 2 * kCopies; ++i) copy(1, i);
        }
#pragma unroll
        for (int r = 0; r < kReads; ++r) read(0, 0, 0, r);
        uint32_t step = 0;
        for (; step + 2 < steps; ++step) multiply_step(step, std::integral_constant<int, 1>());
#pragma unroll 1
        for (; step < steps; ++step) multiply_step(step, std::integral_constant<int, 0>());
    } else {
        for (uint32_t which = 0; which < a.slice_of.d; ++which) {
            const f32x4_t* from = partial_of(which);
#pragma unroll
            for (int i = 0; i < kParts; ++i)
#pragma unroll
                for (int j = 0; j < kParts; ++j)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const f32x4_t v = from[((i * kParts + j) * 4 + u) * 256];
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[i][j][4 * u + r] += v[r];
                    }
        }
    }
    if constexpr (HOW == PART) {
        f32x4_t* to = partial_of(slice);
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int j = 0; j < kParts; ++j)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    f32x4_t v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * u + r];
                    to[((i * kParts + j) * 4 + u) * 256] = v;
                }
        return;
    }
    __syncthreads();        // the tiles' memory becomes the blocks'
    const uint32_t n = a.w.n, m = a.w.m;
    char* block = lds + wave * kOwn;
    constexpr int kSpan = kBlock / 8, kRows = kWave / kSpan, kPasses = kBlock / kRows, kIn = kBlock / 32;     // lanes of a row; rows of a pass
    const uint32_t r0 = lane / kSpan, c0 = lane % kSpan * 8;
#pragma unroll
    for (int bi = 0; bi < kParts / kIn; ++bi)
#pragma unroll
        for (int bj = 0; bj < kParts / kIn; ++bj) {
            const uint32_t i = ti * TILE + i0 + bi * kBlock, j = tj * TILE + j0 + bj * kBlock;     // the block's first row and column
            Parts old[MODE == POLY || (MODE == UPDATE && !SPLIT) ? kPasses : 1];
            Eight<float> x[MODE == UPDATE && SPLIT ? kPasses : 1];
            f16x8_t rest[MODE == UPDATE && !SPLIT ? kPasses : 1];
            float own[MODE != GRAM ? kPasses : 1];                     // the rows' places of the diagonal
            Eight<float> others;
            if constexpr (MODE == POLY) {
#pragma unroll
                for (int k = 0; k < kPasses; ++k) {
                    const f16x8_t* at = piece<SPLIT>(base + a.w.a16 + (size_t)(i + k * kRows + r0) * a.w.pitch(n), j + c0);
                    old[k].hi = at[0];
                    old[k].lo = SPLIT ? at[4] : f16x8_t{};
                    own[k] = reinterpret_cast<const float*>(base + a.w.a_diagonal)[i + k * kRows + r0];
                }
                others = load8(reinterpret_cast<const float*>(base + a.w.a_diagonal) + j, c0, c0 + 8);
            }
            if constexpr (MODE == UPDATE) {
#pragma unroll
                for (int k = 0; k < kPasses; ++k) {
                    const uint32_t row = i + k * kRows + r0;
                    own[k] = reinterpret_cast<const float*>(base + a.w.b_diagonal)[row];
                    if constexpr (SPLIT) {
                        x[k] = load8(reinterpret_cast<const float*>(base + a.w.rest) + (size_t)row * m + j, c0, c0 + 8);
                    } else {
                        old[k].hi = *piece<false>(base + a.q + (size_t)row * a.w.pitch(m), j + c0);
                        rest[k] = *reinterpret_cast<const f16x8_t*>(base + a.w.rest + ((size_t)row * m + j + c0) * 2);
                    }
                }
            }
#pragma unroll
            for (int pi = 0; pi < kIn; ++pi)
#pragma unroll
                for (int pj = 0; pj < kIn; ++pj)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        f32x4_t v;
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = acc[bi * kIn + pi][bj * kIn + pj][4 * u + r];
                        *reinterpret_cast<f32x4_t*>(block + (pi * 32 + c) * kPitch + (pj * 32 + 8 * u + 4 * half) * 4) = v;
                    }
            lanes_meet();
            float v[kPasses][8];
#pragma unroll
            for (int k = 0; k < kPasses; ++k) {
                const char* at = block + (k * kRows + r0) * kPitch + c0 * 4;
                const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(at), hi = *reinterpret_cast<const f32x4_t*>(at + 16);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float s = e < 4 ? lo[e & 3] : hi[e & 3];
                    if constexpr (MODE == GRAM) v[k][e] = s * a.on_sum;
                    if constexpr (MODE == POLY)
                        v[k][e] = fmaf(s, a.on_sum, fmaf(a.on_sum, own[k] + others.get(e), a.on_old) * (SPLIT ? (float)old[k].hi[e] + (float)old[k].lo[e] : (float)old[k].hi[e]));
                    if constexpr (MODE == UPDATE && SPLIT) v[k][e] = fmaf(s, a.on_sum, fmaf(a.on_sum * kScaleX, own[k], a.on_old) * x[k].get(e));
                    if constexpr (MODE == UPDATE && !SPLIT) v[k][e] = fmaf(s, a.on_sum, fmaf(a.on_sum, own[k], a.on_old / kScaleX) * fmaf((float)rest[k][e], 1.0f / kScaleRest, (float)old[k].hi[e]));
                }
            }
            lanes_meet();           // the block is written again: turned, as an image, or with the next one
            if constexpr (MODE != UPDATE) {
                if (i == j) {       // the diagonal goes apart, and is zero in the image
#pragma unroll
                    for (int k = 0; k < kPasses; ++k) {
                        const uint32_t row = k * kRows + r0;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            if (row != c0 + e) continue;
                            if constexpr (MODE == GRAM) reinterpret_cast<float*>(base + a.w.a_diagonal)[i + row] = v[k][e];
                            else reinterpret_cast<float*>(base + a.w.b_diagonal)[i + row] = fmaf(fmaf(a.on_sum, own[k], a.on_old), own[k], v[k][e]);
                            v[k][e] = 0.0f;
                        }
                    }
                }
            }
            if constexpr (MODE == UPDATE) {
                if (a.last) {
                    O* out = reinterpret_cast<O*>(a.out.data) + (int64_t)matrix * a.out.batch;
                    if (!a.tall) {
#pragma unroll
                        for (int k = 0; k < kPasses; ++k) {
                            const uint32_t row = i + k * kRows + r0;
                            if (row < a.rows && j + c0 < a.cols) store8(out + (int64_t)row * a.out.token, j + c0, a.cols, v[k]);
                        }
                        continue;
                    }
#pragma unroll
                    for (int k = 0; k < kPasses; ++k)
                        store8(reinterpret_cast<float*>(block + (k * kRows + r0) * kPitch), c0, c0 + 8, v[k]);
                    lanes_meet();
#pragma unroll
                    for (int k = 0; k < kPasses; ++k) {
                        const uint32_t row = lane % kBlock, col = (k * (kWave / kBlock) + lane / kBlock) * 8;
                        float t[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) t[e] = *reinterpret_cast<const float*>(block + (col + e) * kPitch + row * 4);
                        if (j + row < a.rows && i + col < a.cols) store8(out + (int64_t)(j + row) * a.out.token, i + col, a.cols, t);
                    }
                    lanes_meet();
                    continue;
                }
#pragma unroll
                for (int k = 0; k < kPasses; ++k) put_x<SPLIT>(base, a.w, a.t, i + k * kRows + r0, j + c0, v[k]);
                continue;
            }
            const bool turned = ti != tj;
#pragma unroll
            for (int k = 0; k < kPasses; ++k) {
                const uint32_t row = k * kRows + r0;
                const Parts image = parts_of(v[k]);
                put<SPLIT>(base + a.t + (size_t)(i + row) * a.w.pitch(n), j + c0, image);
                if (turned) {
                    *reinterpret_cast<f16x8_t*>(block + row * kImagePitch + c0 * 2) = image.hi;
                    if constexpr (SPLIT) *reinterpret_cast<f16x8_t*>(block + (kBlock + row) * kImagePitch + c0 * 2) = image.lo;
                }
            }
            if (!turned) continue;
            lanes_meet();
            // lanes of a group of 16 have a column each, of 16; the groups have eight rows each, of 32
#pragma unroll
            for (int k = 0; k < kPasses; ++k) {
                const uint32_t col = k % (kBlock / 16) * 16, row = k / (kBlock / 16) * 32 + lane / 16 * 8;
                const char* at = block + (row + lane % 16 / 4) * kImagePitch + col * 2 + lane % 4 * 8;
                Parts image;
                image.hi = across(at, 4 * kImagePitch);
                if constexpr (SPLIT) image.lo = across(at + kBlock * kImagePitch, 4 * kImagePitch);
                put<SPLIT>(base + a.t + (size_t)(j + col + lane % 16) * a.w.pitch(n), i + row, image);
            }
            lanes_meet();
        }
}

// --------------------------------------------------------------------------------------------- small matrices

struct SmallArgs {
    View x, out;
    Div across;                                  // tiles along m
    uint32_t tall, n, m, steps;                  // n <= m
    double eps;
    float scale;
    float* between;                              // [matrix][n][m]: X where a launch's steps are not all of them
    uint32_t resumes, pauses;                    // X comes from there, is left there
    float a[kMostSmallSteps], b[kMostSmallSteps], c[kMostSmallSteps], image[kMostSmallSteps];     // image: the scale of b A + c A^2
};

// Tiles of a symmetric product of a wavefront's, at most.
constexpr uint32_t kHalves = 3;

// A matrix whose two images fit the shared memory of a workgroup is worked on there from its norm to its last step: with a launch for every product it would be the launches, 80 us for
// five steps of 100 x 131, which take 60 so.  Tiles of 16 by 16 go round among the wavefronts; those of X stay in the registers of theirs, in fp32, and what a step makes of them is what the next one
// starts from.
//
// Layouts of the 16x16x32 instruction, lane l, q = l / 16, c = l % 16:  A row c, k = 8 q + j;  B column c, k = 8 q + j;  D column c, rows 4 q + i.  X's tile
// has its rows along c, so that a lane has four neighbours of a row: A = the columns of X, by transposing reads, B = the rows of b A + c A^2.
template <typename T, typename O, int WAVES, int SLOTS, int BYTES>
__global__ void __launch_bounds__(WAVES * kWave) sdl_orthogonalize_small_kernel(const SmallArgs a)
{
    constexpr int kImages = 2;
    __shared__ __attribute__((aligned(16))) char lds[BYTES];
    __shared__ double sums[WAVES];
    const uint32_t lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), q = lane / 16, c = lane % 16, matrix = blockIdx.x;
    const uint32_t down = (a.n + 15) / 16, across = a.across.d, nk = (a.n + 31) / 32 * 32, mk = (a.m + 31) / 32 * 32;
    const uint32_t pitch_x = mk * 2 + 16, pitch_a = nk * 2 + 16, bytes_x = nk * pitch_x, bytes_a = nk * pitch_a;
    char *const image_x = lds, *const image_a = lds + kImages * bytes_x;
    float *const a_diagonal = reinterpret_cast<float*>(image_a + kImages * bytes_a), *const b_diagonal = a_diagonal + nk;
    // what no tile writes is zero
    for (uint32_t i = threadIdx.x * 16; i < kImages * (bytes_x + bytes_a); i += WAVES * kWave * 16) *reinterpret_cast<u32x4*>(lds + i) = u32x4{0, 0, 0, 0};

    // X's tiles of this wavefront, the s-th of them.  Worked out anew wherever it is asked for: kept for all of them they would take the registers.
    const uint32_t tiles = down * across;
    const auto tile = [&](int s, uint32_t* i, uint32_t* j) {
        uint32_t t = wave;
        asm volatile("" : "+s"(t));
        t += s * WAVES;
        const uint32_t row = div(t, a.across);
        *i = row * 16;
        *j = (t - row * across) * 16;
        return t < tiles;
    };
    f32x4_t x[SLOTS];
    float* const between = a.between + (size_t)matrix * a.n * a.m;
    const T* from = reinterpret_cast<const T*>(a.x.data) + (int64_t)matrix * a.x.batch;
    double squares = 0.0;
    // no load waits for another: what is not there is the last element, and not counted
    const auto load = [&](const auto* at, int64_t down, int64_t over) {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            uint32_t i, j;
            tile(s, &i, &j);
            const uint32_t row = min(i + c, a.n - 1);
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) x[s][r] = (float)at[row * down + min(j + 4 * q + r, a.m - 1) * over];
        }
    };
    if (a.resumes) load(between, a.m, 1);
    else if (a.tall) load(from, 1, a.x.token);
    else load(from, a.x.token, 1);
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        uint32_t i, j;
        const bool there = tile(s, &i, &j);
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
            x[s][r] = there && i + c < a.n && j + 4 * q + r < a.m ? x[s][r] : 0.0f;
            squares += (double)x[s][r] * (double)x[s][r];
        }
    }
#pragma unroll
    for (int k = 32; k; k /= 2) squares += __shfl_xor(squares, k);
    if (lane == 0) sums[wave] = squares;
    __syncthreads();
    squares = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) squares += sums[w];
    const double norm = a.resumes ? 1.0 : sqrt(squares) + a.eps, inverse = norm == 0.0 ? 0.0 : 1.0 / norm;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[s][r] = (float)((double)x[s][r] * inverse);

    // four neighbours of a row of an image, hi and lo
    const auto put4 = [&](char* image, uint32_t bytes, uint32_t pitch, uint32_t row, uint32_t k, const f32x4_t& v) {
        const f16x4_t hi = __builtin_convertvector(v, f16x4_t);
        *reinterpret_cast<f16x4_t*>(image + row * pitch + k * 2) = hi;
        f32x4_t rest;
#pragma unroll
        for (int r = 0; r < 4; ++r) rest[r] = v[r] - (float)hi[r];
        *reinterpret_cast<f16x4_t*>(image + bytes + row * pitch + k * 2) = __builtin_convertvector(rest, f16x4_t);
    };
    const auto put1 = [&](char* image, uint32_t bytes, uint32_t pitch, uint32_t row, uint32_t k, float v) {
        const _Float16 hi = (_Float16)v;
        *reinterpret_cast<_Float16*>(image + row * pitch + k * 2) = hi;
        *reinterpret_cast<_Float16*>(image + bytes + row * pitch + k * 2) = (_Float16)(v - (float)hi);
    };
    const auto along = [&](const char* image, uint32_t pitch, uint32_t row, uint32_t k) {
        return *reinterpret_cast<const f16x8_t*>(image + (row + c) * pitch + (k + 8 * q) * 2);
    };
    const auto across_rows = [&](const char* image, uint32_t pitch, uint32_t k, uint32_t col) {
        typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
        const char* at = image + (k + 8 * q + c / 4) * pitch + (col + c % 4 * 4) * 2;
        const i16x4_t u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)at), v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + 4 * pitch));
        return __builtin_bit_cast(f16x8_t, __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // one tile of rows i of an image times rows j of the same one
    const auto symmetric = [&](const char* image, uint32_t bytes, uint32_t pitch, uint32_t i, uint32_t j, uint32_t kk) {
        f32x4_t d = {};
#pragma unroll 2
        for (uint32_t k = 0; k < kk; k += 32) {
            const f16x8_t p = along(image, pitch, i, k), r = along(image, pitch, j, k);
            const f16x8_t pl = along(image + bytes, pitch, i, k), rl = along(image + bytes, pitch, j, k);
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(p, r, d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(p, rl, d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl, r, d, 0, 0, 0);
        }
        return d;
    };
    // D of rows i and columns j, in its place and in the one across; its diagonal apart
    const auto put_symmetric = [&](uint32_t i, uint32_t j, f32x4_t v, float* diagonal) {
        if (i == j)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                if (4 * q + r != c) continue;
                diagonal[i + c] = v[r];
                v[r] = 0.0f;
            }
        put4(image_a, bytes_a, pitch_a, j + c, i + 4 * q, v);
        if (i != j)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) put1(image_a, bytes_a, pitch_a, i + 4 * q + r, j + c, v[r]);
    };
    // tiles on and under the diagonal: the t-th of them
    const auto place = [](uint32_t t, uint32_t* i, uint32_t* j) {
        // (the root of a square is exact, and t is small)
        const uint32_t row = __builtin_amdgcn_readfirstlane((uint32_t)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f));
        *i = row * 16;
        *j = (t - row * (row + 1) / 2) * 16;
    };
    const uint32_t halves = down * (down + 1) / 2;
    for (uint32_t step = 0; step < a.steps; ++step) {
        // X's image, once everyone has read the one before
        __syncthreads();
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            uint32_t i, j;
            if (tile(s, &i, &j)) put4(image_x, bytes_x, pitch_x, i + c, j + 4 * q, x[s] * kScaleX);
        }
        __syncthreads();
        for (uint32_t t = wave; t < halves; t += WAVES) {
            uint32_t i, j;
            place(t, &i, &j);
            put_symmetric(i, j, symmetric(image_x, bytes_x, pitch_x, i, j, mk) * (kScaleA / (kScaleX * kScaleX)), a_diagonal);
        }
        __syncthreads();
        f32x4_t mix[kHalves];
#pragma unroll
        for (uint32_t s = 0; s < kHalves; ++s) {
            const uint32_t t = s * WAVES + wave;
            if (t >= halves) continue;
            uint32_t i, j;
            place(t, &i, &j);
            const f32x4_t square = symmetric(image_a, bytes_a, pitch_a, i, j, nk);
            const f16x4_t hi = *reinterpret_cast<const f16x4_t*>(image_a + (j + c) * pitch_a + (i + 4 * q) * 2);
            const f16x4_t lo = *reinterpret_cast<const f16x4_t*>(image_a + bytes_a + (j + c) * pitch_a + (i + 4 * q) * 2);
            const float on_square = a.c[step] * a.image[step] / (kScaleA * kScaleA), on_a = a.b[step] * a.image[step] / kScaleA;
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                const float own = a_diagonal[i + 4 * q + r];
                mix[s][r] = i == j && 4 * q + r == c ? fmaf(on_square, fmaf(own, own, square[r]), on_a * own)
                                                     : fmaf(square[r], on_square, fmaf(on_square, own + a_diagonal[j + c], on_a) * ((float)hi[r] + (float)lo[r]));
            }
        }
        __syncthreads();
#pragma unroll
        for (uint32_t s = 0; s < kHalves; ++s) {
            const uint32_t t = s * WAVES + wave;
            if (t >= halves) continue;
            uint32_t i, j;
            place(t, &i, &j);
            put_symmetric(i, j, mix[s], b_diagonal);
        }
        __syncthreads();
        const float on_sum = 1.0f / (a.image[step] * kScaleX);
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            uint32_t i, j;
            if (!tile(s, &i, &j)) continue;
            f32x4_t d = {};
#pragma unroll 2
            for (uint32_t k = 0; k < nk; k += 32) {
                const f16x8_t p = across_rows(image_x, pitch_x, k, j), r = along(image_a, pitch_a, i, k);
                const f16x8_t pl = across_rows(image_x + bytes_x, pitch_x, k, j), rl = along(image_a + bytes_a, pitch_a, i, k);
                d = __builtin_amdgcn_mfma_f32_16x16x32_f16(p, r, d, 0, 0, 0);
                d = __builtin_amdgcn_mfma_f32_16x16x32_f16(p, rl, d, 0, 0, 0);
                d = __builtin_amdgcn_mfma_f32_16x16x32_f16(pl, r, d, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) x[s][r] = fmaf(d[r], on_sum, fmaf(b_diagonal[i + c], 1.0f / a.image[step], a.a[step]) * x[s][r]);
        }
    }
    const auto store = [&](auto* at, int64_t down, int64_t over, float scale) {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            uint32_t i, j;
            if (!tile(s, &i, &j) || i + c >= a.n) continue;
            const uint32_t row = i + c, col = j + 4 * q;
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r)
                if (col + r < a.m) at[row * down + (col + r) * over] = (std::remove_pointer_t<decltype(at)>)(x[s][r] * scale);
        }
    };
    O* out = reinterpret_cast<O*>(a.out.data) + (int64_t)matrix * a.out.batch;
    if (a.pauses) store(between, a.m, 1, 1.0f);
    else if (a.tall) store(out, 1, a.out.token, a.scale);
    else store(out, a.out.token, 1, a.scale);
}

// -------------------------------------------------------------------------------------------------------- host

// Workgroups that are at work at a time.
constexpr uint32_t slots_of(uint32_t tile) { return tile == 256 ? 256 : tile == 128 ? 512 : 1024; }

// Slices of a symmetric product's sums over k values.
uint32_t slices_of(uint32_t batch, uint32_t tile, uint32_t n, uint32_t k, bool split)
{
    if (tile == 256) return 1;
    const uint64_t side = (n + tile - 1) / tile, tiles = batch * (side * (side + 1) / 2), steps = k / (split ? 32 : 64);
    const uint64_t want = std::max<uint64_t>(1, slots_of(tile) / tiles), most = std::max<uint64_t>(1, steps / 8);
    return (uint32_t)std::min(want, most);
}

// Sides of the tiles of the symmetric products and of the updates: those whose rounds of workgroups take least.  Larger tiles read less for every product, smaller ones leave fewer
// compute units without one at the end.  us a step, the same sides for both: four of 2048 x 2048 in bf16 256 183, 128 193, 64 250; 48 of 768 x 768 217, 199, 228; one of 768 x 768
// 78, 38, 27; 4096 x 4096 310, 357, 552.
struct Tiles {
    uint32_t symmetric, update;
};

Tiles tiles_of(uint32_t batch, uint32_t n, uint32_t m, bool split)
{
    Tiles best{};
    double least = 0.0;
    const auto weight = [](uint32_t tile) { return tile == 256 ? 256.0 * 256.0 : tile == 128 ? 2.5 * 128.0 * 128.0 : 6.8 * 64.0 * 64.0; };
    const auto rounds = [](uint64_t tiles, uint32_t tile, uint32_t slices) { return (double)((tiles * slices + slots_of(tile) - 1) / slots_of(tile)) / slices; };
    for (const uint32_t s : {256u, 128u, 64u})
        for (const uint32_t u : {256u, 128u, 64u}) {
            const uint32_t whole = std::max(s, u), N = (n + whole - 1) / whole * whole, M = (m + whole - 1) / whole * whole;     // as they are filled up
            const uint64_t side = N / s, symmetric = batch * (side * (side + 1) / 2), update = (uint64_t)batch * (N / u) * (M / u);
            // a tile's start and end cost as much as so many values of k: with 256 no other workgroup of the compute unit multiplies meanwhile
            const auto longer = [](uint32_t k, uint32_t tile) { return (double)k + (tile == 256 ? 384 : tile); };
            const double cost = weight(s) * (rounds(symmetric, s, slices_of(batch, s, N, M, split)) * longer(M, s) +
                                             rounds(symmetric, s, slices_of(batch, s, N, N, split)) * longer(N, s)) +
                                weight(u) * rounds(update, u, 1) * longer(N, u);
            if (best.update == 0 || cost < least) best = Tiles{s, u}, least = cost;
        }
    return best;
}

// Sums of squares of a matrix: enough workgroups for all compute units.
uint32_t parts_of(uint32_t batch) { return std::max(8u, std::min(kMostParts, 2048u / batch)); }

// Whether images are two: for results in fp32, and of matrices of up to 256 rows (the fewer of rows and columns).  What one image costs most is a matrix of rank one, of which the diagonal of
// b A + c A^2 meets X and the rest of it X's image: 0.42 / rows of the results (root mean square), and up to 250 rows that is more than the 0.00166 of bf16's own rounding.  With one image and with
// two, with that rounding: 16 x 4000 0.021 and 0.0017, 64 x 64 0.0068 and 0.0017, 128 x 512 0.0037, 200 x 300 0.0028, 256 x 1024 0.0025; then 384 x 384 0.0020, 768 x 768 0.00175, 2048 x 2048 0.0017.  Of
// a momentum with noise 0.0017 to 0.0018 whatever the size.  us: 300 of 64 x 64 27 with one and 35 with two, 8 of 100 x 131 42, 62, 48 of 128 x 512 94, 161, 4 of 200 x 300 86, 109,
// 8 of 256 x 1024 101, 157, 8 of 768 x 768 203, 538.
constexpr uint32_t kMostSplit = 256;
bool is_split(uint32_t rows, uint32_t cols, sdl_dtype_t out) { return out == SDL_DTYPE_FP32 || std::min(rows, cols) <= kMostSplit; }

struct Layout {
    Work w;
    Tiles tiles;
    size_t squares, partial, bytes;
    uint32_t parts, gram_slices, poly_slices;
};

Layout layout_of(uint32_t batch, uint32_t rows, uint32_t cols, bool split)
{
    Layout l{};
    const uint32_t n = rows < cols ? rows : cols, m = rows < cols ? cols : rows;
    l.tiles = tiles_of(batch, n, m, split);
    const uint32_t whole = std::max(l.tiles.symmetric, l.tiles.update);
    Work& w = l.w;
    w.split = split;
    w.n = (n + whole - 1) / whole * whole;
    w.m = (m + whole - 1) / whole * whole;
    size_t at = 0;
    const auto place = [&at](size_t bytes) {
        const size_t here = at;
        at += (bytes + 127) / 128 * 128;
        return here;
    };
    w.x16 = place((size_t)w.n * w.pitch(w.m));
    w.x16_other = place((size_t)w.n * w.pitch(w.m));
    w.rest = place((size_t)w.n * w.m * (split ? 4 : 2));
    w.a16 = place((size_t)w.n * w.pitch(w.n));
    w.b16 = place((size_t)w.n * w.pitch(w.n));
    w.a_diagonal = place(w.n * sizeof(float));
    w.b_diagonal = place(w.n * sizeof(float));
    w.each = at;
    l.parts = parts_of(batch);
    l.squares = (size_t)batch * w.each;
    l.partial = l.squares + ((size_t)batch * l.parts * sizeof(double) + 127) / 128 * 128;
    l.gram_slices = slices_of(batch, l.tiles.symmetric, w.n, w.m, split);
    l.poly_slices = slices_of(batch, l.tiles.symmetric, w.n, w.n, split);
    const uint32_t slices = std::max(l.gram_slices, l.poly_slices), side = w.n / l.tiles.symmetric;
    l.bytes = l.partial + (slices > 1 ? (size_t)batch * (side * (side + 1) / 2) * slices * l.tiles.symmetric * l.tiles.symmetric * sizeof(float) : 0);
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
    // zeros of the derivative a + 3 b u + 5 c u^2: one from terms of the same sign, the other from the two's product, so that none is lost where c is next to nothing.
    // One that is infinite or no number is none.
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (d >= 0.0) {
        const double q = -0.5 * (3.0 * b + std::copysign(std::sqrt(d), b));
        look(q / (5.0 * c));
        look(a / q);
    }
    return most;
}

// Of the matrix b A + c A^2, where no singular value of X is above h: as much as fp16 has room for.
float image_scale(double b, double c, double h)
{
    const double bound = std::fabs(b) * h * h + std::fabs(c) * h * h * h * h;
    return (float)std::exp2(std::min(14.0, std::floor(std::log2(32768.0 / std::max(bound, 1e-30)))));
}

template <int TILE, bool SPLIT, int MODE, typename O>
int product_of(const ProductArgs& a, uint32_t batch, hipStream_t st)
{
    const uint32_t groups = batch * a.tiles.d;
    if constexpr (MODE != UPDATE && TILE != 256) {
        if (a.slice_of.d > 1) {
            hipLaunchKernelGGL((sdl_orthogonalize_product_kernel<TILE, SPLIT, MODE, PART, O>), dim3(groups * a.slice_of.d), dim3(256), 0, st, a);
            if (launched() != SDL_OK) return SDL_ERR_DEVICE;
            hipLaunchKernelGGL((sdl_orthogonalize_product_kernel<TILE, SPLIT, MODE, JOIN, O>), dim3(groups), dim3(256), 0, st, a);
            return launched();
        }
    }
    hipLaunchKernelGGL((sdl_orthogonalize_product_kernel<TILE, SPLIT, MODE, WHOLE, O>), dim3(groups), dim3(256), 0, st, a);
    return launched();
}

template <bool SPLIT, int MODE, typename O>
int product(const ProductArgs& a, uint32_t tile, uint32_t batch, hipStream_t st)
{
    return tile == 256 ? product_of<256, SPLIT, MODE, O>(a, batch, st) : tile == 128 ? product_of<128, SPLIT, MODE, O>(a, batch, st) : product_of<64, SPLIT, MODE, O>(a, batch, st);
}

template <bool SPLIT, typename O>
int steps_of(const Layout& l, uint32_t batch, uint32_t rows, uint32_t cols, const float* coefficients, uint32_t steps, float scale, const sdl_view_t* out,
             hipStream_t st)
{
    const Work& w = l.w;
    const uint32_t per = SPLIT ? 32 : 64, side = w.n / l.tiles.symmetric, down = w.n / l.tiles.update, across = w.m / l.tiles.update;
    size_t now = w.x16, other = w.x16_other;
    double h = 1.0;
    for (uint32_t s = 0; s < steps; ++s) {
        const float* each = coefficients + 3 * (size_t)s;
        const double ca = each[0], cb = each[1], cc = each[2];
        const float scale_b = image_scale(cb, cc, h);
        h = reach(ca, cb, cc, h);
        ProductArgs a{};
        a.w = w;
        a.partial = reinterpret_cast<f32x4_t*>(w.base + l.partial);
        a.slice_of = make_div(l.gram_slices);
        a.p = a.q = now;
        a.t = w.a16;
        a.pitch_p = a.pitch_q = w.pitch(w.m);
        a.steps = w.m / per;
        a.tiles = make_div(side * (side + 1) / 2);
        a.on_sum = kScaleA / (kScaleX * kScaleX);
        if (product<SPLIT, GRAM, float>(a, l.tiles.symmetric, batch, st) != SDL_OK) return SDL_ERR_DEVICE;
        a.slice_of = make_div(l.poly_slices);
        a.p = a.q = w.a16;
        a.t = w.b16;
        a.pitch_p = a.pitch_q = w.pitch(w.n);
        a.steps = w.n / per;
        a.on_old = (float)(cb / kScaleA * scale_b);
        a.on_sum = (float)(cc / ((double)kScaleA * kScaleA) * scale_b);
        if (product<SPLIT, POLY, float>(a, l.tiles.symmetric, batch, st) != SDL_OK) return SDL_ERR_DEVICE;
        a.p = w.b16;
        a.q = now;
        a.t = other;
        a.pitch_q = w.pitch(w.m);
        a.tiles = make_div(down * across);
        a.across = make_div(across);
        a.last = s + 1 == steps;
        const double to = a.last ? scale : 1.0;
        a.on_old = (float)(ca * to);
        a.on_sum = (float)(to / ((double)scale_b * kScaleX));
        a.out = kernel_view(out);
        a.tall = rows > cols;
        a.rows = rows;
        a.cols = cols;
        if (product<SPLIT, UPDATE, O>(a, l.tiles.update, batch, st) != SDL_OK) return SDL_ERR_DEVICE;
        std::swap(now, other);
    }
    return SDL_OK;
}

// Wavefronts of a workgroup, tiles of X that each of them keeps, and shared memory of the kernels of small matrices.  A step is five stretches between barriers, of which a wavefront's
// tiles come one after the other: the more wavefronts the shorter, down to a tile each, and for many matrices as few as fill the compute units.  us, with 8 and 16 wavefronts:
// 30 of 64 x 64 26.3, 23.1; 300 34.7, 43.6; 4000 187, 330.  2000 of 24 x 24 with 4 wavefronts 28, with 16 100; with room for four tiles of a wavefront 30 instead of 23 for one.
struct Small {
    uint32_t waves, slots, bytes;
};
constexpr Small kSmall[] = {{4, 1, 15 * 1024}, {8, 2, 39 * 1024}, {8, 6, 39 * 1024}, {16, 2, 39 * 1024}, {16, 4, 159 * 1024}, {16, 6, 159 * 1024}, {16, 10, 159 * 1024}};

bool fits(const Small& k, uint32_t n, uint32_t m)
{
    const uint64_t down = (n + 15) / 16, across = (m + 15) / 16, nk = (n + 31) / 32 * 32, mk = (m + 31) / 32 * 32;
    return 2 * nk * (mk * 2 + 16 + nk * 2 + 16) + 2 * nk * 4 <= k.bytes && down * across <= k.waves * k.slots && down * (down + 1) / 2 <= k.waves * kHalves;
}

bool is_small(uint32_t n, uint32_t m)
{
    return std::any_of(std::begin(kSmall), std::end(kSmall), [=](const Small& k) { return fits(k, n, m); });
}
static_assert(2 * (kMostSplit + 1) * (kMostSplit + 1) * 2 > 160 * 1024, "matrices that have one image are not small");

// What a call is to be given, whatever its steps: X of small matrices in fp32, between launches of kMostSmallSteps steps each (with the layout of the others 65535 matrices of 16 x 16
// had to come with 5.4 GB, and this is 67 MB).
size_t workspace_of(uint32_t batch, uint32_t rows, uint32_t cols, bool split)
{
    const uint32_t n = std::min(rows, cols), m = std::max(rows, cols);
    return is_small(n, m) ? (size_t)batch * n * m * sizeof(float) : layout_of(batch, rows, cols, split).bytes;
}

template <typename T, typename O>
int small(const SmallArgs& a, uint32_t batch, hipStream_t st)
{
#define SDL_LAUNCH(N) \
    hipLaunchKernelGGL((sdl_orthogonalize_small_kernel<T, O, kSmall[N].waves, kSmall[N].slots, kSmall[N].bytes>), dim3(batch), dim3(kSmall[N].waves * kWave), 0, st, a)
    // more than one for a compute unit, or too few tiles for sixteen wavefronts
    const bool many = batch > 256 || ((a.n + 15) / 16) * ((a.m + 15) / 16) < 16;
    if (many && fits(kSmall[0], a.n, a.m)) SDL_LAUNCH(0);
    else if (many && fits(kSmall[1], a.n, a.m)) SDL_LAUNCH(1);
    else if (many && fits(kSmall[2], a.n, a.m)) SDL_LAUNCH(2);
    else if (fits(kSmall[3], a.n, a.m)) SDL_LAUNCH(3);
    else if (fits(kSmall[4], a.n, a.m)) SDL_LAUNCH(4);
    else if (fits(kSmall[5], a.n, a.m)) SDL_LAUNCH(5);
    else SDL_LAUNCH(6);
#undef SDL_LAUNCH
    return launched();
}

template <typename T>
int small_of(const SmallArgs& a, sdl_dtype_t out, uint32_t batch, hipStream_t st)
{
    return out == SDL_DTYPE_FP32 ? small<T, float>(a, batch, st) : small<T, __bf16>(a, batch, st);
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
    return workspace_of(batch, rows, cols, is_split(rows, cols, out_dtype));
}

int sdl_orthogonalize(const sdl_view_t* x, uint32_t batch, uint32_t rows, uint32_t cols, sdl_dtype_t dtype, const float* coefficients, uint32_t steps, float eps,
                      float scale, const sdl_view_t* out, sdl_dtype_t out_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!known(dtype) || !known(out_dtype) || steps == 0 || !coefficients) return SDL_ERR_INVALID_ARG;
    if (!(eps >= 0.0f && eps - eps == 0.0f) || !(scale - scale == 0.0f)) return SDL_ERR_INVALID_ARG;
    double h = 1.0;
    for (uint32_t s = 0; s < steps; ++s) {
        h = reach(coefficients[3 * (size_t)s], coefficients[3 * (size_t)s + 1], coefficients[3 * (size_t)s + 2], h);
        if (!(h <= 2.0)) return SDL_ERR_INVALID_ARG;
    }
    int rc = check_shape(batch, rows, cols);
    if (rc != SDL_OK || batch == 0 || rows == 0 || cols == 0) return rc;
    if ((rc = check_view(x, dtype)) != SDL_OK || (rc = check_output(out, out_dtype, batch, rows, 1)) != SDL_OK) return rc;
    // in x's place only as x lies there: a small matrix may be written before another one is read
    if (out->data == x->data && (out_dtype != dtype || (batch > 1 && out->stride_batch != x->stride_batch) || (rows > 1 && out->stride_token != x->stride_token)))
        return SDL_ERR_INVALID_ARG;
    const bool split = is_split(rows, cols, out_dtype);
    if (!workspace || workspace_bytes < workspace_of(batch, rows, cols, split)) return SDL_ERR_INVALID_ARG;
    if (!aligned_to(workspace, 16)) return SDL_ERR_ALIGNMENT;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t n = rows < cols ? rows : cols, m = rows < cols ? cols : rows;
    if (is_small(n, m)) {
        SmallArgs a{kernel_view(x), kernel_view(out), make_div((m + 15) / 16), rows > cols, n, m, 0, (double)eps, scale, static_cast<float*>(workspace), 0, 0, {}, {}, {}, {}};
        h = 1.0;
        const float* each = coefficients;
        for (uint32_t left = steps; left; left -= a.steps) {
            a.steps = std::min(kMostSmallSteps, left);
            a.resumes = left < steps;
            a.pauses = left > a.steps;
            for (uint32_t s = 0; s < a.steps; ++s, each += 3) {
                a.a[s] = each[0];
                a.b[s] = each[1];
                a.c[s] = each[2];
                a.image[s] = image_scale(a.b[s], a.c[s], h);
                h = reach(a.a[s], a.b[s], a.c[s], h);
            }
            rc = dtype == SDL_DTYPE_BF16 ? small_of<__bf16>(a, out_dtype, batch, st) : small_of<float>(a, out_dtype, batch, st);
            if (rc != SDL_OK) return rc;
        }
        return SDL_OK;
    }
    Layout l = layout_of(batch, rows, cols, split);
    l.w.base = static_cast<char*>(workspace);
    FirstArgs a{};
    a.x = kernel_view(x);
    a.rows = rows;
    a.cols = cols;
    a.tall = rows > cols;
    a.parts = l.parts;
    a.groups = make_div((cols + 7) / 8);
    a.squares = reinterpret_cast<double*>(l.w.base + l.squares);
    a.eps = (double)eps;
    a.w = l.w;
    if (dtype == SDL_DTYPE_BF16) rc = split ? first<__bf16, true>(a, batch, st) : first<__bf16, false>(a, batch, st);
    else rc = split ? first<float, true>(a, batch, st) : first<float, false>(a, batch, st);
    if (rc != SDL_OK) return rc;
    if (out_dtype == SDL_DTYPE_FP32) return steps_of<true, float>(l, batch, rows, cols, coefficients, steps, scale, out, st);
    return split ? steps_of<true, __bf16>(l, batch, rows, cols, coefficients, steps, scale, out, st) : steps_of<false, __bf16>(l, batch, rows, cols, coefficients, steps, scale, out, st);
}

}  // extern "C"
