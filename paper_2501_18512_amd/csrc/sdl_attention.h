// Device code that attention's forward and backward kernels share (gfx950).  Internal to csrc/.
//
// Layouts of the 32x32 matrix instructions, for lane l, half = l / 32, c = l % 32:
//   A (32 x 16)  row c,    k = 8 half + j        B (16 x 32)  column c, k = 8 half + j        j = 0..7
//   D (32 x 32)  column c, row 8 (i / 4) + 4 half + i % 4                                     i = 0..15
// The sum over k may run in any order as long as A and B agree on it.  Eight registers i = 8 u .. 8 u + 7 of a D tile hold the rows
// 16 u + order(half, j) of their column, order(half, j) = 8 (j / 4) + 4 half + j % 4: they are a B operand of a second product, as
// they stand, whose A operand takes its k in that order.  So the scores are formed with the queries (or keys) that a
// lane keeps as columns, and probabilities never move between lanes.
#pragma once

#include "sdl_operand.h"

namespace sdl_device {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Kernels come for widths of 32, 64, 96 and 128, tiles of shared memory have rows of 64 or 128.
constexpr int tile_width(int width) { return width <= 64 ? 64 : 128; }

// One operand of a product over 16 values of k: eight elements a lane.
template <typename T> struct Frag;
template <> struct Frag<__bf16> { bf16x8_t v; };
template <> struct Frag<float> { float v[8]; };

__device__ __forceinline__ void mma(f32x16_t& d, const Frag<__bf16>& a, const Frag<__bf16>& b)
{
    d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, d, 0, 0, 0);
}
// fp32: one instruction has k = 0, 1 in the two halves; the j-th takes k = j and 8 + j
__device__ __forceinline__ void mma(f32x16_t& d, const Frag<float>& a, const Frag<float>& b)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) d = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], d, 0, 0, 0);
}

// The 16x16 instructions, 32 values of k: lane l has row or column l % 16 and k = 8 (l / 16) + j; D is column l % 16, rows 4 (l / 16) + i.
__device__ __forceinline__ void mma16(f32x4_t& d, const Frag<__bf16>& a, const Frag<__bf16>& b)
{
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, d, 0, 0, 0);
}
__device__ __forceinline__ void mma16(f32x4_t& d, const Frag<float>& a, const Frag<float>& b, int n = 8)
{
#pragma unroll
    for (int j = 0; j < n; ++j) d = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], d, 0, 0, 0);
}

__device__ __forceinline__ void set_frag(Frag<__bf16>& f, const Eight<__bf16>& x) { f.v = __builtin_bit_cast(bf16x8_t, x.w); }
__device__ __forceinline__ void set_frag(Frag<float>& f, const Eight<float>& x)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = x.get(j);
}

// Registers 8 u .. 8 u + 7 of a D tile as an operand.  bf16: probabilities and their gradients are rounded to nearest here, as the matrix instructions take both operands in one
// type; the sums over them stay in fp32.  Two such parts a number would keep 16 bits for twice the products behind the softmax.  Error against 64 bits, where the inputs' type
// costs the results one rounding as well: out 0.0020 for 0.0015 with nothing else rounded (a prompt of 8192), 0.00029 for 0.00022 (one query, lse in the mean); all results of a forward and backward
// pass 0.0024 for 0.0017.
__device__ __forceinline__ Frag<__bf16> frag_of(const f32x16_t& d, int u, __bf16)
{
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = pack_bf16(d[8 * u + 2 * j], d[8 * u + 2 * j + 1]);
    return Frag<__bf16>{__builtin_bit_cast(bf16x8_t, w)};
}
__device__ __forceinline__ Frag<float> frag_of(const f32x16_t& d, int u, float)
{
    Frag<float> f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = d[8 * u + j];
    return f;
}

// The same number, for the compiler another one every time: what is worked out from it is worked out there, and not kept in registers through a loop.
__device__ __forceinline__ int anew(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// A tile of rows of HD elements in shared memory, as the copies below can lay it down: groups of 1024 bytes, 16 bytes apart, and within a
// group the 16-byte pieces of row x swapped around by an xor of some of their number's bits with a value of x.  Neither the reads along rows (eight lanes,
// eight rows, one piece) nor the ones across them (four rows, four pieces) meet in a bank, and the offsets of a lane's reads differ by
// constants but for a few.
template <typename T, int HD>
struct Tile {
    static constexpr int kPieces = HD * (int)sizeof(T) / 16;     // of a row
    static constexpr int kGroup = kWave / kPieces;                // rows of a group
    static constexpr int kGroupBytes = kWave * 16 + 16;
    static constexpr int kMask = kPieces == 8 ? 6 : kPieces == 16 ? 12 : 4;
    static_assert(kPieces == 8 || kPieces == 16 || kPieces == 32, "widths of 64 and 128");

    static constexpr int bytes(int rows) { return rows / kGroup * kGroupBytes; }
    static __device__ __forceinline__ int swap(int x)
    {
        return kPieces == 8 ? ((x & 2) << 1) | ((x & 4) >> 1) : x << 2;
    }
    static __device__ __forceinline__ int place(int x, int p) { return ((p & kMask) ^ swap(x)) + (p & ~kMask); }    // its own inverse
    static __device__ __forceinline__ int at(int r, int p)
    {
        const int x = r % kGroup;
        return r / kGroup * kGroupBytes + x * (kPieces * 16) + place(x, p) * 16;
    }

    static __device__ __forceinline__ void put(char* tile, int r, int c8, const Eight<T>& v)
    {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u32x4*>(tile + at(r, c8)) = v.w;
        } else {
            *reinterpret_cast<u32x4*>(tile + at(r, 2 * c8)) = v.lo;
            *reinterpret_cast<u32x4*>(tile + at(r, 2 * c8 + 1)) = v.hi;
        }
    }
    // elements [8 c8, 8 c8 + 8) of row r
    static __device__ __forceinline__ Frag<T> along(const char* tile, int r, int c8)
    {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            f.v = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(tile + at(r, c8)));
        } else {
            const u32x4 a = *reinterpret_cast<const u32x4*>(tile + at(r, 2 * c8)), b = *reinterpret_cast<const u32x4*>(tile + at(r, 2 * c8 + 1));
#pragma unroll
            for (int j = 0; j < 4; ++j) f.v[j] = u2f(a[j]), f.v[4 + j] = u2f(b[j]);
        }
        return f;
    }
    // For the 16x16 instructions: column d0 + lane % 16 of the rows 4 (lane / 16) + i and, bf16, 16 more, i = 0..3.
    static __device__ __forceinline__ Frag<T> across16(const char* tile, int d0)
    {
        const int lane = threadIdx.x & (kWave - 1), quarter = lane >> 4;
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
            const int r = 4 * quarter + ((lane & 15) >> 2), p = (d0 >> 3) + ((lane & 2) >> 1), q = (lane & 1) * 8;
            const i16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(tile + at(r, p) + q));
            const i16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(tile + at(r + 16, p) + q));
            const bf16x4_t x = __builtin_bit_cast(bf16x4_t, a), y = __builtin_bit_cast(bf16x4_t, b);
            f.v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            const int d = d0 + (lane & 15);
#pragma unroll
            for (int i = 0; i < 4; ++i) f.v[i] = u2f(*reinterpret_cast<const uint32_t*>(tile + at(4 * quarter + i, d >> 2) + (d & 3) * 4));
        }
        return f;
    }
    // column d0 + lane % 32 of the rows r0 + order(half, j), r0 a multiple of 16.  bf16: the transposing read gives lane i of 16 the i-th
    // column of a block of 4 rows and 16 columns, of which lane 4 r + q names the q-th quarter of row r.
    static __device__ __forceinline__ Frag<T> across(const char* tile, int r0, int d0, int lane)
    {
        const int half = lane >> 5;
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
            const int r = 4 * half + ((lane & 15) >> 2), p = (d0 >> 3) + ((lane & 16) >> 3) + ((lane & 2) >> 1), q = (lane & 1) * 8;
            const i16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(tile + at(r0 + r, p) + q));
            const i16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(tile + at(r0 + r + 8, p) + q));
            const bf16x4_t x = __builtin_bit_cast(bf16x4_t, a), y = __builtin_bit_cast(bf16x4_t, b);
            f.v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            const int d = d0 + (lane & 31);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = r0 + 8 * (j / 4) + 4 * half + j % 4;
                f.v[j] = u2f(*reinterpret_cast<const uint32_t*>(tile + at(r, d >> 2) + (d & 3) * 4));
            }
        }
        return f;
    }
};

// The same reads of a tile named by its offset in shared memory, from offsets of the lane that are worked out once: in bf16 a read's address is one of a few
// registers and a constant.  Rows are named by the first of a group of 32, of which `along` reads the lane's.  For the kernel of dk and dv, whose registers are full: it
// spent half of its vector instructions on addresses.  The others have registers for what the compiler keeps of Tile's reads, and gain nothing.
template <typename T, int HD>
struct LaneReads {
    typedef Tile<T, HD> Smem;
    int lane;
    __device__ __forceinline__ LaneReads(int lane_) : lane(lane_) {}
    static __device__ __forceinline__ const char* tile_at(uint32_t tile)
    {
        return (const char*)(const __attribute__((address_space(3))) char*)(uintptr_t)tile;
    }
    __device__ __forceinline__ Frag<T> along(uint32_t tile, int r0, int i) const { return Smem::along(tile_at(tile), r0 + (lane & 31), 2 * i + (lane >> 5)); }
    __device__ __forceinline__ Frag<T> across(uint32_t tile, int r0, int n) const { return Smem::across(tile_at(tile), r0, n * 32, lane); }
};
template <int HD>
struct LaneReads<__bf16, HD> {
    typedef Tile<__bf16, HD> Smem;
    static constexpr int kStep = Smem::kMask & -Smem::kMask;        // pieces that keep their order
    uint32_t along_[4], across_[HD / 32];
    __device__ __forceinline__ LaneReads(int lane)
    {
        const int c = lane & 31, half = lane >> 5, r = 4 * half + ((lane & 15) >> 2), p = ((lane & 16) >> 3) + ((lane & 2) >> 1);
#pragma unroll
        for (int k = 0; k < 4; ++k) along_[k] = (uint32_t)anew(Smem::at(c, k * kStep + half));
#pragma unroll
        for (int n = 0; n < HD / 32; ++n) across_[n] = (uint32_t)anew(Smem::at(r, n * 4 + p) + (lane & 1) * 8);
    }
    __device__ __forceinline__ Frag<__bf16> along(uint32_t tile, int r0, int i) const
    {
        typedef const __attribute__((address_space(3))) u32x4 lds_u32x4;
        const uint32_t at = along_[2 * i / kStep] + tile + r0 / Smem::kGroup * Smem::kGroupBytes + 2 * i % kStep * 16;
        return Frag<__bf16>{__builtin_bit_cast(bf16x8_t, *(lds_u32x4*)(uintptr_t)at)};
    }
    __device__ __forceinline__ Frag<__bf16> across(uint32_t tile, int r0, int n) const
    {
        typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
        const uint32_t at = across_[n] + tile + r0 / Smem::kGroup * Smem::kGroupBytes;
        const i16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)at);
        const i16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(uintptr_t)(at + 8 / Smem::kGroup * Smem::kGroupBytes));
        const bf16x4_t x = __builtin_bit_cast(bf16x4_t, a), y = __builtin_bit_cast(bf16x4_t, b);
        return Frag<__bf16>{__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7)};
    }
};

template <typename T>
__device__ __forceinline__ T* at_row(const View& v, uint32_t b, uint32_t token, uint32_t head)
{
    return reinterpret_cast<T*>(v.data) + ((int64_t)b * v.batch + (int64_t)token * v.token + (int64_t)head * v.head);
}

// Copies of tiles into shared memory that bypass the registers: a wavefront's instruction brings 64 pieces of 16 bytes, which land
// one behind the other, so that the rearrangement of a row's pieces is made in the addresses they come from.  The compiler does not see these
// copies: loads_done() is to come before the barrier after which a tile is read.
__device__ __forceinline__ uint32_t lds_offset(const void* p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// (ONCE: data that no one reads again goes past the caches.)
template <bool ONCE>
__device__ __forceinline__ void copy_piece(const char* base, uint32_t offset, uint32_t to)
{
    // Five wait states between a vector instruction that writes a scalar register (the base may come from a lane) and the load that reads it, of which the write of m0 is one: the
    // compiler does not look in here.  m0 itself needs one; the compiler holds nothing in that register from one instruction to the next (naming it as overwritten is warned
    // of for that reason), and these kernels have no other instruction that reads it.  The wait costs 0 to 1 % of a kernel.
    if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %1 nt" : : "v"(offset), "s"(base), "s"(to) : "memory");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(to) : "memory");
}
// Four bytes a lane, from any addresses.
__device__ __forceinline__ void copy_word(const float* from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(from), "s"(to) : "memory");
}
__device__ __forceinline__ void own_loads_done() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory"); }
// Waits for this wavefront's copies and reads of shared memory, then for the workgroup.
__device__ __forceinline__ void loads_done()
{
    own_loads_done();
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// A workgroup of WAVES wavefronts brings tiles of ROWS consecutive tokens of one head.  The offset of a lane's piece from the first row of
// its share is the same in every tile, unsigned and under 2^32: ASYNC is for rows that start on 16 bytes and lie less than 2^24 bytes apart, up to 256 of them.  The other way
// takes any element alignment and any distance and goes through registers.
template <typename T, int HD, int ROWS, int WAVES, bool ASYNC, bool ONCE = false>
struct TileCopy {
    typedef Tile<T, HD> Smem;
    static constexpr int kPieces = Smem::kPieces;
    static constexpr int kStep = Smem::kGroup * WAVES;                      // rows of all wavefronts' instructions
    static constexpr int kCopies = ROWS / kStep;
    static_assert(ROWS % kStep == 0, "whole copies");
    static_assert(!ASYNC || ROWS <= 256, "offsets of 32 bits");

    const char* base;       // first row of the head
    int64_t stride;         // bytes between tokens
    uint32_t width;         // elements of a row

    __device__ __forceinline__ TileCopy(const View& v, uint32_t b, uint32_t head, uint32_t width_)
    {
        base = reinterpret_cast<const char*>(at_row<T>(v, b, 0, head));
        stride = v.token * (int64_t)sizeof(T);
        width = width_;
    }
    // Once: pieces behind the width are never brought, and have to be zero.
    __device__ __forceinline__ void clear(char* tile) const
    {
        if (!ASYNC || width == HD) return;
        for (int i = threadIdx.x; i < ROWS * kPieces; i += WAVES * kWave)
            if ((i % kPieces) * 16 >= (int)(width * sizeof(T))) *reinterpret_cast<u32x4*>(tile + Smem::at(i / kPieces, i % kPieces)) = u32x4{0, 0, 0, 0};
    }
    // Rows [row0, row0 + ROWS) of `rows`; what lies behind the last row is that row again.
    __device__ __forceinline__ void bring(char* tile, int32_t row0, int32_t rows) const
    {
        if constexpr (ASYNC) {
            const uint32_t lane = threadIdx.x & (kWave - 1), wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
            const uint32_t row = wave * Smem::kGroup + lane / kPieces, to = lds_offset(tile) + wave * Smem::kGroupBytes;
            const uint32_t piece = (uint32_t)Smem::place(lane / kPieces, lane % kPieces);       // that comes to lie where the lane's 16 bytes land
            const char* from = base + row0 * stride;
            if (row0 + ROWS <= rows && width == HD) {
#pragma unroll
                for (int i = 0; i < kCopies; ++i) copy_piece<ONCE>(from + i * kStep * stride, row * (uint32_t)stride + piece * 16, to + i * (WAVES * Smem::kGroupBytes));
            } else if (piece * 16 < width * sizeof(T)) {
#pragma unroll
                for (int i = 0; i < kCopies; ++i)
                    copy_piece<ONCE>(from, min(row + i * kStep, (uint32_t)(rows - 1 - row0)) * (uint32_t)stride + piece * 16, to + i * (WAVES * Smem::kGroupBytes));
            }
        } else {
#pragma unroll 4
            for (int i = threadIdx.x; i < ROWS * (HD / 8); i += WAVES * kWave) {
                const int r = i / (HD / 8), c8 = i % (HD / 8);
                const T* from = reinterpret_cast<const T*>(base + (int64_t)min(row0 + r, rows - 1) * stride);
                Smem::put(tile, r, c8, load8_ends(from, c8 * 8, width));
            }
        }
    }
};

// Host: whether the tiles of a view may be brought by the asynchronous copies (whose kernels take rows of whole groups of eight elements).
inline bool async_rows(const View& v, uint32_t width, size_t size)
{
    const int64_t bytes = v.token * (int64_t)size;
    return aligned_to(v.data, 16) && width % 8 == 0 && v.batch * (int64_t)size % 16 == 0 && v.head * (int64_t)size % 16 == 0 &&
           bytes % 16 == 0 && bytes >= 0 && bytes < (1 << 24);
}

// x of lane l and of lane l ^ 32
__device__ __forceinline__ float half_max(float x)
{
    const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(f2u(x), f2u(x), false, false));
    return fmaxf(u2f(p[0]), u2f(p[1]));
}
__device__ __forceinline__ float half_sum(float x)
{
    const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(f2u(x), f2u(x), false, false));
    return u2f(p[0]) + u2f(p[1]);
}

// the same over the four lanes l % 16, + 16, + 32, + 48
__device__ __forceinline__ float quarter_max(float x)
{
    const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(f2u(x), f2u(x), false, false));
    return half_max(fmaxf(u2f(p[0]), u2f(p[1])));
}
__device__ __forceinline__ float quarter_sum(float x)
{
    const u32x2 p = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(f2u(x), f2u(x), false, false));
    return half_sum(u2f(p[0]) + u2f(p[1]));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Four neighbouring elements of a row of n from element `at` on.  WHOLE: n is a multiple of four.
template <bool WHOLE = false, typename T>
__device__ __forceinline__ void store4(T* row, uint32_t at, uint32_t n, float a, float b, float c, float d)
{
    if constexpr (WHOLE) {
        if (at >= n) return;
        n = at + 4;
    }
    if (at + 4 <= n) {
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<u32x2_elem*>(row + at) = u32x2_elem{pack_bf16(a, b), pack_bf16(c, d)};
        else
            *reinterpret_cast<u32x4_f32elem*>(row + at) = u32x4_f32elem{f2u(a), f2u(b), f2u(c), f2u(d)};
        return;
    }
    const float v[4] = {a, b, c, d};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (at + j < n) row[at + j] = (T)v[j];
}

// The problem, as every kernel takes it.  The query heads of a key head are taken together: row r of a (batch, key head)
// is query token r / group, head r % group of the group, so that keys and values are read once for all of them and the
// gradients of a shared head are one sum.
struct Attention {
    View q, k, v, out, d_out, dq, dk, dv;
    float* lse;                 // [batch][heads][queries]
    float* row_stats;           // backward: -lse and -D, of that shape each, in the workspace
    const int32_t* q_len;
    const int32_t* k_len;
    Div group;                  // query heads of a key head
    uint32_t queries, keys, kv_heads, width, batch;
    float scale, scale_log2;    // and times log2(e)
    uint32_t causal;
    uint32_t spread;            // all keys and values fit the cache of a die (4 MB)
};

// One (batch, key head) of it: valid lengths, and which keys a row sees.  The last valid query stands at the last valid key.
struct Sequence {
    uint32_t b, g;
    int32_t nq, nk;             // valid queries, keys
    int32_t shift;              // query t sees keys up to t + shift (causal)

    __device__ __forceinline__ Sequence(const Attention& a, uint32_t b_, uint32_t g_) : b(b_), g(g_)
    {
        nq = (int32_t)a.queries;
        nk = (int32_t)a.keys;
        if (a.q_len) nq = min(nq, max(a.q_len[b], 0));
        if (a.k_len) nk = min(nk, max(a.k_len[b], 0));
        shift = nk - nq;
    }
    // keys that valid query t sees: [0, seen(t))
    __device__ __forceinline__ int32_t seen(const Attention& a, int32_t t) const
    {
        return a.causal ? max(0, min(nk, t + shift + 1)) : nk;
    }
    // keys that one at least of `n` rows from `row` on sees
    __device__ __forceinline__ int32_t most_seen(const Attention& a, uint32_t row, uint32_t n) const
    {
        const uint32_t rows = a.queries * a.group.d;
        if (row >= rows || nq == 0) return 0;
        const int32_t first = (int32_t)div(row, a.group), last = min((int32_t)div(min(row + n, rows) - 1, a.group), nq - 1);
        return last < first ? 0 : seen(a, last);
    }
};

// A launch takes less than 2^32 threads along x.  Workgroups are numbered through rows of kGridX of them (a multiple of the dies, and 2^31 threads at 512 each); those of the last
// row that are too many have nothing to do.
constexpr uint32_t kGridX = 1u << 22;
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * kGridX + blockIdx.x; }
inline dim3 grid_of(uint64_t groups) { return groups <= kGridX ? dim3((uint32_t)groups) : dim3(kGridX, (uint32_t)((groups + kGridX - 1) / kGridX)); }

// Consecutive workgroups go to different compute dies (eight, each with its own cache of 16 channels, which take turns every 256 bytes).  The `each`
// workgroups of a unit, a (batch, key head), read the same keys and values and stay on two dies.  Where the rows of a head lie 4 KB apart, as 16
// heads of 128 do, all of them are in one channel: so a pair of dies has 16 units at work at a time, each die a half of every unit's workgroups,
// and, as a pair's units move on by one head from row to row of four and once more every four rows, they are of different heads (and of all
// sequences, whose lengths may differ).  Units that are left over are spread over all dies, and so are all of them where every die's cache has room
// for all (`spread`): lengths that differ between a few units would leave dies idle.
struct Place {
    uint32_t unit, within;

    __device__ __forceinline__ Place(uint32_t id, uint32_t units, uint32_t each, bool spread)
    {
        const uint32_t rows = spread ? 0 : units >> 2, left = units - rows * 4, of_pair = rows * each;
        if (id < 4 * of_pair) {
            const bool odd_one = id >= of_pair / 2 * 8;         // the last of every pair, where their number is odd
            const uint32_t die = id & 7u, pair = odd_one ? id - of_pair / 2 * 8 : die >> 1, x = odd_one ? of_pair - 1 : (id >> 3) * 2 + (die & 1u);
            const uint32_t set = x / (16 * each), in_set = x - set * 16 * each, n = min(16u, rows - 16 * set);
            within = in_set / n;
            uint32_t i = in_set - within * n;
            if ((n & 1u) == 0) i ^= within & 1u;                // or a die would see every other unit only
            const uint32_t row = set * 16 + i;
            unit = row * 4 + ((pair - row - (row >> 2)) & 3u);
        } else {
            const uint32_t rest = id - 4 * of_pair;
            within = rest / left;
            unit = rows * 4 + (rest - within * left + within) % left;       // moves on, or eight units would keep to a die each
        }
    }
};

// A small problem that is cut into splits: the workgroups that have something to do come first, or two of them would share a compute unit while others had none
// (a unit that is done with an empty one takes the next).  How many splits of a (unit, block) are of use depends on the lengths, so every wavefront counts them for
// itself, 64 pairs at a time, until it comes to workgroup `id`; false: there are fewer.  Four causal fp32 sequences of 1, 173, 345 and 517 tokens, 6 heads over 2 of width
// 80: forward 24 -> 17 us, dq 32 -> 22, dk and dv 46 -> 30.
template <typename Count>
__device__ __forceinline__ bool pick_item(uint32_t id, uint32_t units, uint32_t blocks, Count count, uint32_t& unit, uint32_t& nth_block, uint32_t& split)
{
    const uint32_t lane = threadIdx.x & (kWave - 1), pairs = units * blocks;
    for (uint32_t first = 0; first < pairs; first += kWave) {
        const uint32_t i = min(first + lane, pairs - 1), b = i / units, u = i - b * units;
        const uint32_t n = first + lane < pairs ? count(u, b) : 0;
        const uint32_t upto = lane_scan(n);
        const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)upto, kWave - 1);
        if (id < all) {
            const int who = __builtin_popcountll(__ballot(upto <= id));
            unit = (uint32_t)__builtin_amdgcn_readlane((int)u, who);
            nth_block = (uint32_t)__builtin_amdgcn_readlane((int)b, who);
            split = id - (uint32_t)__builtin_amdgcn_readlane((int)(upto - n), who);
            return true;
        }
        id -= all;
    }
    return false;
}
// Host: where that pays.
inline bool pick_items(const Attention& p, uint64_t blocks, uint32_t splits)
{
    return p.spread && splits > 1 && (p.causal || p.q_len || p.k_len) && blocks * p.batch * p.kv_heads <= 256;
}

// Host: whether the kernels take such a problem.
inline bool sdl_attention_shape(uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads, uint32_t width, sdl_dtype_t dtype)
{
    constexpr uint64_t kMost = 0x40000000u;
    return known(dtype) && kv_heads != 0 && heads % kv_heads == 0 && width != 0 && width <= SDL_ATTENTION_MAX_WIDTH && keys <= kMost &&
           (uint64_t)queries * heads <= kMost && (uint64_t)batch * heads <= kMost;
}

// Host: the checks that do not look at the arrays, and the arguments that do not depend on the pass.
inline int sdl_attention_problem(Attention& p, uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads,
                                 uint32_t width, sdl_dtype_t dtype, float scale, int causal, const int32_t* q_len, const int32_t* k_len)
{
    // from 2^-100 on, the backward pass' lse / scale fits as well; up to 2^127, the scale times log2(e)
    if (!(scale >= 0x1p-100f) || scale > 0x1p127f || !known(dtype) || width == 0) return SDL_ERR_INVALID_ARG;
    if (kv_heads == 0 ? heads != 0 : heads % kv_heads != 0) return SDL_ERR_INVALID_ARG;
    if (heads && !sdl_attention_shape(batch, queries, keys, heads, kv_heads, width, dtype)) return SDL_ERR_UNSUPPORTED;
    if (!aligned_to(q_len, 4) || !aligned_to(k_len, 4)) return SDL_ERR_ALIGNMENT;
    p.q_len = q_len;
    p.k_len = k_len;
    p.group = make_div(heads ? heads / kv_heads : 1);
    p.queries = queries;
    p.keys = keys;
    p.kv_heads = kv_heads;
    p.width = width;
    p.batch = batch;
    p.scale = scale;
    p.scale_log2 = scale * kLog2e;
    p.causal = causal != 0;
    p.spread = 2 * (uint64_t)batch * keys * kv_heads * width * dtype_size(dtype) <= (4u << 20);
    return SDL_OK;
}

}  // namespace sdl_device
