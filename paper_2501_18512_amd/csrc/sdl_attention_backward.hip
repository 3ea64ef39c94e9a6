// Attention, backward (gfx950):  P = exp(S - lse);  D = rowsum(d_out out);  dS = P (d_out v^T - D);
//                                dq = scale dS k;  dk = scale dS^T q;  dv = P^T d_out.
//
// Two kernels, which both form S and d_out v^T again: 7 products of the size of S instead of the 5 that one kernel for all three would
// take.  That one would have to add every key tile's share of dq up in memory, by fp32 atomics in an order of their own or through a buffer
// per key tile: at 256 keys a workgroup and width 128 the two products more cost 131 kFLOP a row and tile, about 0.1 ns at the
// rate of a large product, the sums 1 KB or more of traffic, about 0.2 ns.
//   dq       rows are a wavefront's own, as in the forward pass: S^T = k q^T and dP^T = v d_out^T leave dS^T where dq^T = k^T dS^T wants it
//   dk, dv   keys are a wavefront's own: S = q k^T and dP = d_out v^T leave P and dS where dv^T = d_out^T P and dk^T = q^T dS want them
// D is worked out by the first and read by the second.  Where the workgroups are too few to fill the chip, a chunk of the keys (or of the
// rows) goes to a workgroup each, which leaves its sums in the workspace, and a third kernel adds them up in order.
//
// In bf16 the registers allow two wavefronts on a SIMD, which keep the matrix units busy for half of the cycles in long sequences and for 37 % in 4 causal ones of 2048 tokens.  2 sequences
// of 4096 tokens, 16 heads of 128, no mask: 384 us for dq and 495 for dk and dv, 780 TFLOP/s of the five products that count, 1090 of the seven; 4 causal ones of 2048: 127 and 166 (140 and 187 on
// another card); 8 of 1024, 12 heads of 64: 44 and 50.  In fp32 the matrix instructions bound it: 118 to 125 TFLOP/s of seven products at width 128 and no mask, 109 to 113 in 4 causal
// sequences of 2048 (a library product 155).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "sdl_attention.h"

namespace {

using namespace sdl_device;

constexpr int kWaves = 4, kRows = 32 * kWaves;          // of the kernel of dq

// Query tokens (kernel of dk and dv) and keys (kernel of dq) that go through shared memory at a time, and the wavefronts of the former, 32 keys each.  A tile
// has to last as long as the next one takes to come.  bf16 at widths over 64: eight wavefronts, as two workgroups of four would have room for tiles of 32 tokens
// only (v of their keys lies in shared memory as well).  Up to 64: 128 tokens a tile instead of 64, 96 -> 91 us for the backward pass of 8 sequences of 1024 tokens
// and 12 heads of 64 (three workgroups a compute unit, which tiles of 64 leave room for, are no faster); 128 keys a tile would take the registers of the third wavefront
// on a SIMD, 91 -> 93 us.  At width 96 v would have room in the registers, with four wavefronts a workgroup: 159 -> 170 us for 4 sequences of 1024, 32 heads over 8.
__host__ __device__ constexpr int tile_of(bool bf16, bool wide) { return bf16 ? (wide ? 64 : 128) : 32; }
__host__ __device__ constexpr int key_tile_of(bool bf16) { return bf16 ? 64 : 32; }
__host__ __device__ constexpr int key_waves(bool bf16, bool wide) { return bf16 && wide ? 8 : 4; }

// In bf16 the sums of a tile's products S and dP of the kernel of dk and dv start from -lse / scale and -D, in place of subtractions of them afterwards: the reads go straight
// to the registers of the sums (with the addresses of LaneReads, 4 sequences of 2048 tokens, 16 heads of 128: 200 -> 185 us).  In fp32 a sum of up to 128 products beside a
// larger number would lose digits that are wanted.
__host__ __device__ constexpr bool from_stats(bool bf16) { return bf16; }

struct BackwardArgs {
    Attention p;
    float* part;            // sums of the splits: [split][batch][key head][row][width], or [split][dk, dv][batch][key head][key][width]
    uint32_t blocks;        // of rows or keys, per (batch, key head)
    uint32_t splits, chunk; // chunk: keys of a split, or tiles of query tokens
    uint32_t by_heads;      // dk, dv: query heads of a split, or 0 where chunks are of tiles
    uint32_t pick;          // splits of no use come last
    uint32_t tile, keys;    // tokens of a tile, keys of a block
    uint64_t stats;         // rows of all sequences: the workspace has their -lse (base 2, or over the scale), then their -D
};

// The query tokens that see a key of a block, in tiles, head by head of the group.
struct Seers {
    int32_t begin, end, per_head, tiles;

    __device__ __forceinline__ Seers(const Attention& p, const Sequence& s, int32_t key0, int32_t tile)
    {
        end = key0 < s.nk ? s.nq : 0;
        begin = p.causal ? min(max(0, key0 - s.shift), s.nq) / tile * tile : 0;
        per_head = end > begin ? (end - begin + tile - 1) / tile : 0;
        tiles = per_head * (int32_t)p.group.d;
    }
};

template <typename T, int W, bool ASYNC>
__global__ void __launch_bounds__(kWaves * kWave, sizeof(T) == 2 ? 2 : 1) sdl_attention_dq_kernel(const BackwardArgs a)
{
    constexpr int HD = tile_width(W), kSteps = W / 16, kOut = W / 32, kTile = key_tile_of(sizeof(T) == 2), kParts = kTile / 32;
    typedef Tile<T, HD> Smem;
    __shared__ __attribute__((aligned(16))) char ks[2][Smem::bytes(kTile)];
    __shared__ __attribute__((aligned(16))) char vs[2][Smem::bytes(kTile)];
    const Attention& p = a.p;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c = lane & 31, half = lane >> 5;

    uint32_t unit, nth, split;
    if (a.pick) {
        const auto splits = [&](uint32_t u, uint32_t n) {
            return ((uint32_t)Sequence(p, u / p.kv_heads, 0).most_seen(p, (a.blocks - 1 - n) * kRows, kRows) + a.chunk - 1) / a.chunk;
        };
        if (!pick_item(blockIdx.x, p.batch * p.kv_heads, a.blocks, splits, unit, nth, split)) return;
    } else {
        const uint32_t units = p.batch * p.kv_heads, each = a.blocks * a.splits;
        if (workgroup() >= units * each) return;
        const Place place(workgroup(), units, each, p.spread);
        unit = place.unit;
        nth = place.within / a.splits;
        split = place.within % a.splits;
    }
    const uint32_t block = a.blocks - 1 - nth;           // the longest first
    const Sequence s(p, unit / p.kv_heads, unit % p.kv_heads);

    const uint32_t n_rows = p.queries * p.group.d;
    const uint32_t row = block * kRows + wave * 32 + c;
    const uint32_t row_in = min(row, n_rows - 1);
    const int32_t t = (int32_t)div(row_in, p.group);
    const uint32_t head = s.g * p.group.d + (row_in - (uint32_t)t * p.group.d);
    const bool valid = row < n_rows && t < s.nq;
    const int32_t sees = valid ? s.seen(p, t) : 0;
    const int32_t t_first = (int32_t)div(min(block * kRows, n_rows - 1), p.group);
    const int32_t t_last = min((int32_t)div(min(block * kRows + kRows, n_rows) - 1, p.group), s.nq - 1);
    const int32_t key_begin = (int32_t)(split * a.chunk);
    const int32_t keys = min(t_last < t_first ? 0 : s.seen(p, t_last), key_begin + (int32_t)a.chunk);     // of this split: [key_begin, keys)
    const int32_t every = t_last < t_first ? 0 : s.seen(p, t_first);
    if (a.splits > 1 && key_begin >= keys) return;       // a chunk that no row sees is not looked at when the sums are added

    Frag<T> q[kSteps], g[kSteps];
    float delta = 0.0f;
    {
        const uint32_t n = valid ? p.width : 0;
        const T* src = at_row<T>(p.q, s.b, (uint32_t)t, head);
        const T* src_g = at_row<T>(p.d_out, s.b, (uint32_t)t, head);
        const T* src_o = at_row<T>(p.out, s.b, (uint32_t)t, head);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const Eight<T> x = load_eight<ASYNC>(src_g, k * 16 + half * 8, n), y = load_eight<ASYNC>(src_o, k * 16 + half * 8, n);
            set_frag(q[k], load_eight<ASYNC>(src, k * 16 + half * 8, n));
            set_frag(g[k], x);
#pragma unroll
            for (int j = 0; j < 8; ++j) delta = __builtin_fmaf(x.get(j), y.get(j), delta);
        }
        delta = half_sum(delta);
    }
    const uint64_t stat = ((uint64_t)s.b * p.kv_heads * p.group.d + head) * p.queries + (uint32_t)t;
    const float lse2 = sees > 0 ? p.lse[stat] * kLog2e : 0.0f;
    const TileCopy<T, HD, kTile, kWaves, ASYNC> copy_k(p.k, s.b, s.g, p.width), copy_v(p.v, s.b, s.g, p.width);
#pragma unroll
    for (int i = 0; i < 2; ++i) copy_k.clear(ks[i]), copy_v.clear(vs[i]);

    if (key_begin < keys) {
        copy_k.bring(ks[0], key_begin, s.nk);
        copy_v.bring(vs[0], key_begin, s.nk);
    }
    const int32_t wave_keys = s.most_seen(p, block * kRows + wave * 32, 32);      // from there on the wavefront helps with the copies only
    int32_t now = 0;
    // D from the stored result has that one's rounding in it, which counts where few keys share a row.  Rows of up to two tiles of keys, the first ones of a causal
    // sequence among them, take it from its definition, the sum of P (d_out v^T), in a turn of its own: 8 sequences of 1024 tokens, 12 heads of 64, error of dq and dk
    // against 64 bits 0.0025 without and 0.0024 with it (0.0017 is one rounding to bf16, 0.0024 two: the operand's and the result's).
    if (sizeof(T) == 2 && keys > 0 && keys <= 2 * kTile && split == 0) {
        delta = 0.0f;
        for (int32_t key0 = 0; key0 < keys; key0 += kTile, now ^= 1) {
            loads_done();
            const int32_t next = key0 + kTile < keys ? key0 + kTile : 0;        // and the first one again for what follows
            copy_k.bring(ks[now ^ 1], next, s.nk);
            copy_v.bring(vs[now ^ 1], next, s.nk);
#pragma unroll 1
            for (int n = 0; n < kParts; ++n) {
                f32x16_t sc = {}, dp = {};
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    mma(sc, Smem::along(ks[now], n * 32 + c, 2 * k + half), q[k]);
                    mma(dp, Smem::along(vs[now], n * 32 + c, 2 * k + half), g[k]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + n * 32 + 8 * (i / 4) + 4 * half + i % 4 < sees) delta = __builtin_fmaf(exp2_fast(__builtin_fmaf(sc[i], p.scale_log2, -lse2)), dp[i], delta);
            }
        }
        delta = half_sum(delta);
    }
    if (row < n_rows && half == 0 && split == 0) {
        p.row_stats[stat] = from_stats(sizeof(T) == 2) ? -lse2 / p.scale_log2 : -lse2;
        p.row_stats[a.stats + stat] = -delta;
    }

    f32x16_t acc[kOut] = {};
    for (int32_t key0 = key_begin; key0 < keys; key0 += kTile, now ^= 1) {
        const char *k_now = ks[now], *v_now = vs[now];
        loads_done();               // this tile is there, and all are done with the one before it
        if (key0 + kTile < keys) {
            copy_k.bring(ks[now ^ 1], key0 + kTile, s.nk);
            copy_v.bring(vs[now ^ 1], key0 + kTile, s.nk);
        }
        if (key0 >= wave_keys) continue;
        f32x16_t sc[kParts] = {}, dp[kParts] = {};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            if (sizeof(T) == 4 && W <= 96 && k * 16 >= (int)p.width) break;
#pragma unroll
            for (int n = 0; n < kParts; ++n) {
                mma(sc[n], Smem::along(k_now, n * 32 + c, 2 * k + half), q[k]);
                mma(dp[n], Smem::along(v_now, n * 32 + c, 2 * k + half), g[k]);
            }
        }
#pragma unroll
        for (int n = 0; n < kParts; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[n][i] = exp2_fast(__builtin_fmaf(sc[n][i], p.scale_log2, -lse2)) * (dp[n][i] - delta);
        if (key0 + kTile > every) {
#pragma unroll
            for (int n = 0; n < kParts; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + n * 32 + 8 * (i / 4) + 4 * half + i % 4 >= sees) sc[n][i] = 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kTile / 16; ++u) {
            const Frag<T> ds = frag_of(sc[u / 2], u % 2, T());
#pragma unroll
            for (int n = 0; n < kOut; ++n) mma(acc[n], Smem::across(k_now, u * 16, n * 32, lane), ds);
        }
    }
    if (row >= n_rows) return;
    if (a.splits > 1) {
        float* dst = a.part + ((((uint64_t)split * p.batch + s.b) * p.kv_heads + s.g) * n_rows + row) * p.width;
#pragma unroll
        for (int n = 0; n < kOut; ++n)
#pragma unroll
            for (int i = 0; i < 16; i += 4) store4<ASYNC>(dst, n * 32 + 2 * i + 4 * half, p.width, acc[n][i], acc[n][i + 1], acc[n][i + 2], acc[n][i + 3]);
        return;
    }
    T* dst = at_row<T>(p.dq, s.b, (uint32_t)t, head);
    const float by = p.scale;
#pragma unroll
    for (int n = 0; n < kOut; ++n)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const bool some = sees > 0;
            store4<ASYNC>(dst, n * 32 + 2 * i + 4 * half, p.width, some ? acc[n][i] * by : 0.0f, some ? acc[n][i + 1] * by : 0.0f,
                   some ? acc[n][i + 2] * by : 0.0f, some ? acc[n][i + 3] * by : 0.0f);
        }
}

template <typename T, int W, bool ASYNC>
__global__ void __launch_bounds__(key_waves(sizeof(T) == 2, W > 64) * kWave, sizeof(T) == 2 ? 2 : 1) sdl_attention_dkv_kernel(const BackwardArgs a)
{
    constexpr int HD = tile_width(W), kSteps = W / 16, kOut = W / 32, kTile = tile_of(sizeof(T) == 2, W > 64), kWaves = key_waves(sizeof(T) == 2, HD > 64), kKeys = 32 * kWaves;
    typedef Tile<T, HD> Smem;
    constexpr bool kFromStats = from_stats(sizeof(T) == 2);
    // At width 128 k and v together would not leave the sums their registers (256 a lane, two wavefronts on a SIMD).
    constexpr bool kShareV = HD > 64;
    struct Stage {
        char q[Smem::bytes(kTile)], g[Smem::bytes(kTile)];
        float stats[2][kTile];          // -lse (base 2, or over the scale), -D
    };
    __shared__ __attribute__((aligned(16))) struct {
        Stage stage[2];
        char v[kShareV ? Smem::bytes(kKeys) : 16];
    } mem;
    const Attention& p = a.p;
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), c = lane & 31, half = lane >> 5;

    uint32_t unit, block, split;                         // the longest first
    if (a.pick) {
        const auto splits = [&](uint32_t u, uint32_t n) {
            const Seers of(p, Sequence(p, u / p.kv_heads, 0), (int32_t)(n * kKeys), kTile);
            const int32_t chunk = (int32_t)(a.by_heads ? a.by_heads * of.per_head : a.chunk);
            return of.tiles ? (uint32_t)((of.tiles + chunk - 1) / chunk) : 0u;
        };
        if (!pick_item(blockIdx.x, p.batch * p.kv_heads, a.blocks, splits, unit, block, split)) return;
    } else {
        const uint32_t units = p.batch * p.kv_heads, each = a.blocks * a.splits;
        if (workgroup() >= units * each) return;
        const Place place(workgroup(), units, each, p.spread);
        unit = place.unit;
        block = place.within / a.splits;
        split = place.within % a.splits;
    }
    const Sequence s(p, unit / p.kv_heads, unit % p.kv_heads);

    const int32_t key0 = (int32_t)(block * kKeys), wave_key0 = key0 + wave * 32, key = wave_key0 + c;
    Frag<T> k[kSteps], v[kShareV ? 1 : kSteps];
    {
        const uint32_t n = key < s.nk ? p.width : 0, at = (uint32_t)max(0, min(key, s.nk - 1));
        const T* src_k = at_row<T>(p.k, s.b, at, s.g);
        const T* src_v = at_row<T>(p.v, s.b, at, s.g);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            set_frag(k[i], load_eight<ASYNC>(src_k, i * 16 + half * 8, n));
            if constexpr (!kShareV) set_frag(v[i], load_eight<ASYNC>(src_v, i * 16 + half * 8, n));
        }
    }
    const Seers seers(p, s, key0, kTile);
    const int32_t chunk = (int32_t)(a.by_heads ? a.by_heads * seers.per_head : a.chunk);
    const int32_t t_begin = seers.begin, t_end = seers.end, tile0 = (int32_t)split * chunk, tiles = min(seers.tiles, tile0 + chunk);
    if (a.splits > 1 && tile0 >= tiles) return;      // nothing there for this split, and nothing is looked at when the sums are added

    // from which token on the lane's key is seen, a key of the wavefront, and every one
    const int32_t never = 0x7fffff00;
    const int32_t t_key = key < s.nk ? (p.causal ? key - s.shift : 0) : never;
    const int32_t t_some = wave_key0 < s.nk ? (p.causal ? wave_key0 - s.shift : 0) : never;
    const int32_t t_full = wave_key0 + 32 <= s.nk ? (p.causal ? wave_key0 + 31 - s.shift : 0) : never;

    f32x16_t dk[kOut] = {}, dv[kOut] = {};
    const int32_t skip = seers.per_head > 0 ? tile0 / seers.per_head : 0;
    uint32_t next_head = s.g * p.group.d + skip;          // what is brought next
    int32_t next_t = t_begin + (tile0 - skip * seers.per_head) * kTile;
    auto bring = [&](Stage& to) __attribute__((always_inline)) {
        TileCopy<T, HD, kTile, kWaves, ASYNC>(p.q, s.b, next_head, p.width).bring(to.q, next_t, t_end);
        TileCopy<T, HD, kTile, kWaves, ASYNC>(p.d_out, s.b, next_head, p.width).bring(to.g, next_t, t_end);
        if (wave == 0) {
            const float* from = p.row_stats + ((uint64_t)s.b * p.kv_heads * p.group.d + next_head) * p.queries;
#pragma unroll
            for (int i = 0; i < 2 * kTile; i += kWave)
                copy_word(from + (uint32_t)min(next_t + (i + lane) % kTile, t_end - 1) + (i + lane >= kTile ? a.stats : 0), lds_offset(to.stats[0] + i));
        }
        next_t += kTile;
        if (next_t >= t_end) next_t = t_begin, ++next_head;
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        TileCopy<T, HD, kTile, kWaves, ASYNC>(p.q, s.b, next_head, p.width).clear(mem.stage[i].q);
        TileCopy<T, HD, kTile, kWaves, ASYNC>(p.d_out, s.b, next_head, p.width).clear(mem.stage[i].g);
    }
    int32_t t0 = next_t;
    if (tile0 < tiles) {
        if constexpr (kShareV) {
            const TileCopy<T, HD, kKeys, kWaves, ASYNC> copy_v(p.v, s.b, s.g, p.width);
            copy_v.clear(mem.v);
            copy_v.bring(mem.v, key0, s.nk);
        }
        bring(mem.stage[0]);
    }
    const LaneReads<T, HD> reads(lane);
    for (int32_t tile = tile0, now = 0; tile < tiles; ++tile, now ^= 1) {
        loads_done();               // this tile is there, and all are done with the one before it
        if (tile + 1 < tiles) bring(mem.stage[now ^ 1]);
        const Stage& in = mem.stage[now];
        const uint32_t in_q = lds_offset(in.q), in_g = lds_offset(in.g);
#pragma unroll
        for (int part = 0; part < kTile; part += 32) {
            if (t0 + part + 31 < t_some) continue;
            uint32_t v_at = lds_offset(mem.v) + wave * 32 / Smem::kGroup * Smem::kGroupBytes;
            asm volatile("" : "+s"(v_at));         // the lane's addresses in it would take four registers through the loop
            f32x16_t sc = {}, dp = {};
            if constexpr (kFromStats) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[i] = in.stats[0][part + 8 * (i / 4) + 4 * half + i % 4], dp[i] = in.stats[1][part + 8 * (i / 4) + 4 * half + i % 4];
            }
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (sizeof(T) == 4 && W <= 96 && i * 16 >= (int)p.width) break;
                mma(sc, reads.along(in_q, part, i), k[i]);
                if constexpr (kShareV)
                    mma(dp, reads.along(in_g, part, i), reads.along(v_at, 0, i));
                else
                    mma(dp, reads.along(in_g, part, i), v[i]);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = part + 8 * (i / 4) + 4 * half + i % 4;
                sc[i] = exp2_fast(kFromStats ? sc[i] * p.scale_log2 : __builtin_fmaf(sc[i], p.scale_log2, in.stats[0][r]));
                dp[i] = sc[i] * (kFromStats ? dp[i] : dp[i] + in.stats[1][r]);
            }
            // unless every row of the tile sees every key of the wavefront
            if (t0 < t_full || t0 + kTile > t_end) {
                const int32_t t = t0 + part + 4 * half, first = t_key - t, end = t_end - t;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (8 * (i / 4) + i % 4 < first || 8 * (i / 4) + i % 4 >= end) sc[i] = 0.0f, dp[i] = 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const Frag<T> pr = frag_of(sc, u, T()), ds = frag_of(dp, u, T());
#pragma unroll
                for (int n = 0; n < kOut; ++n) {
                    mma(dv[n], reads.across(in_g, part + u * 16, n), pr);
                    mma(dk[n], reads.across(in_q, part + u * 16, n), ds);
                }
            }
        }
        t0 += kTile;
        if (t0 >= t_end) t0 = t_begin;
    }
    if (key >= (int32_t)p.keys) return;
    if (a.splits > 1) {
        const uint64_t each = (uint64_t)p.batch * p.kv_heads * p.keys;
        float* dst = a.part + (2 * split * each + ((uint64_t)s.b * p.kv_heads + s.g) * p.keys + (uint32_t)key) * p.width;
#pragma unroll
        for (int n = 0; n < kOut; ++n)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const uint32_t at = n * 32 + 2 * i + 4 * half;
                store4<ASYNC>(dst, at, p.width, dk[n][i], dk[n][i + 1], dk[n][i + 2], dk[n][i + 3]);
                store4<ASYNC>(dst + each * p.width, at, p.width, dv[n][i], dv[n][i + 1], dv[n][i + 2], dv[n][i + 3]);
            }
        return;
    }
    T* dst_k = at_row<T>(p.dk, s.b, (uint32_t)key, s.g);
    T* dst_v = at_row<T>(p.dv, s.b, (uint32_t)key, s.g);
    const bool some = key < s.nk;
#pragma unroll
    for (int n = 0; n < kOut; ++n)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const uint32_t at = n * 32 + 2 * i + 4 * half;
            store4<ASYNC>(dst_k, at, p.width, some ? dk[n][i] * p.scale : 0.0f, some ? dk[n][i + 1] * p.scale : 0.0f,
                   some ? dk[n][i + 2] * p.scale : 0.0f, some ? dk[n][i + 3] * p.scale : 0.0f);
            store4<ASYNC>(dst_v, at, p.width, some ? dv[n][i] : 0.0f, some ? dv[n][i + 1] : 0.0f, some ? dv[n][i + 2] : 0.0f, some ? dv[n][i + 3] : 0.0f);
        }
}

// The sums of the splits added up, in order: four elements a thread.  DQ: rows; otherwise keys, of dk and dv.
template <typename T, bool DQ>
__global__ void __launch_bounds__(256) sdl_attention_add_kernel(const BackwardArgs a, const Div quarters, const uint64_t n)
{
    const Attention& p = a.p;
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= n) return;
    const uint32_t line = div((uint32_t)id, quarters), at = ((uint32_t)id - line * quarters.d) * 4;       // line: [dk, dv][batch][key head][row or key]
    const uint32_t per = DQ ? p.queries * p.group.d : p.keys, bg = line / per, i = line - bg * per;
    const uint32_t heads = p.batch * p.kv_heads, which = DQ ? 0 : bg / heads, within = bg - which * heads;
    const Sequence s(p, within / p.kv_heads, within % p.kv_heads);
    uint32_t used, token, head;
    if constexpr (DQ) {
        token = div(i, p.group);
        head = s.g * p.group.d + (i - token * p.group.d);
        const uint32_t sees = (int32_t)token < s.nq ? (uint32_t)s.seen(p, (int32_t)token) : 0;
        used = (sees + a.chunk - 1) / a.chunk;
    } else {
        token = i;
        head = s.g;
        const Seers seers(p, s, (int32_t)(i / a.keys * a.keys), (int32_t)a.tile);
        used = (int32_t)i < s.nk ? (a.by_heads ? (seers.tiles ? a.splits : 0) : ((uint32_t)seers.tiles + a.chunk - 1) / a.chunk) : 0;
    }
    const float* src = a.part + (uint64_t)line * p.width + at;
    const uint64_t step = (DQ ? 1 : 2) * (uint64_t)heads * per * p.width;
    f32x4_t sum = {};
    if (at + 4 <= p.width) {
#pragma unroll 4
        for (uint32_t k = 0; k < used; ++k) sum += *reinterpret_cast<const f32x4_elem*>(src + k * step);
    } else {
        for (uint32_t k = 0; k < used; ++k)
            for (uint32_t j = 0; j < 4; ++j) sum[j] += at + j < p.width ? src[k * step + j] : 0.0f;
    }
    if (DQ || which == 0) sum *= p.scale;
    T* dst = at_row<T>(DQ ? p.dq : which ? p.dv : p.dk, s.b, token, head);
    store4(dst, at, p.width, sum[0], sum[1], sum[2], sum[3]);
}

// How the work is cut.  A problem with fewer workgroups than compute units (256) is cut into chunks of the long axis, into 512 of them, or, as an fp32 tile takes the
// matrix units 16 times as long, 1024, down to those that pay for a workgroup's start and for the sums that it leaves (256 keys or rows, in fp32 64):
// backward pass of four ragged fp32 sequences of up to 517 tokens 77 / 62 us with 512 / 1024, and 77 with 128 rows at least; of 8192 bf16 tokens for 4 heads 432 / 464,
// of 1024 for 8 heads 55 and, with 128 rows at least, 63.
struct Cut {
    uint32_t chunk, splits, by_heads;
};

Cut cut(uint64_t groups, uint64_t tiles, uint64_t tile, sdl_dtype_t dtype)          // in tiles
{
    uint64_t n = tiles;
    if (groups < 256) {
        const uint64_t least = (dtype == SDL_DTYPE_BF16 ? 256 : 64) / tile, fill = dtype == SDL_DTYPE_BF16 ? 512 : 1024;
        n = (tiles * groups + fill - 1) / fill;
        if (n < least) n = least;
    }
    if (n < 1) n = 1;
    return Cut{(uint32_t)n, tiles <= n ? 1u : (uint32_t)((tiles + n - 1) / n), 0};
}

// The rows of a key block, of `group` query heads with `tiles` tiles each.  By heads where they are enough: a causal sequence's first keys are seen by many rows and its
// last by few, and workgroups of all lengths, the longest first, end together sooner than chunks of one length do
// (16 heads over 4, 8192 tokens of width 128: backward pass 1307 us by chunks, 1008 by heads; 4 sequences of 1024, 32 over 8 of width 96: 182 and 166).
Cut cut_rows(uint64_t groups, uint64_t group, uint64_t tiles, uint64_t tile, sdl_dtype_t dtype)
{
    if (group > 1 && groups < 512 && groups * group >= 256) {
        const uint64_t each = (group * groups + 511) / 512;
        return Cut{(uint32_t)(each * tiles), (uint32_t)((group + each - 1) / each), (uint32_t)each};
    }
    return cut(groups, tiles * group, tile, dtype);
}

struct Plan {
    uint64_t row_blocks, key_blocks, heads;
    Cut keys, rows;         // of the kernel of dq, of the one of dk and dv
    size_t stats, part;     // rows of statistics, of two floats each, and the floats of the sums
    size_t floats() const { return (2 * stats + 3) / 4 * 4 + part; }
};

Plan plan_of(uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads, uint32_t width, sdl_dtype_t dtype)
{
    Plan w{};
    const bool bf16 = dtype == SDL_DTYPE_BF16;
    const uint64_t group = heads / kv_heads, rows = queries * group, tile = tile_of(bf16, width > 64), key_tile = key_tile_of(bf16), block = 32 * key_waves(bf16, width > 64);
    w.heads = (uint64_t)batch * kv_heads;
    w.row_blocks = (rows + kRows - 1) / kRows;
    w.key_blocks = (keys + block - 1) / block;
    w.keys = cut(w.row_blocks * w.heads, (keys + key_tile - 1) / key_tile, key_tile, dtype);
    w.rows = cut_rows(w.key_blocks * w.heads, group, (queries + tile - 1) / tile, tile, dtype);
    w.stats = (size_t)batch * heads * queries;
    const size_t of_keys = w.keys.splits > 1 ? (size_t)w.keys.splits * w.heads * rows * width : 0;
    const size_t of_rows = w.rows.splits > 1 ? (size_t)w.rows.splits * 2 * w.heads * keys * width : 0;
    w.part = of_keys > of_rows ? of_keys : of_rows;
    return w;
}

template <typename T, bool DQ>
int add(const BackwardArgs& a, uint64_t lines, hipStream_t st)
{
    const uint32_t quarters = (a.p.width + 3) / 4;
    const uint64_t n = lines * quarters;
    hipLaunchKernelGGL((sdl_attention_add_kernel<T, DQ>), dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, st, a, make_div(quarters), n);
    return launched();
}

template <typename T, int W>
int backward(BackwardArgs& a, const Plan& plan, hipStream_t st)
{
    const Attention& p = a.p;
    constexpr bool bf16 = sizeof(T) == 2;
    constexpr int key_threads = key_waves(bf16, W > 64) * kWave;
    a.tile = tile_of(bf16, W > 64);
    a.keys = 32 * key_waves(bf16, W > 64);
    a.stats = plan.stats;
    if (plan.row_blocks) {
        a.blocks = (uint32_t)plan.row_blocks;
        a.splits = plan.keys.splits;
        a.chunk = plan.keys.chunk * key_tile_of(bf16);
        a.pick = pick_items(p, plan.row_blocks, a.splits);
        const dim3 grid = grid_of(plan.row_blocks * plan.heads * plan.keys.splits);
        if (async_rows(p.k, p.width, sizeof(T)) && async_rows(p.v, p.width, sizeof(T)))
            hipLaunchKernelGGL((sdl_attention_dq_kernel<T, W, true>), grid, dim3(kWaves * kWave), 0, st, a);
        else
            hipLaunchKernelGGL((sdl_attention_dq_kernel<T, W, false>), grid, dim3(kWaves * kWave), 0, st, a);
        int rc = launched();
        if (rc == SDL_OK && a.splits > 1) rc = add<T, true>(a, (uint64_t)p.queries * p.group.d * plan.heads, st);
        if (rc != SDL_OK) return rc;
    }
    if (!plan.key_blocks) return SDL_OK;
    a.blocks = (uint32_t)plan.key_blocks;
    a.splits = plan.rows.splits;
    a.chunk = plan.rows.chunk;
    a.by_heads = plan.rows.by_heads;
    a.pick = pick_items(p, plan.key_blocks, a.splits);
    const dim3 grid = grid_of(plan.key_blocks * plan.heads * plan.rows.splits);
    if (async_rows(p.q, p.width, sizeof(T)) && async_rows(p.d_out, p.width, sizeof(T)) && async_rows(p.v, p.width, sizeof(T)))
        hipLaunchKernelGGL((sdl_attention_dkv_kernel<T, W, true>), grid, dim3(key_threads), 0, st, a);
    else
        hipLaunchKernelGGL((sdl_attention_dkv_kernel<T, W, false>), grid, dim3(key_threads), 0, st, a);
    int rc = launched();
    if (rc == SDL_OK && a.splits > 1) rc = add<T, false>(a, 2 * (uint64_t)p.keys * plan.heads, st);
    return rc;
}

}  // namespace

extern "C" {

size_t sdl_attention_backward_workspace_bytes(uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads, uint32_t width,
                                              sdl_dtype_t dtype)
{
    if (heads == 0 || !sdl_attention_shape(batch, queries, keys, heads, kv_heads, width, dtype)) return 0;
    const Plan w = plan_of(batch, queries, keys, heads, kv_heads, width, dtype);
    return w.floats() * sizeof(float);
}

int sdl_attention_backward(const sdl_view_t* d_out, const sdl_view_t* q, const sdl_view_t* k, const sdl_view_t* v, const sdl_view_t* out,
                           const float* lse, uint32_t batch, uint32_t queries, uint32_t keys, uint32_t heads, uint32_t kv_heads,
                           uint32_t width, sdl_dtype_t dtype, float scale, int causal, const int32_t* q_len, const int32_t* k_len,
                           const sdl_view_t* dq, const sdl_view_t* dk, const sdl_view_t* dv, void* workspace, size_t workspace_bytes,
                           void* stream)
{
    if (heads == 0) heads = kv_heads, queries = 0;          // keys that no head reads: their gradients are written all the same
    BackwardArgs a{};
    int rc = sdl_attention_problem(a.p, batch, queries, keys, heads, kv_heads, width, dtype, scale, causal, q_len, k_len);
    if (rc != SDL_OK) return rc;
    if (batch == 0 || heads == 0 || (queries == 0 && keys == 0)) return SDL_OK;
    const Plan w = plan_of(batch, queries, keys, heads, kv_heads, width, dtype);
    // numbers of workgroups, and of threads that add sums up, that fit 31 bits
    constexpr uint64_t kMost = 0x7fffffffu;
    if (w.row_blocks * w.heads > kMost / w.keys.splits || w.key_blocks * w.heads > kMost / w.rows.splits) return SDL_ERR_UNSUPPORTED;
    if (w.keys.splits > 1 && (uint64_t)batch * queries * heads * ((width + 3) / 4) > kMost) return SDL_ERR_UNSUPPORTED;
    if (w.rows.splits > 1 && 2 * (uint64_t)batch * kv_heads * keys * ((width + 3) / 4) > kMost) return SDL_ERR_UNSUPPORTED;
    if (queries) {
        if ((rc = check_view(d_out, dtype)) != SDL_OK || (rc = check_view(q, dtype)) != SDL_OK || (rc = check_view(out, dtype)) != SDL_OK) return rc;
        if ((rc = check_output(dq, dtype, batch, queries, heads)) != SDL_OK) return rc;
        if (!lse || !workspace) return SDL_ERR_INVALID_ARG;
        if (!aligned_to(lse, 4) || !aligned_to(workspace, 4)) return SDL_ERR_ALIGNMENT;
        if (workspace_bytes < w.floats() * sizeof(float)) return SDL_ERR_INVALID_ARG;
        a.p.d_out = kernel_view(d_out);
        a.p.q = kernel_view(q);
        a.p.out = kernel_view(out);
        a.p.dq = kernel_view(dq);
        a.p.lse = const_cast<float*>(lse);
        a.p.row_stats = static_cast<float*>(workspace);
        a.part = a.p.row_stats + (w.floats() - w.part);
    }
    if (keys) {
        if ((rc = check_view(k, dtype)) != SDL_OK || (rc = check_view(v, dtype)) != SDL_OK) return rc;
        if ((rc = check_output(dk, dtype, batch, keys, kv_heads)) != SDL_OK || (rc = check_output(dv, dtype, batch, keys, kv_heads)) != SDL_OK) return rc;
        a.p.k = kernel_view(k);
        a.p.v = kernel_view(v);
        a.p.dk = kernel_view(dk);
        a.p.dv = kernel_view(dv);
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool bf16 = dtype == SDL_DTYPE_BF16;
    if (width <= 32) return bf16 ? backward<__bf16, 32>(a, w, st) : backward<float, 32>(a, w, st);
    if (width <= 64) return bf16 ? backward<__bf16, 64>(a, w, st) : backward<float, 64>(a, w, st);
    if (width <= 96) return bf16 ? backward<__bf16, 96>(a, w, st) : backward<float, 96>(a, w, st);
    return bf16 ? backward<__bf16, 128>(a, w, st) : backward<float, 128>(a, w, st);
}

}  // extern "C"
