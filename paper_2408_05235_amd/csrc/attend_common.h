// What the attention's kernels share: 16-bit types, matrix instructions, the
// visible tokens of a row, and the parts of a split sequence.
#pragma once

#include <float.h>

#include "cache_rows.h"
#include "device_util.h"

namespace tl {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

template <bool F16>
__device__ __forceinline__ float to_float(uint16_t x) {
    if (F16) return (float)__builtin_bit_cast(_Float16, x);
    return __builtin_bit_cast(float, (uint32_t)x << 16);
}

template <bool F16>
__device__ __forceinline__ uint16_t from_float(float x) {
    if (F16) return __builtin_bit_cast(uint16_t, (_Float16)x);
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// Two values rounded to nearest even, the first in the low half.
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if (F16) return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// Whether a half word's two values hold an infinity or a NaN.
template <bool F16>
__device__ __forceinline__ bool not_finite2(uint32_t x) {
    constexpr uint32_t e = F16 ? 0x7c00u : 0x7f80u;
    return (x & e) == e || (x >> 16 & e) == e;
}
template <bool F16>
__device__ __forceinline__ uint32_t finite_or_zero2(uint32_t x) {
    constexpr uint32_t e = F16 ? 0x7c00u : 0x7f80u;
    return ((x & e) == e ? 0 : x & 0xffffu) | ((x >> 16 & e) == e ? 0 : x & 0xffff0000u);
}

// acc + A B for A 16 x 32 and B 32 x 16: lane (i = lane % 16, g = lane / 16)
// holds A[i][8g .. 8g + 7] and B[8g .. 8g + 7][i], and acc[4g .. 4g + 3][i].
template <bool F16>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 acc) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc,
                                                      0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                       acc, 0, 0, 0);
}

// acc + A B for A 32 x 16 and B 16 x 32: lane (i = lane % 32, g = lane / 32)
// holds A[i][8g .. 8g + 7] and B[8g .. 8g + 7][i], and acc element e is row 8
// (e / 4) + 4 g + e % 4 of column i.
template <bool F16>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 acc) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc,
                                                      0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                       acc, 0, 0, 0);
}

// What weights are relative to before any score (then the largest score so
// far, or a little less, before scaling): finite, so that no difference of two is NaN; a
// score below it is -inf, whose weight is 0.
constexpr float kNone = -FLT_MAX;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Weights are rounded to the 16-bit type for the product with the values: the
// matrix units take no more, and the output has no more (each is off by up to
// 2^-9 of itself in bf16 and 2^-12 in f16; their sum is taken in 32 bits, before the
// rounding).  Against 64 bits the output of one token is off by 1.9e-3 of itself so
// and by 1.65e-3 (its own rounding) with weights of 32 bits; a second product, with
// what the rounding leaves, would cost few_rows 0.2 to 0.8% alone and 1.4% beside
// tile_rows, and tile_rows half as many matrix instructions again.  f16 has no normal numbers below 2^-14: with a largest weight of 1
// those of less than 2^-25 would vanish, of which a long sequence can have many.  So
// weights are relative to 2^-LIFT times the largest and at most 2^15 (tile_rows
// lets them grow by 2^kGrowTiles before it scales its sums down): those of 2^-29
// (few_rows) and 2^-21 (tile_rows) of the largest are still normal.  bf16 has the
// exponents of 32 bits, and values up to their end: weights are at most 1, so that
// sums hold as much as sum w |v| does.  (-4 is a constant of the instruction: 32768
// tokens through a window of 4096 take 560 us so, and 564 with 2^8 and -8.)
// tile_rows' sums keep the lift, which cancels in the output (kUnliftTiles for
// what does not).
template <bool F16>
constexpr float kLiftFew = F16 ? 15.0f : 0.0f;
template <bool F16>
constexpr float kGrowTiles = F16 ? 8.0f : 4.0f;
template <bool F16>
constexpr float kLiftTiles = F16 ? 7.0f : -kGrowTiles<F16>;
template <bool F16>
constexpr float kLiftedTiles = F16 ? 128.0f : 1.0f / 16.0f;         // 2^kLiftTiles
template <bool F16>
constexpr float kUnliftTiles = 1.0f / kLiftedTiles<F16>;

// 2^(scaled difference of two scores): the difference first, which is exact for
// near scores however large they are.
__device__ __forceinline__ float weight(float score, float than, float score_scale, float lift = 0.0f) {
    return exp2_fast(fmaf(score - than, score_scale, lift));
}

// The tokens that rows at positions first .. last see, as a list of tiles of TILE
// tokens: `sink` tiles from 0, the others from tile `from`; tokens are below `end`.
struct TileList {
    int32_t sink, from, count;
    int64_t end;
    __device__ __forceinline__ int32_t tile(int32_t v) const { return v < sink ? v : from + (v - sink); }
};

template <int TILE>
__device__ __forceinline__ TileList visible_tiles(const CacheView& c, int32_t window, int32_t sinks, int64_t first,
                                                  int64_t last) {
    TileList r;
    r.end = max(min(last + 1, table_tokens(c)), (int64_t)0);
    const int64_t lo = window > 0 ? max(first - window + 1, (int64_t)0) : 0;
    r.from = (int32_t)min(lo / TILE, r.end / TILE);
    const int64_t s = min((int64_t)sinks, min(lo, r.end));
    r.sink = (int32_t)min((s + TILE - 1) / TILE, (int64_t)r.from);
    r.count = r.sink + max((int32_t)((r.end + TILE - 1) / TILE) - r.from, 0);
    return r;
}

// Whether a row at position p sees token t.
__device__ __forceinline__ bool sees(int32_t window, int32_t sinks, int32_t p, int32_t t) {
    return t <= p && (window == 0 || t > p - window || t < sinks);
}

// Where the parts of a split call go: per slot (a row of a workgroup) and
// part, first all sums [slots][parts][D], then (the score that weights are
// relative to, their sum)
// [slots][parts][2].
struct Parts {
    int32_t count;          // 1 = not split
    int32_t tokens;         // of a part, at least
    float* sums;
    float* stats;
};

// A launch of the attention's kernels.
struct AttendLaunch {
    AttendParams a;
    float score_scale;      // scale x log2 e
    Parts few;              // of sequences with few rows: a slot per row of a
                            // sequence and KV head
    int32_t row_tiles;      // ... row tiles of a sequence and head
    int32_t slot_rows;      // ... slots of a sequence and head
    bool wide;              // ... with eight wavefronts a workgroup
    Parts tiles;            // of the others: a slot per token and head
    int64_t tile_count;     // row tiles, gaps included
    int32_t tile_per;       // ... a number for so many rows
    bool tile_each;         // ... and one for each sequence
};

// Sequences of up to so many rows (new tokens x query heads of a KV head) are
// few_rows', the others tile_rows'.  64 sequences of 16 to 1280 tokens with 16 rows
// take 62 us so and 113 in tile_rows, 128 with 8 rows of 16 to 4352 250 and 339.  A
// wavefront of few_rows holds 16 rows and more would read everything again; in
// tile_rows 17 to 64 rows leave most of a workgroup's 256 empty: those 64 sequences
// with 20, 32 and 64 rows take 94, 83 and 70 us, 256 of 500 tokens 174, 168 and 190
// (112 with 16 rows; reading once takes 74).
constexpr int kFewRows = 16;

// A workgroup's wavefronts, and the rows that they have in tile_rows: two
// wavefronts a SIMD where their registers allow it.
constexpr int kWaveRows = 32;
constexpr int tile_waves(int head_dim) { return head_dim > 128 ? 4 : 8; }
constexpr int tile_rows_of(int head_dim) { return tile_waves(head_dim) * kWaveRows; }

// Both kinds of sequences in one launch, few_blocks workgroups for those with
// few rows.
hipError_t launch_mixed(const AttendLaunch& f, int64_t few_blocks, hipStream_t stream);

template <bool F16>
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
    const uint4 v = *(const uint4*)p;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = to_float<F16>((uint16_t)w[i]);
        x[2 * i + 1] = to_float<F16>((uint16_t)(w[i] >> 16));
    }
}

__device__ __forceinline__ float log_sum(float top, float all, float score_scale) {
    return all == 0.0f ? -INFINITY : fmaf(top, score_scale, log2f(all)) * kLn2;
}

// One row by itself over the tokens of tiles v0 .. v1 - 1, as the definition
// has it: a wavefront's halves take a token each in turn, 8 elements a lane.
// The way of rows whose step holds values that are not finite and that only
// some of its rows see, and where speed does not matter.
struct RowSums {
    float acc[8];           // of elements 8 (lane % 32) ..
    float m, l;             // the largest score, not scaled, and the sum of weights
};

template <bool F16, int TILE>
__device__ RowSums row_alone(const AttendParams& P, int64_t b, int64_t token, int32_t head, int32_t pos,
                             const TileList& tiles, int32_t v0, int32_t v1, float score_scale) {
    const CacheView& c = P.c;
    const int lane = lane_id(), half = lane / 32, d = (lane & 31) * 8;
    const bool in = d < c.head_dim;
    RowSums r = {{}, kNone, 0.0f};
    float q[8] = {};
    if (in) load8<F16>(P.query + token * P.query_token_stride + (int64_t)head * P.query_head_stride + d, q);
    const int32_t* const table_row = c.table + b * c.table_width;
    const int64_t at0 = (int64_t)(head / P.group) * c.head_stride + d;
    for (int32_t v = v0; v < v1; ++v) {
#pragma unroll 1
        for (int k = half; k < TILE; k += 2) {
            const int64_t t = (int64_t)tiles.tile(v) * TILE + k;
            const int64_t at = t < tiles.end && sees(P.window, P.sinks, pos, (int32_t)t)
                                   ? token_offset(c, table_row, (int32_t)t) : -1;
            float x[8] = {};
            if (in && at >= 0) load8<F16>(c.key + at + at0, x);
            float dot = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) dot = fmaf(q[e], x[e], dot);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
            if (at < 0) continue;
            const float m2 = fmaxf(r.m, dot);
            const float keep = weight(r.m, m2, score_scale), w = weight(dot, m2, score_scale);
            r.l = fmaf(r.l, keep, w);
            if (in) load8<F16>(c.value + at + at0, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) r.acc[e] = fmaf(r.acc[e], keep, w * x[e]);
            r.m = m2;
        }
    }
    const float mo = __shfl_xor(r.m, 32), lo = __shfl_xor(r.l, 32);
    const float m2 = fmaxf(r.m, mo), a = weight(r.m, m2, score_scale), z = weight(mo, m2, score_scale);
    r.l = r.l * a + lo * z;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.acc[e] = r.acc[e] * a + __shfl_xor(r.acc[e], 32) * z;
    r.m = m2;
    return r;
}

// WAVES wavefronts join the parts of a slot, in an order that the parts' number
// gives, to output row `to` (token x n_heads + head): each looks at all parts'
// statistics, a part a lane; then LANES lanes with 4 elements each take every
// (WAVES x 64 / LANES)th part.  Nothing waits for the part before: a part without
// weight is read all the same and left out by its factor of 0.  With WAVES > 1 the
// whole workgroup works on one slot.  `unlift`: what brings the parts' sums of
// weights to a largest weight of 1.
template <bool F16, int LANES, int WAVES>
__device__ __forceinline__ void join_row(const AttendLaunch& F, const Parts& parts, int64_t slot, int64_t to,
                                         float unlift) {
    const AttendParams& P = F.a;
    constexpr int kGroups = kWave / LANES;
    __shared__ f32x4 sums_of[WAVES > 1 ? WAVES - 1 : 1][LANES];
    const int wave = WAVES > 1 ? threadIdx.x / kWave : 0;
    const int lane = lane_id(), n = parts.count, D = P.c.head_dim;
    const float2* const st = (const float2*)parts.stats + slot * n;
    const float* const sums = parts.sums + slot * n * D;
    const int group = lane / LANES, d = lane % LANES * 4;
    float top = kNone;
    for (int k = lane; k < n; k += kWave) top = fmaxf(top, st[k].y == 0.0f ? kNone : st[k].x);
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    float all = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (int k0 = 0; k0 < n; k0 += kWave) {
        const float2 y = k0 + lane < n ? st[k0 + lane] : make_float2(kNone, 0.0f);
        const float f = y.y == 0.0f ? 0.0f : weight(y.x, top, F.score_scale);
        all = fmaf(y.y, f, all);
        const int m = min(n - k0, kWave);
#pragma unroll 8
        for (int k = wave * kGroups; k < m; k += WAVES * kGroups) {
            const int part = min(k + group, m - 1);
            const float there = __shfl(f, part), w = k + group < m ? there : 0.0f;
            f32x4 v = {0, 0, 0, 0};
            if (d < D) v = *(const f32x4*)(sums + (int64_t)(k0 + part) * D + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = w == 0.0f ? o[e] : fmaf(v[e], w, o[e]);
        }
    }
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) all += __shfl_xor(all, s);
#pragma unroll
    for (int s = LANES; s < kWave; s <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], s);
    if constexpr (WAVES > 1) {
        if (wave > 0 && group == 0) sums_of[wave - 1][lane] = o;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < WAVES - 1; ++w) {
            const f32x4 y = sums_of[w][lane % LANES];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += y[e];
        }
    }
    const float f = all == 0.0f ? 0.0f : 1.0f / all;
    if (all == 0.0f) o = f32x4{0, 0, 0, 0};
    if (group == 0 && d < D)
        *(uint2*)(P.out + to * D + d) = make_uint2(pack2<F16>(o[0] * f, o[1] * f), pack2<F16>(o[2] * f, o[3] * f));
    if (lane == 0 && P.lse) P.lse[to] = log_sum(top, all * unlift, F.score_scale);
}

}  // namespace tl
