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

// The softmax's maximum before any score: finite, so that no difference of
// two maxima is NaN; a score below it is -inf, whose weight is 0.
constexpr float kNone = -FLT_MAX;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

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

// Where the parts of a split call go: per row (token x n_heads + head) and
// part, first all sums [rows][parts][D], then (maximum in log2, sum of weights)
// [rows][parts][2].
struct Parts {
    int32_t count;          // 1 = not split
    int32_t tokens;         // of a part, at least
    float* sums;
    float* stats;
};

}  // namespace tl
