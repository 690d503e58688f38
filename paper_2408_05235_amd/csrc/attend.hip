// Attention of new tokens over the paged cache (tl_attend).
//
// A wavefront takes one query row of one head and passes once over the tokens
// that it sees, with the running maximum and sum of the softmax: lanes hold 8
// elements of the head each, so that several cached tokens are taken at a
// time, one per group of lanes, and the groups' softmaxes are joined at the end.
#include <hip/hip_runtime.h>

#include <float.h>

#include "cache.h"
#include "cache_rows.h"
#include "device_util.h"
#include "tl_internal.h"

namespace tl {
namespace {

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

constexpr int kRowWaves = 4;
constexpr float kNone = -FLT_MAX;       // the maximum before any score (scores below it are -inf)

// LPK lanes per cached token.
template <bool F16, int LPK>
__global__ __launch_bounds__(kRowWaves * kWave) void row_kernel(AttendParams P) {
    const CacheView& c = P.c;
    const int64_t item = (int64_t)blockIdx.x * kRowWaves + threadIdx.x / kWave;
    if (item >= c.n_tokens * P.n_heads) return;
    const int64_t i = item / P.n_heads;
    const int32_t h = (int32_t)(item - i * P.n_heads);
    int64_t b;
    if (!find_seq(c, i, &b)) return;
    const SeqRows s = seq_rows(c, b);
    if (i < s.first || i - s.first >= s.n) return;
    const int64_t pos = (int64_t)s.length - s.n + (i - s.first);
    const int lane = lane_id(), group = lane / LPK, d = (lane % LPK) * 8;
    const bool in = d < c.head_dim;
    float q[8] = {}, acc[8] = {};
    if (in) load8<F16>(P.query + i * P.query_token_stride + h * P.query_head_stride + d, q);
    float m = kNone, l = 0.0f;
    const int32_t* const row = c.table + b * c.table_width;
    const int64_t head = (int64_t)(h / P.group) * c.head_stride + d;
    const int64_t end = min(pos + 1, table_tokens(c));
    const int64_t from = P.window > 0 ? max(pos - P.window + 1, (int64_t)0) : 0;
    const int64_t sinks = min((int64_t)P.sinks, from);       // tokens [0, sinks) and [from, end)
    const int64_t n = end < from ? min(sinks, max(end, (int64_t)0)) : sinks + (end - from);
    for (int64_t k = group; k < n; k += kWave / LPK) {
        const int32_t t = (int32_t)(k < sinks ? k : from + (k - sinks));
        const int64_t at = token_offset(c, row, t);
        if (at < 0) continue;
        float x[8] = {};
        if (in) load8<F16>(c.key + at + head, x);
        float dot = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = fmaf(q[e], x[e], dot);
#pragma unroll
        for (int o = LPK / 2; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
        const float sc = dot * P.scale;
        const float m2 = fmaxf(m, sc);
        const float keep = __expf(m - m2), w = __expf(sc - m2);
        l = fmaf(l, keep, w);
        if (in) load8<F16>(c.value + at + head, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(acc[e], keep, w * x[e]);
        m = m2;
    }
#pragma unroll
    for (int o = LPK; o < kWave; o <<= 1) {
        const float mo = __shfl_xor(m, o), lo = __shfl_xor(l, o);
        const float m2 = fmaxf(m, mo), a = __expf(m - m2), z = __expf(mo - m2);
        l = l * a + lo * z;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = acc[e] * a + __shfl_xor(acc[e], o) * z;
        m = m2;
    }
    if (group == 0 && in) {
        uint16_t* const out = P.out + item * c.head_dim + d;
        for (int e = 0; e < 8; ++e) out[e] = from_float<F16>(l == 0.0f ? 0.0f : acc[e] / l);
        if (P.lse && d == 0) P.lse[item] = l == 0.0f ? -INFINITY : m + logf(l);
    }
}

template <bool F16>
void launch_rows(const AttendParams& p, dim3 grid, hipStream_t stream) {
    const dim3 block(kRowWaves * kWave);
    if (p.c.head_dim <= 64) hipLaunchKernelGGL((row_kernel<F16, 8>), grid, block, 0, stream, p);
    else if (p.c.head_dim <= 128) hipLaunchKernelGGL((row_kernel<F16, 16>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((row_kernel<F16, 32>), grid, block, 0, stream, p);
}

}  // namespace

hipError_t launch_attend(const AttendParams& p, hipStream_t stream) {
    const int64_t blocks = (p.c.n_tokens * p.n_heads + kRowWaves - 1) / kRowWaves;
    if (!grid_fits(blocks, kRowWaves * kWave)) return hipErrorInvalidConfiguration;
    if (p.f16) launch_rows<true>(p, dim3((unsigned)blocks), stream);
    else launch_rows<false>(p, dim3((unsigned)blocks), stream);
    return hipGetLastError();
}

}  // namespace tl
