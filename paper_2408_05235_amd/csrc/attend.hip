// Attention of new tokens over the paged cache (tl_attend): sequences with few
// rows, the join of split sequences, and the dispatch.
//
// Rows of a sequence and a KV head are its new tokens times the query heads
// that share the head.  A sequence of up to 16 rows (one new token, or a few) is
// bound by reading its keys and values once.
#include <hip/hip_runtime.h>

#include <float.h>

#include <algorithm>

#include "attend_common.h"
#include "cache.h"
#include "cache_rows.h"
#include "device_util.h"
#include "tl_internal.h"

namespace tl {
namespace {

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

// One row by itself over the tokens of tiles v0 .. v1 - 1, as the definition
// has it: a wavefront's halves take a token each in turn, 8 elements a lane.
// The way of rows whose step holds values that are not finite and that only
// some of its rows see, and where speed does not matter.
struct RowSums {
    float acc[8];           // of elements 8 (lane % 32) ..
    float m, l;             // the maximum in log2 and the sum of weights
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
            const float sc = dot * score_scale;
            const float m2 = fmaxf(r.m, sc);
            const float keep = exp2_fast(r.m - m2), w = exp2_fast(sc - m2);
            r.l = fmaf(r.l, keep, w);
            if (in) load8<F16>(c.value + at + at0, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) r.acc[e] = fmaf(r.acc[e], keep, w * x[e]);
            r.m = m2;
        }
    }
    const float mo = __shfl_xor(r.m, 32), lo = __shfl_xor(r.l, 32);
    const float m2 = fmaxf(r.m, mo), a = exp2_fast(r.m - m2), z = exp2_fast(mo - m2);
    r.l = r.l * a + lo * z;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.acc[e] = r.acc[e] * a + __shfl_xor(r.acc[e], 32) * z;
    r.m = m2;
    return r;
}

constexpr int kRowWaves = 4;

// Rows of sequences with more than `few` rows, a wavefront each.
template <bool F16>
__global__ __launch_bounds__(kRowWaves * kWave) void row_kernel(AttendParams P, int few, float score_scale) {
    const CacheView& c = P.c;
    const int64_t item = (int64_t)blockIdx.x * kRowWaves + threadIdx.x / kWave;
    if (item >= c.n_tokens * P.n_heads) return;
    const int64_t i = item / P.n_heads;
    const int32_t h = (int32_t)(item - i * P.n_heads);
    int64_t b;
    if (!find_seq(c, i, &b)) return;
    const SeqRows s = seq_rows(c, b);
    if (i < s.first || i - s.first >= s.n) return;
    if ((int64_t)s.n * P.group <= few) return;
    const int32_t pos = s.length - s.n + (int32_t)(i - s.first);
    const TileList tiles = visible_tiles<32>(c, P.window, P.sinks, pos, pos);
    const RowSums y = row_alone<F16, 32>(P, b, i, h, pos, tiles, 0, tiles.count, score_scale);
    const int lane = lane_id(), d = lane * 8;
    if (lane < 32 && d < c.head_dim) {
        uint16_t* const out = P.out + item * c.head_dim + d;
        for (int e = 0; e < 8; ++e) out[e] = from_float<F16>(y.l == 0.0f ? 0.0f : y.acc[e] / y.l);
        if (P.lse && d == 0) P.lse[item] = y.l == 0.0f ? -INFINITY : (y.m + log2f(y.l)) * kLn2;
    }
}

constexpr int kFewRows = 16;
constexpr int kFewWaves = 4;
constexpr int kFewThreads = kFewWaves * kWave;
constexpr int kFewTile = 32;            // tokens of a wavefront's step

struct FewParams {
    AttendParams a;
    Parts parts;
    int32_t row_tiles;                  // of a sequence and head, without q_offset
    float score_scale;                  // scale x log2 e
};

__device__ __forceinline__ int64_t shuffle64(int64_t x, int lane) {
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)x, lane), hi = (uint32_t)__shfl((int)(x >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// One part of one sequence and KV head, up to 16 rows: the matrix products
// run as K Q^T and V^T P^T, so that a lane keeps one row (lane % 16)
// throughout: its scores, weights, running maximum and sums; weights go from
// the first product's result to the second's operand without leaving their
// lane, as both take the tokens 4g .. 4g + 3 and 16 + 4g .. of a step in lane
// group g = lane / 16.  Each lane loads whole pieces of value rows and turns
// them (8 tokens x DP / 16 elements) in registers.  Four wavefronts take steps of 32
// tokens in turn, and join their sums in LDS at the end.
//
// DP: head_dim or the next of 64, 128, 256; pieces beyond head_dim are zero.
template <bool F16, int DP, bool EXACT>
__global__ __launch_bounds__(kFewThreads) void few_rows_kernel(FewParams F) {
    constexpr int kSteps = DP / 32;     // matrix instructions of a score
    constexpr int kPer = DP / 16;       // elements of a value row in a lane
    const AttendParams& P = F.a;
    const CacheView& c = P.c;
    const int D = EXACT ? DP : c.head_dim;
    const int wave = threadIdx.x / kWave, lane = lane_id(), n = lane & 15, g = lane >> 4;

    // part fastest, then the head, then the rows' tile, then the sequence
    int64_t x = blockIdx.x;
    const int32_t part = (int32_t)(x % F.parts.count);
    x /= F.parts.count;
    const int32_t kvh = (int32_t)(x % c.n_kv_heads);
    x /= c.n_kv_heads;
    const int32_t row_tile = (int32_t)(x % F.row_tiles);
    const int64_t b = x / F.row_tiles;
    const SeqRows s = seq_rows(c, b);
    const int64_t rows = (int64_t)s.n * P.group;
    if (rows == 0 || (c.q_offset && rows > kFewRows)) return;
    const int32_t row = row_tile * kFewRows + n;
    const bool real = row < rows;
    const int32_t token = real ? row / P.group : 0;
    const int32_t head = kvh * P.group + (real ? row - token * P.group : 0);
    const int32_t base = s.length - s.n;                     // position of the first new token
    const int32_t pos = base + token;

    const TileList tiles = visible_tiles<kFewTile>(c, P.window, P.sinks, base, (int64_t)base + s.n - 1);
    const int32_t per = max(F.parts.tokens / kFewTile, (tiles.count + F.parts.count - 1) / F.parts.count);
    const int32_t v_end = (int32_t)min((int64_t)tiles.count, (int64_t)(part + 1) * per);
    const int64_t v_first = (int64_t)part * per;

    f32x4 acc[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) acc[j] = f32x4{0, 0, 0, 0};
    float m = kNone, l = 0.0f;
    bool special = false;               // this lane's values need the rows one by one

    if (v_first + wave < v_end) {
        u32x4 q[kSteps];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int d = 32 * k + 8 * g;
            q[k] = u32x4{0, 0, 0, 0};
            if (real && (EXACT || d < D))
                q[k] = *(const u32x4*)(P.query + (s.first + token) * P.query_token_stride +
                                       (int64_t)head * P.query_head_stride + d);
        }
        const int32_t* const table_row = c.table + b * c.table_width;
        const uint16_t* const keys = c.key + (int64_t)kvh * c.head_stride;
        const uint16_t* const values = c.value + (int64_t)kvh * c.head_stride;
        // lane l % 32 looks up token l % 32 of the step
        auto lookup = [&](int32_t v) -> int64_t {
            const int64_t t = (int64_t)tiles.tile(v) * kFewTile + (lane & 31);
            return t < tiles.end ? token_offset(c, table_row, (int32_t)t) : -1;
        };
        int64_t at = lookup((int32_t)v_first + wave);
        for (int32_t v = (int32_t)v_first + wave; v < v_end; v += kFewWaves) {
            const int32_t t0 = tiles.tile(v) * kFewTile;
            const uint32_t there = (uint32_t)__ballot(at >= 0);     // tokens of the step that have a page
            const int64_t at0 = max(at, (int64_t)0);
            u32x4 k[2][kSteps];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint16_t* const p = keys + shuffle64(at0, 16 * h + n) + 8 * g;
#pragma unroll
                for (int e = 0; e < kSteps; ++e) {
                    if (EXACT || 32 * e + 8 * g < D) k[h][e] = *(const u32x4*)(p + 32 * e);
                    else k[h][e] = u32x4{0, 0, 0, 0};
                }
            }
            uint32_t w[8][kPer / 2];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint16_t* const p = values + shuffle64(at0, 16 * (e / 4) + 4 * g + e % 4) + kPer * n;
#pragma unroll
                for (int y = 0; y < kPer; y += 8) {
                    if constexpr (kPer == 4) {
                        uint2 z = make_uint2(0, 0);
                        if (EXACT || kPer * n < D) z = *(const uint2*)p;
                        w[e][0] = z.x;
                        w[e][1] = z.y;
                    } else {
                        u32x4 z = {0, 0, 0, 0};
                        if (EXACT || kPer * n + y < D) z = *(const u32x4*)(p + y);
#pragma unroll
                        for (int u = 0; u < 4; ++u) w[e][y / 2 + u] = z[u];
                    }
                }
            }
            if (v + kFewWaves < v_end) at = lookup(v + kFewWaves);

            f32x4 sc[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                sc[h] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < kSteps; ++e) sc[h] = mfma16<F16>(k[h][e], q[e], sc[h]);
            }
            // every row sees every token of most steps
            const int32_t t_last = t0 + kFewTile - 1;
            const bool full = there == 0xffffffffu && t_last <= base &&
                              (P.window == 0 || t0 > base + s.n - 1 - P.window || t_last < P.sinks);
            if (!full) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int32_t u = 16 * h + 4 * g + i;
                        if (!(there >> u & 1) || !sees(P.window, P.sinks, pos, t0 + u)) sc[h][i] = -INFINITY;
                    }
                // values that no row sees are not used, whatever they are
                // (a token's first row that may see it is the one at its position)
                const int32_t t = t0 + (lane & 31), last = base + s.n - 1, first = max(base, t);
                const uint32_t any =
                    there & (uint32_t)__ballot(first <= last && sees(P.window, P.sinks, first, t));
                const uint32_t all =
                    (uint32_t)__ballot(sees(P.window, P.sinks, base, t) && sees(P.window, P.sinks, last, t));
                if (any & ~all) {
                    // values that some rows see and others do not: one that is
                    // not finite would reach the others as 0 x value
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int y = 0; y < kPer / 2; ++y) special |= not_finite2<F16>(w[e][y]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int32_t u = 16 * (e / 4) + 4 * g + e % 4;
                    if (!(any >> u & 1))
#pragma unroll
                        for (int y = 0; y < kPer / 2; ++y) w[e][y] = 0;
                }
            }
            // the softmax's step: lanes n, n + 16, n + 32 and n + 48 hold row n
            float top = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                              fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m2 = fmaxf(m, top * F.score_scale);
            const float keep = exp2_fast(m - m2);
            m = m2;
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = exp2_fast(fmaf(sc[e / 4][e % 4], F.score_scale, -m));
            float sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
            l = fmaf(l, keep, sum);     // of this lane's tokens
            const u32x4 pw = {pack2<F16>(p[0], p[1]), pack2<F16>(p[2], p[3]), pack2<F16>(p[4], p[5]),
                              pack2<F16>(p[6], p[7])};
#pragma unroll
            for (int j = 0; j < kPer; ++j) acc[j] *= keep;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
                u32x4 a;
#pragma unroll
                for (int y = 0; y < 4; ++y) a[y] = __builtin_amdgcn_perm(w[2 * y + 1][j / 2], w[2 * y][j / 2], sel);
                acc[j] = mfma16<F16>(a, pw, acc[j]);
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
    }

    // join the wavefronts: acc[j][i] is element kPer * (4 g + i) + j of row n
    __shared__ float sums[kFewWaves][kFewRows][DP + 4];
    __shared__ float stats[kFewWaves][kFewRows][2];
    if (real) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kPer; j += 4)
                *(f32x4*)&sums[wave][n][kPer * (4 * g + i) + j] = f32x4{acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]};
        if (g == 0) {
            stats[wave][n][0] = m;
            stats[wave][n][1] = l;
        }
    }
    const int here = (int)min((int64_t)kFewRows, rows - (int64_t)row_tile * kFewRows);
    if (__syncthreads_or(special)) {
        for (int r = wave; r < here; r += kFewWaves) {
            const int32_t rr = row_tile * kFewRows + r, tok = rr / P.group;
            RowSums y = row_alone<F16, kFewTile>(P, b, s.first + tok, kvh * P.group + (rr - tok * P.group), base + tok,
                                                 tiles, (int32_t)v_first, v_end, F.score_scale);
            const int d = (lane & 31) * 8;
            if (lane < 32 && d < D) {
                *(f32x4*)&sums[0][r][d] = f32x4{y.acc[0], y.acc[1], y.acc[2], y.acc[3]};
                *(f32x4*)&sums[0][r][d + 4] = f32x4{y.acc[4], y.acc[5], y.acc[6], y.acc[7]};
            }
            if (lane < kFewWaves) {
                stats[lane][r][0] = lane == 0 ? y.m : kNone;
                stats[lane][r][1] = lane == 0 ? y.l : 0.0f;
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < (kFewWaves - 1) * here * DP; e += kFewThreads)
            sums[1 + e / (here * DP)][e / DP % here][e % DP] = 0.0f;
        __syncthreads();
    }
    for (int e = threadIdx.x; e < here * (DP / 4); e += kFewThreads) {
        const int r = e / (DP / 4), d = (e - r * (DP / 4)) * 4;
        float top = stats[0][r][0];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) top = fmaxf(top, stats[w][r][0]);
        float all = 0.0f;
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            const float f = exp2_fast(stats[w][r][0] - top);
            all = fmaf(stats[w][r][1], f, all);
            const f32x4 y = *(const f32x4*)&sums[w][r][d];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(y[i], f, o[i]);
        }
        const int32_t rr = row_tile * kFewRows + r, tok = rr / P.group;
        const int64_t to = (s.first + tok) * P.n_heads + kvh * P.group + (rr - tok * P.group);
        if (F.parts.count > 1) {
            const int64_t slot = to * F.parts.count + part;
            if (d < D && all != 0.0f) *(f32x4*)(F.parts.sums + slot * D + d) = o;
            if (d == 0) *(float2*)(F.parts.stats + slot * 2) = make_float2(top, all);
        } else {
            const float f = all == 0.0f ? 0.0f : 1.0f / all;
            if (all == 0.0f) o = f32x4{0, 0, 0, 0};
            if (d < D)
                *(uint2*)(P.out + to * D + d) = make_uint2(pack2<F16>(o[0] * f, o[1] * f), pack2<F16>(o[2] * f, o[3] * f));
            if (d == 0 && P.lse) P.lse[to] = all == 0.0f ? -INFINITY : (top + log2f(all)) * kLn2;
        }
    }
}

// A wavefront per row joins its parts in their order.
template <bool F16>
__global__ __launch_bounds__(kFewThreads) void join_kernel(FewParams F) {
    const AttendParams& P = F.a;
    const CacheView& c = P.c;
    const int64_t r = (int64_t)blockIdx.x * kFewWaves + threadIdx.x / kWave;
    if (r >= c.n_tokens * P.n_heads) return;
    const int64_t i = r / P.n_heads;
    int64_t b;
    if (!find_seq(c, i, &b)) return;
    const SeqRows s = seq_rows(c, b);
    if (i < s.first || i - s.first >= s.n) return;
    if (c.q_offset && (int64_t)s.n * P.group > kFewRows) return;
    const int lane = lane_id(), n = F.parts.count, D = c.head_dim;
    const float2* const st = (const float2*)F.parts.stats + r * n;
    float top = kNone;
    for (int k = lane; k < n; k += kWave) top = fmaxf(top, st[k].x);
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float* const sums = F.parts.sums + r * n * D;
    const int d = lane * 4;
    float all = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    for (int k = 0; k < n; ++k) {
        const float2 y = st[k];
        if (y.y == 0.0f) continue;      // an empty part: its sums are not written
        const float f = exp2_fast(y.x - top);
        all = fmaf(y.y, f, all);
        if (d < D) {
            const f32x4 v = *(const f32x4*)(sums + (int64_t)k * D + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(v[e], f, o[e]);
        }
    }
    const float f = all == 0.0f ? 0.0f : 1.0f / all;
    if (all == 0.0f) o = f32x4{0, 0, 0, 0};
    if (d < D) *(uint2*)(P.out + r * D + d) = make_uint2(pack2<F16>(o[0] * f, o[1] * f), pack2<F16>(o[2] * f, o[3] * f));
    if (lane == 0 && P.lse) P.lse[r] = all == 0.0f ? -INFINITY : (top + log2f(all)) * kLn2;
}

template <bool F16, int DP>
void launch_few_dim(const FewParams& f, dim3 grid, hipStream_t stream) {
    if (f.a.c.head_dim == DP) hipLaunchKernelGGL((few_rows_kernel<F16, DP, true>), grid, dim3(kFewThreads), 0, stream, f);
    else hipLaunchKernelGGL((few_rows_kernel<F16, DP, false>), grid, dim3(kFewThreads), 0, stream, f);
}

template <bool F16>
void launch_few(const FewParams& f, dim3 grid, hipStream_t stream) {
    if (f.a.c.head_dim <= 64) launch_few_dim<F16, 64>(f, grid, stream);
    else if (f.a.c.head_dim <= 128) launch_few_dim<F16, 128>(f, grid, stream);
    else launch_few_dim<F16, 256>(f, grid, stream);
}

constexpr int64_t kPartAlign = 256;

int64_t part_bytes(const AttendParams& p) {
    const int64_t rows = p.c.n_tokens * p.n_heads;
    return rows * (p.c.head_dim + 2) * (int64_t)sizeof(float);
}

// Row tiles of a sequence and head for the few-rows kernel.
int32_t few_row_tiles(const AttendParams& p) { return p.c.q_offset ? 1 : (p.group + kFewRows - 1) / kFewRows; }

// How far the tokens of a sequence are split: into parts of at least
// kMinPart tokens (a step of each wavefront) as long as there are fewer than
// kFillBlocks workgroups, and of at most kMaxPart, so that a long sequence does
// not end alone.
constexpr int64_t kMinPart = kFewWaves * kFewTile, kMaxPart = 4096, kFillBlocks = 768, kMostParts = 256;

int64_t wanted_parts(const AttendParams& p) {
    int64_t tokens = (int64_t)p.c.table_width * p.c.page_tokens;
    if (p.max_length > 0) tokens = std::min<int64_t>(tokens, p.max_length);
    if (p.window > 0) tokens = std::min<int64_t>(tokens, (int64_t)p.window + p.sinks + kFewTile);
    const int64_t blocks = p.c.n_seqs * p.c.n_kv_heads * few_row_tiles(p);
    const int64_t fill = std::min((kFillBlocks + blocks - 1) / blocks, (tokens + kMinPart - 1) / kMinPart);
    return std::max<int64_t>(1, std::min(std::max(fill, (tokens + kMaxPart - 1) / kMaxPart), kMostParts));
}

}  // namespace

uint64_t attend_workspace_bytes(const AttendParams& p) {
    if (p.c.n_tokens == 0 || p.c.n_seqs == 0) return 0;
    const int64_t n = wanted_parts(p);
    return n > 1 ? (uint64_t)(n * part_bytes(p) + kPartAlign) : 0;
}

hipError_t launch_attend(const AttendParams& p, hipStream_t stream) {
    FewParams f;
    f.a = p;
    f.row_tiles = few_row_tiles(p);
    f.score_scale = p.scale * kLog2e;
    int64_t n = wanted_parts(p);
    if (p.workspace_bytes < (uint64_t)kPartAlign) n = 1;
    else n = std::max<int64_t>(1, std::min<int64_t>(n, (int64_t)((p.workspace_bytes - kPartAlign) / part_bytes(p))));
    int64_t tokens = (int64_t)p.c.table_width * p.c.page_tokens;
    if (p.max_length > 0) tokens = std::min<int64_t>(tokens, p.max_length);
    f.parts.count = (int32_t)n;
    f.parts.tokens = (int32_t)kMinPart;
    f.parts.sums = (float*)p.workspace;
    f.parts.stats = nullptr;
    if (n > 1) {
        const int64_t sums = p.c.n_tokens * p.n_heads * n * p.c.head_dim * (int64_t)sizeof(float);
        f.parts.stats = (float*)((unsigned char*)p.workspace + (sums + kPartAlign - 1) / kPartAlign * kPartAlign);
    }
    const int64_t few = p.c.n_seqs * p.c.n_kv_heads * f.row_tiles * n;
    if (!grid_fits(few, kFewThreads)) return hipErrorInvalidConfiguration;
    if (p.f16) launch_few<true>(f, dim3((unsigned)few), stream);
    else launch_few<false>(f, dim3((unsigned)few), stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t row_blocks = (p.c.n_tokens * p.n_heads + kRowWaves - 1) / kRowWaves;
    if (!grid_fits(row_blocks, kFewThreads)) return hipErrorInvalidConfiguration;
    if (n > 1) {
        if (p.f16) hipLaunchKernelGGL((join_kernel<true>), dim3((unsigned)row_blocks), dim3(kFewThreads), 0, stream, f);
        else hipLaunchKernelGGL((join_kernel<false>), dim3((unsigned)row_blocks), dim3(kFewThreads), 0, stream, f);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.c.q_offset) {
        const dim3 grid((unsigned)row_blocks), block(kRowWaves * kWave);
        if (p.f16) hipLaunchKernelGGL((row_kernel<true>), grid, block, 0, stream, p, kFewRows, f.score_scale);
        else hipLaunchKernelGGL((row_kernel<false>), grid, block, 0, stream, p, kFewRows, f.score_scale);
    }
    return hipGetLastError();
}

}  // namespace tl
