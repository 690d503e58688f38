// Attention of sequences with few rows: the work of one workgroup, which is
// bound by reading the sequence's keys and values once.
#pragma once

#include "attend_common.h"

namespace tl {

constexpr int kFewTile = 32;            // tokens of a wavefront's step

__device__ __forceinline__ int64_t shuffle64(int64_t x, int lane) {
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)x, lane), hi = (uint32_t)__shfl((int)(x >> 32), lane);
    return (int64_t)((uint64_t)hi << 32 | lo);
}

template <bool STREAM>
__device__ __forceinline__ u32x4 load_once(const uint16_t* p) {
    if (STREAM) return __builtin_nontemporal_load((const u32x4*)p);
    return *(const u32x4*)p;
}

// The wavefronts' sums of a workgroup.
template <int WAVES, int DP>
struct FewLds {
    float sums[WAVES][kFewRows][DP + 4];
    float stats[WAVES][kFewRows][2];
};

// One part of one sequence and KV head, up to 16 rows: the matrix products
// run as K Q^T and V^T P^T, so that a lane keeps one row (lane % 16)
// throughout: its scores, weights, running maximum and sums; weights go from
// the first product's result to the second's operand without leaving their
// lane, as both take the tokens 4g .. 4g + 3 and 16 + 4g .. of a step in lane
// group g = lane / 16.  Each lane loads whole pieces of value rows and turns
// them (8 tokens x DP / 16 elements) in registers.  The wavefronts take steps of 32
// tokens in turn, and join their sums in LDS at the end.
//
// DP: head_dim or the next of 64, 128, 256; pieces beyond head_dim are zero.
// EXACT: head_dim is DP, without the tests for that (256 sequences of 16 to 4352
// tokens, 20 heads of 128: 0.90 ms, 0.93 with them; a prompt of 8192 in tile_rows, 8
// heads of 256: 0.36 and 0.39).
// STREAM: keys and values are read once and not kept in the caches (256
// requests 902 us, 968 without; but 780 and 717 us beside tile_rows).
template <bool F16, int DP, bool EXACT, int WAVES, bool STREAM>
__device__ __forceinline__ void few_rows(const AttendLaunch& F, int64_t block, FewLds<WAVES, DP>& lds) {
    constexpr int kThreads = WAVES * kWave;
    constexpr int kSteps = DP / 32;     // matrix instructions of a score
    constexpr int kPer = DP / 16;       // elements of a value row in a lane
    const AttendParams& P = F.a;
    const CacheView& c = P.c;
    const int D = EXACT ? DP : c.head_dim;
    const int wave = threadIdx.x / kWave, lane = lane_id(), n = lane & 15, g = lane >> 4;

    // part fastest, then the head, then the rows' tile, then the sequence
    int64_t x = block;
    const int32_t part = (int32_t)(x % F.few.count);
    x /= F.few.count;
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
    const int32_t per = max(F.few.tokens / kFewTile, (tiles.count + F.few.count - 1) / F.few.count);
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
        for (int32_t v = (int32_t)v_first + wave; v < v_end; v += WAVES) {
            const int32_t t0 = tiles.tile(v) * kFewTile;
            const uint32_t there = (uint32_t)__ballot(at >= 0);     // tokens of the step that have a page
            const int64_t at0 = max(at, (int64_t)0);
            u32x4 k[2][kSteps];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint16_t* const p = keys + shuffle64(at0, 16 * h + n) + 8 * g;
#pragma unroll
                for (int e = 0; e < kSteps; ++e) {
                    if (EXACT || 32 * e + 8 * g < D) k[h][e] = load_once<STREAM>(p + 32 * e);
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
                        if (EXACT || kPer * n + y < D) z = load_once<STREAM>(p + y);
#pragma unroll
                        for (int u = 0; u < 4; ++u) w[e][y / 2 + u] = z[u];
                    }
                }
            }
            if (v + WAVES < v_end) at = lookup(v + WAVES);

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
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int32_t u = 16 * (e / 4) + 4 * g + e % 4;
                    if (!(any >> u & 1))
#pragma unroll
                        for (int y = 0; y < kPer / 2; ++y) w[e][y] = 0;
                }
                if (any & ~all) {
                    // values that some rows see and others do not: one that is
                    // not finite would reach the others as 0 x value
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int y = 0; y < kPer / 2; ++y) special |= not_finite2<F16>(w[e][y]);
                }
            }
            // the softmax's step: lanes n, n + 16, n + 32 and n + 48 hold row n
            float top = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                              fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m2 = fmaxf(m, top);
            const float keep = weight(m, m2, F.score_scale);
            m = m2;
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = weight(sc[e / 4][e % 4], m, F.score_scale, kLiftFew<F16>);
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
        if constexpr (F16) {
            constexpr float kBack = 1.0f / 32768.0f;        // 2^-lift
            l *= kBack;
#pragma unroll
            for (int j = 0; j < kPer; ++j) acc[j] *= kBack;
        }
    }

    // join the wavefronts: acc[j][i] is element kPer * (4 g + i) + j of row n
    auto& sums = lds.sums;
    auto& stats = lds.stats;
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
        for (int r = wave; r < here; r += WAVES) {
            const int32_t rr = row_tile * kFewRows + r, tok = rr / P.group;
            RowSums y = row_alone<F16, kFewTile>(P, b, s.first + tok, kvh * P.group + (rr - tok * P.group), base + tok,
                                                 tiles, (int32_t)v_first, v_end, F.score_scale);
            const int d = (lane & 31) * 8;
            if (lane < 32 && d < D) {
                *(f32x4*)&sums[0][r][d] = f32x4{y.acc[0], y.acc[1], y.acc[2], y.acc[3]};
                *(f32x4*)&sums[0][r][d + 4] = f32x4{y.acc[4], y.acc[5], y.acc[6], y.acc[7]};
            }
            if (lane < WAVES) {
                stats[lane][r][0] = lane == 0 ? y.m : kNone;
                stats[lane][r][1] = lane == 0 ? y.l : 0.0f;
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < (WAVES - 1) * here * DP; e += kThreads)
            sums[1 + e / (here * DP)][e / DP % here][e % DP] = 0.0f;
        __syncthreads();
    }
    for (int e = threadIdx.x; e < here * (DP / 4); e += kThreads) {
        const int r = e / (DP / 4), d = (e - r * (DP / 4)) * 4;
        float top = stats[0][r][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, stats[w][r][0]);
        float all = 0.0f;
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = weight(stats[w][r][0], top, F.score_scale);
            all = fmaf(stats[w][r][1], f, all);
            const f32x4 y = *(const f32x4*)&sums[w][r][d];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(y[i], f, o[i]);
        }
        const int32_t rr = row_tile * kFewRows + r, tok = rr / P.group;
        const int64_t to = (s.first + tok) * P.n_heads + kvh * P.group + (rr - tok * P.group);
        if (F.few.count > 1) {
            const int64_t slot = ((b * c.n_kv_heads + kvh) * F.slot_rows + rr) * F.few.count + part;
            if (d < D && all != 0.0f) *(f32x4*)(F.few.sums + slot * D + d) = o;
            if (d == 0) *(float2*)(F.few.stats + slot * 2) = make_float2(top, all);
        } else {
            const float f = all == 0.0f ? 0.0f : 1.0f / all;
            if (all == 0.0f) o = f32x4{0, 0, 0, 0};
            if (d < D)
                *(uint2*)(P.out + to * D + d) = make_uint2(pack2<F16>(o[0] * f, o[1] * f), pack2<F16>(o[2] * f, o[3] * f));
            if (d == 0 && P.lse) P.lse[to] = log_sum(top, all, F.score_scale);
        }
    }
}

}  // namespace tl
