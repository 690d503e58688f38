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

constexpr int kFewWaves = 4;
constexpr int kFewThreads = kFewWaves * kWave;
constexpr int kFewTile = 32;            // tokens of a wavefront's step

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
__global__ __launch_bounds__(kFewThreads) void few_rows_kernel(AttendLaunch F) {
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
            const int64_t slot =
                (((b * F.row_tiles + row_tile) * c.n_kv_heads + kvh) * kFewRows + r) * F.parts.count + part;
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

template <bool F16>
__global__ __launch_bounds__(kFewThreads) void join_few_kernel(AttendLaunch F) {
    const AttendParams& P = F.a;
    const int64_t slot = (int64_t)blockIdx.x * kFewWaves + threadIdx.x / kWave;
    int64_t x = slot / kFewRows;
    const int32_t kvh = (int32_t)(x % P.c.n_kv_heads);
    x /= P.c.n_kv_heads;
    const int64_t b = x / F.row_tiles;
    const SeqRows s = seq_rows(P.c, b);
    const int64_t rows = (int64_t)s.n * P.group, row = x % F.row_tiles * kFewRows + slot % kFewRows;
    if ((P.c.q_offset && rows > kFewRows) || row >= rows) return;
    const int64_t token = row / P.group;
    join_row<F16>(F, slot, (s.first + token) * P.n_heads + kvh * P.group + (row - token * P.group));
}

template <bool F16, int DP>
void launch_few_dim(const AttendLaunch& f, dim3 grid, hipStream_t stream) {
    if (f.a.c.head_dim == DP) hipLaunchKernelGGL((few_rows_kernel<F16, DP, true>), grid, dim3(kFewThreads), 0, stream, f);
    else hipLaunchKernelGGL((few_rows_kernel<F16, DP, false>), grid, dim3(kFewThreads), 0, stream, f);
}

template <bool F16>
void launch_few(const AttendLaunch& f, dim3 grid, hipStream_t stream) {
    if (f.a.c.head_dim <= 64) launch_few_dim<F16, 64>(f, grid, stream);
    else if (f.a.c.head_dim <= 128) launch_few_dim<F16, 128>(f, grid, stream);
    else launch_few_dim<F16, 256>(f, grid, stream);
}

// Row tiles of a sequence and head for few_rows_kernel.
int32_t few_row_tiles(const AttendParams& p) { return p.c.q_offset ? 1 : (p.group + kFewRows - 1) / kFewRows; }
int64_t few_blocks(const AttendParams& p) { return p.c.n_seqs * p.c.n_kv_heads * few_row_tiles(p); }

// Which kernels a call needs, from what the host knows.
bool needs_few(const AttendParams& p) { return p.group <= kFewRows || !p.c.q_offset; }
bool needs_tiles(const AttendParams& p) { return p.c.q_offset && p.c.n_tokens * p.group > kFewRows; }

// How far the tokens of a sequence are split: as long as there are fewer
// workgroups than fill the chip, into parts of at least `least` tokens, and
// into parts of at most `most`.
struct SplitRule {
    int64_t fill, least, most;
};
// few_rows_kernel: three workgroups a CU; a step of each wavefront; and a
// long sequence does not end alone.
constexpr SplitRule kSplitFew = {768, kFewWaves * kFewTile, 4096};
// tile_kernel: a workgroup a CU.
constexpr SplitRule kSplitTiles = {256, 512, INT64_MAX};
constexpr int64_t kMostParts = 256;

int64_t wanted_parts(const AttendParams& p, const SplitRule& rule, int64_t blocks) {
    int64_t tokens = (int64_t)p.c.table_width * p.c.page_tokens;
    if (p.max_length > 0) tokens = std::min<int64_t>(tokens, p.max_length);
    if (p.window > 0) tokens = std::min<int64_t>(tokens, (int64_t)p.window + p.sinks);
    const int64_t fill = std::min((rule.fill + blocks - 1) / blocks, (tokens + rule.least - 1) / rule.least);
    const int64_t n = std::max(fill, tokens / rule.most + (tokens % rule.most != 0));
    return std::max<int64_t>(1, std::min(n, kMostParts));
}

constexpr int64_t kAlign = 256;
int64_t aligned(int64_t bytes) { return (bytes + kAlign - 1) / kAlign * kAlign; }
int64_t sums_bytes(const AttendParams& p, int64_t slots, int64_t parts) {
    return aligned(slots * parts * p.c.head_dim * (int64_t)sizeof(float));
}
int64_t parts_bytes(const AttendParams& p, int64_t slots, int64_t parts) {
    return parts > 1 ? sums_bytes(p, slots, parts) + aligned(slots * parts * 2 * (int64_t)sizeof(float)) : 0;
}

// Takes room for up to `want` parts from the workspace's front.
Parts take_parts(AttendParams* p, const SplitRule& rule, int64_t slots, int64_t want) {
    while (want > 1 && (uint64_t)parts_bytes(*p, slots, want) > p->workspace_bytes) --want;
    Parts r = {(int32_t)want, (int32_t)rule.least, nullptr, nullptr};
    if (want > 1) {
        unsigned char* const at = (unsigned char*)p->workspace;
        r.sums = (float*)at;
        r.stats = (float*)(at + sums_bytes(*p, slots, want));
        p->workspace = at + parts_bytes(*p, slots, want);
        p->workspace_bytes -= (uint64_t)parts_bytes(*p, slots, want);
    }
    return r;
}

}  // namespace

uint64_t attend_workspace_bytes(const AttendParams& p) {
    if (p.c.n_tokens == 0 || p.c.n_seqs == 0) return 0;
    uint64_t n = 0;
    if (needs_few(p))
        n += (uint64_t)parts_bytes(p, few_blocks(p) * kFewRows, wanted_parts(p, kSplitFew, few_blocks(p)));
    if (needs_tiles(p)) n += (uint64_t)parts_bytes(p, tile_slots(p), wanted_parts(p, kSplitTiles, tile_blocks(p)));
    return n;
}

hipError_t launch_attend(const AttendParams& p, hipStream_t stream) {
    AttendLaunch f{};
    f.a = p;
    f.row_tiles = few_row_tiles(p);
    f.score_scale = p.scale * kLog2e;
    if (needs_few(p)) {
        const int64_t blocks = few_blocks(p);
        f.parts = take_parts(&f.a, kSplitFew, blocks * kFewRows, wanted_parts(p, kSplitFew, blocks));
        if (!grid_fits(blocks * f.parts.count, kFewThreads)) return hipErrorInvalidConfiguration;
        const dim3 grid((unsigned)(blocks * f.parts.count)), block(kFewThreads);
        if (p.f16) launch_few<true>(f, grid, stream);
        else launch_few<false>(f, grid, stream);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && f.parts.count > 1) {
            const dim3 joins((unsigned)(blocks * (kFewRows / kFewWaves)));
            if (!grid_fits(joins.x, kFewThreads)) return hipErrorInvalidConfiguration;
            if (p.f16) hipLaunchKernelGGL((join_few_kernel<true>), joins, block, 0, stream, f);
            else hipLaunchKernelGGL((join_few_kernel<false>), joins, block, 0, stream, f);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    if (!needs_tiles(p)) return hipSuccess;
    f.parts = take_parts(&f.a, kSplitTiles, tile_slots(p), wanted_parts(p, kSplitTiles, tile_blocks(p)));
    return launch_tiles(f, stream);
}

}  // namespace tl
