// Attention of new tokens over the paged cache: sequences with many rows
// (prompts and chunks of them).
//
// Rows of a sequence and a KV head are its new tokens times the query heads that
// share the head, token by token; so the heads of a group share every key and value
// that is read, and 128 rows are few tokens wide.
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

constexpr int kTileWaves = 4;
constexpr int kTileThreads = kTileWaves * kWave;
constexpr int kWaveRows = 32;
constexpr int kTileRows = kTileWaves * kWaveRows;       // rows of a workgroup
constexpr int kKeys = 64;                               // cached tokens of a step

// Row tiles are numbered through the batch with gaps: sequence b's begin at
// floor(q_offset[b] x group / kTileRows) + b, which leaves room for all of
// them, and needs no sum over the batch.
__device__ __forceinline__ int64_t first_tile(const AttendParams& P, int64_t b) {
    return clamp_offset(P.c, P.c.q_offset[b]) * P.group / kTileRows + b;
}

// The last sequence whose first tile is at most `tile`: 64 ways at a time.
__device__ __forceinline__ int64_t tile_seq(const AttendParams& P, int64_t tile) {
    int64_t lo = 0, hi = P.c.n_seqs;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane_id() * step;
        const bool below = at < hi && first_tile(P, at) <= tile;
        const int k = max(__popcll(__ballot(below)) - 1, 0);
        lo += k * step;
        hi = min(lo + step, hi);
    }
    return lo;
}

// 128 rows of one sequence and KV head over one part of its tokens, 32 rows a
// wavefront.  The products run as K Q^T and V^T P^T (32 x 32 matrix instructions), so
// that a lane keeps one row (lane % 32) throughout: scores, weights, maximum and
// sums; the first product's result is the second's operand as it lies: in both,
// lane group g = lane / 32 has the tokens 4 g .. 4 g + 3 and 8 + 4 g .. of
// each 16.  Keys are staged in LDS row by row and values turned, in that order of
// tokens; 16-byte pieces are exchanged (xor) so that neither the writes nor the
// reads of a piece by 8 lanes meet in a bank.  While a step is computed the next
// one's keys and values are under way in registers, and the one after that is
// looked up in the page table.
template <bool F16, int DP, bool EXACT>
__global__ __launch_bounds__(kTileThreads, DP > 128 ? 1 : 2) void tile_kernel(AttendLaunch F) {
    constexpr int kSteps = DP / 16;                     // matrix instructions of a score
    constexpr int kBlocks = DP / 32;                    // of 32 elements of the output
    constexpr int kPieces = DP / 8;                     // 16-byte pieces of a row
    constexpr int kKeyLoads = kKeys * kPieces / kTileThreads;       // pieces a thread stages
    constexpr int kQuads = kKeys / 4 * kPieces / kTileThreads;      // 4 tokens x 8 elements it turns
    static_assert(kKeyLoads >= 1);
    constexpr int kQuadThreads = kKeys / 4 * kPieces;   // < kTileThreads for DP = 64
    constexpr int kTurns = kQuads > 0 ? kQuads : 1;
    const AttendParams& P = F.a;
    const CacheView& c = P.c;
    const int D = EXACT ? DP : c.head_dim;
    const int tid = threadIdx.x, wave = tid / kWave, lane = lane_id(), n = lane & 31, g = lane >> 5;

    __shared__ u32x4 key_lds[2][kKeys * kPieces];
    __shared__ u32x4 value_lds[2][DP * (kKeys / 8)];
    __shared__ int64_t where[2][kKeys];
    __shared__ uint64_t present[2];

    // KV head fastest, then the part, then the row tile, the last (longest) first
    int64_t x = blockIdx.x;
    const int32_t kvh = (int32_t)(x % c.n_kv_heads);
    x /= c.n_kv_heads;
    const int32_t part = (int32_t)(x % F.parts.count);
    x /= F.parts.count;
    const int64_t tile = (int64_t)(gridDim.x / ((uint32_t)c.n_kv_heads * (uint32_t)F.parts.count)) - 1 - x;
    const int64_t b = tile_seq(P, tile);
    const SeqRows s = seq_rows(c, b);
    const int64_t rows = (int64_t)s.n * P.group;
    const int64_t row0 = (tile - first_tile(P, b)) * kTileRows;
    if (rows <= kFewRows || row0 < 0 || row0 >= rows) return;

    const int32_t base = s.length - s.n;                // position of the first new token
    const int64_t row = row0 + wave * kWaveRows + n;
    const bool real = row < rows;
    const int32_t token = (int32_t)((real ? row : rows - 1) / P.group);
    const int32_t head = kvh * P.group + (int32_t)((real ? row : rows - 1) - (int64_t)token * P.group);
    const int32_t pos = base + token;
    // positions of the workgroup's rows, and of the wavefront's
    const int32_t first_pos = base + (int32_t)(row0 / P.group);
    const int32_t last_pos = base + (int32_t)((min(row0 + kTileRows, rows) - 1) / P.group);
    const int64_t wave_row = row0 + wave * kWaveRows;
    const bool idle = wave_row >= rows;
    const int32_t wave_first = base + (int32_t)(wave_row / P.group);
    const int32_t wave_last = base + (int32_t)((min(wave_row + kWaveRows, rows) - 1) / P.group);

    const TileList tiles = visible_tiles<kKeys>(c, P.window, P.sinks, first_pos, last_pos);
    const int32_t per = max(F.parts.tokens / kKeys, (tiles.count + F.parts.count - 1) / F.parts.count);
    const int32_t v_first = (int32_t)min((int64_t)tiles.count, (int64_t)part * per);
    const int32_t v_end = (int32_t)min((int64_t)tiles.count, (int64_t)(part + 1) * per);

    f32x16 acc[kBlocks];
#pragma unroll
    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[j][i] = 0.0f;
    float m = kNone, l = 0.0f;
    bool special = false;               // this thread's values need the rows one by one

    if (v_first < v_end) {
        u32x4 q[kSteps];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int d = 16 * k + 8 * g;
            q[k] = u32x4{0, 0, 0, 0};
            if (real && (EXACT || d < D))
                q[k] = *(const u32x4*)(P.query + (s.first + token) * P.query_token_stride +
                                       (int64_t)head * P.query_head_stride + d);
        }
        const int32_t* const table_row = c.table + b * c.table_width;
        const uint16_t* const keys = c.key + (int64_t)kvh * c.head_stride;
        const uint16_t* const values = c.value + (int64_t)kvh * c.head_stride;

        // where token lane of step v lies; -1: it has no page, or no row sees it
        auto lookup = [&](int32_t v) -> int64_t {
            const int64_t t = (int64_t)tiles.tile(v) * kKeys + lane;
            if (t >= tiles.end || !sees(P.window, P.sinks, max(first_pos, (int32_t)t), (int32_t)t)) return -1;
            return token_offset(c, table_row, (int32_t)t);
        };
        auto keep_lookup = [&](int buffer, int64_t at) {
            const uint64_t mask = __ballot(at >= 0);
            where[buffer][lane] = at;
            if (lane == 0) present[buffer] = mask;
        };
        u32x4 key_regs[kKeyLoads];
        u32x4 value_regs[kTurns][4];
        // loads of the step whose tokens are in where[buffer]
        auto load = [&](int buffer) {
#pragma unroll
            for (int i = 0; i < kKeyLoads; ++i) {
                const int e = tid + i * kTileThreads, t = e / kPieces, piece = e % kPieces;
                const int64_t at = where[buffer][t];
                key_regs[i] = u32x4{0, 0, 0, 0};
                if (at >= 0 && (EXACT || piece * 8 < D)) key_regs[i] = *(const u32x4*)(keys + at + piece * 8);
            }
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                const int e = tid + i * kTileThreads, quad = e / kPieces, piece = e % kPieces;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    value_regs[i][u] = u32x4{0, 0, 0, 0};
                    if (kQuadThreads < kTileThreads && e >= kQuadThreads) continue;
                    const int64_t at = where[buffer][4 * quad + u];
                    if (at >= 0 && (EXACT || piece * 8 < D)) value_regs[i][u] = *(const u32x4*)(values + at + piece * 8);
                }
            }
        };
        // values that some rows see and others do not: one that is not finite
        // would reach the others as 0 x value
        auto look_at = [&](int32_t v) {
            const int32_t t0 = tiles.tile(v) * kKeys, t_last = t0 + kKeys - 1;
            if (t_last <= first_pos && (P.window == 0 || t0 > last_pos - P.window || t_last < P.sinks)) return;
#pragma unroll
            for (int i = 0; i < kTurns; ++i)
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int y = 0; y < 4; ++y) special |= not_finite2<F16>(value_regs[i][u][y]);
        };
        auto store = [&](int buffer) {
#pragma unroll
            for (int i = 0; i < kKeyLoads; ++i) {
                const int e = tid + i * kTileThreads, t = e / kPieces, piece = e % kPieces;
                key_lds[buffer][t * kPieces + (piece ^ (t & (kPieces - 1) & 15))] = key_regs[i];
            }
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                const int e = tid + i * kTileThreads, quad = e / kPieces, piece = e % kPieces;
                if (kQuadThreads < kTileThreads && e >= kQuadThreads) continue;
                // tokens 4 quad ..: step 16 (quad / 4), upper half, lane group
                const int to = 2 * (quad / 4) + (quad & 1), half = quad >> 1 & 1;
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    const uint32_t sel = y & 1 ? 0x07060302u : 0x05040100u;
                    const int d = 8 * piece + y;
                    uint2 z;
                    z.x = __builtin_amdgcn_perm(value_regs[i][1][y / 2], value_regs[i][0][y / 2], sel);
                    z.y = __builtin_amdgcn_perm(value_regs[i][3][y / 2], value_regs[i][2][y / 2], sel);
                    ((uint2*)&value_lds[buffer][d * (kKeys / 8) + (to ^ y ^ (piece & 7))])[half] = z;
                }
            }
        };

        if (wave == 0) {
            keep_lookup(0, lookup(v_first));
            if (v_first + 1 < v_end) keep_lookup(1, lookup(v_first + 1));
        }
        __syncthreads();
        load(0);
        look_at(v_first);
        store(0);
        __syncthreads();
        for (int32_t v = v_first; v < v_end; ++v) {
            const int buffer = (v - v_first) & 1;
            const int32_t t0 = tiles.tile(v) * kKeys, t_last = t0 + kKeys - 1;
            const uint64_t there = present[buffer];
            int64_t at = -1;
            if (v + 1 < v_end) load(buffer ^ 1);
            if (wave == 0 && v + 2 < v_end) at = lookup(v + 2);
            if (!idle && t0 <= wave_last) {
                f32x16 sc[2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sc[h][i] = 0.0f;
#pragma unroll
                for (int k = 0; k < kSteps; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int t = 32 * h + n, piece = 2 * k + g;
                        sc[h] = mfma32<F16>(key_lds[buffer][t * kPieces + (piece ^ (t & (kPieces - 1) & 15))], q[k], sc[h]);
                    }
                const bool full = there == ~0ull && t_last <= wave_first &&
                                  (P.window == 0 || t0 > wave_last - P.window || t_last < P.sinks);
                if (!full) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int u = 32 * h + 8 * (i / 4) + 4 * g + i % 4;
                            if (!(there >> u & 1) || !sees(P.window, P.sinks, pos, t0 + u)) sc[h][i] = -INFINITY;
                        }
                }
                float top = sc[0][0];
#pragma unroll
                for (int i = 1; i < 32; ++i) top = fmaxf(top, sc[i / 16][i % 16]);
                top = fmaxf(top, __shfl_xor(top, 32));
                // The sums are only scaled down when the maximum has grown by
                // more than 2^8 for some row: weights up to 2^8 lose nothing.
                const float m2 = fmaxf(m, top * F.score_scale);
                if (__any(m2 > m + 8.0f)) {
                    const float keep = exp2_fast(m - m2);
                    l *= keep;
                    m = m2;
#pragma unroll
                    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[j][i] *= keep;
                }
                float sum[4] = {0, 0, 0, 0};
                u32x4 w[2][2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float a = exp2_fast(fmaf(sc[h][i], F.score_scale, -m));
                        const float z = exp2_fast(fmaf(sc[h][i + 1], F.score_scale, -m));
                        sum[i / 2 % 4] += a + z;
                        w[h][i / 8][i % 8 / 2] = pack2<F16>(a, z);
                    }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int j = 0; j < kBlocks; ++j) {
                        const int d = 32 * j + n, piece = 2 * y + g;
                        acc[j] = mfma32<F16>(value_lds[buffer][d * (kKeys / 8) + (piece ^ (d & 7) ^ (d >> 3 & 7))],
                                             w[y / 2][y % 2], acc[j]);
                    }
            }
            if (v + 1 < v_end) {
                look_at(v + 1);
                store(buffer ^ 1);
            }
            __syncthreads();
            // where[buffer] was read in the step before
            if (wave == 0 && v + 2 < v_end) keep_lookup(buffer, at);
            __syncthreads();
        }
        l += __shfl_xor(l, 32);
    }

    const int64_t to = (s.first + token) * P.n_heads + head;
    const bool split = F.parts.count > 1;
    const int64_t slot0 = (tile * c.n_kv_heads + kvh) * kTileRows;       // of the parts' rows
    if (__syncthreads_or(special)) {
        for (int r = 0; r < kWaveRows; ++r) {
            const int64_t rr = wave_row + r;
            if (rr >= rows) break;
            const int32_t tok = (int32_t)(rr / P.group), hd = kvh * P.group + (int32_t)(rr - (int64_t)tok * P.group);
            const RowSums y = row_alone<F16, kKeys>(P, b, s.first + tok, hd, base + tok, tiles, v_first, v_end, F.score_scale);
            const int64_t out = (s.first + tok) * P.n_heads + hd, part_slot = (slot0 + rr - row0) * F.parts.count + part;
            const int d = (lane & 31) * 8;
            if (lane < 32 && d < D) {
                const float f = y.l == 0.0f ? 0.0f : 1.0f / y.l;
                for (int e = 0; e < 8; ++e) {
                    if (split) F.parts.sums[part_slot * D + d + e] = y.acc[e];
                    else P.out[out * D + d + e] = from_float<F16>(y.l == 0.0f ? 0.0f : y.acc[e] * f);
                }
            }
            if (lane == 0) {
                if (split) *(float2*)(F.parts.stats + part_slot * 2) = make_float2(y.m, y.l);
                else if (P.lse) P.lse[out] = y.l == 0.0f ? -INFINITY : (y.m + log2f(y.l)) * kLn2;
            }
        }
        return;
    }
    if (!real) return;
    const int64_t slot = (slot0 + row - row0) * F.parts.count + part;
    const float f = split ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * j + 2 * i + 4 * g;
            if (!EXACT && d >= D) continue;
            f32x4 o = {acc[j][i], acc[j][i + 1], acc[j][i + 2], acc[j][i + 3]};
            if (split) {
                if (l != 0.0f) *(f32x4*)(F.parts.sums + slot * D + d) = o;
            } else {
                if (l == 0.0f) o = f32x4{0, 0, 0, 0};
                *(uint2*)(P.out + to * D + d) = make_uint2(pack2<F16>(o[0] * f, o[1] * f), pack2<F16>(o[2] * f, o[3] * f));
            }
        }
    if (g == 0) {
        if (split) *(float2*)(F.parts.stats + slot * 2) = make_float2(m, l);
        else if (P.lse) P.lse[to] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
    }
}

template <bool F16>
__global__ __launch_bounds__(kTileThreads) void join_tiles_kernel(AttendLaunch F) {
    const AttendParams& P = F.a;
    const int64_t slot = (int64_t)blockIdx.x * kTileWaves + threadIdx.x / kWave;
    int64_t x = slot / kTileRows;
    const int32_t kvh = (int32_t)(x % P.c.n_kv_heads);
    const int64_t tile = x / P.c.n_kv_heads, b = tile_seq(P, tile);
    const SeqRows s = seq_rows(P.c, b);
    const int64_t rows = (int64_t)s.n * P.group, row = (tile - first_tile(P, b)) * kTileRows + slot % kTileRows;
    if (rows <= kFewRows || row < 0 || row >= rows) return;
    const int64_t token = row / P.group;
    join_row<F16>(F, slot, (s.first + token) * P.n_heads + kvh * P.group + (row - token * P.group));
}

template <bool F16, int DP>
void launch_dim(const AttendLaunch& f, dim3 grid, hipStream_t stream) {
    const dim3 block(kTileThreads);
    if (f.a.c.head_dim == DP) hipLaunchKernelGGL((tile_kernel<F16, DP, true>), grid, block, 0, stream, f);
    else hipLaunchKernelGGL((tile_kernel<F16, DP, false>), grid, block, 0, stream, f);
}

template <bool F16>
void launch_type(const AttendLaunch& f, dim3 grid, hipStream_t stream) {
    if (f.a.c.head_dim <= 64) launch_dim<F16, 64>(f, grid, stream);
    else if (f.a.c.head_dim <= 128) launch_dim<F16, 128>(f, grid, stream);
    else launch_dim<F16, 256>(f, grid, stream);
}

}  // namespace

int64_t tile_blocks(const AttendParams& p) {
    return (p.c.n_tokens * p.group / kTileRows + p.c.n_seqs) * p.c.n_kv_heads;
}

int64_t tile_slots(const AttendParams& p) { return tile_blocks(p) * kTileRows; }

hipError_t launch_tiles(const AttendLaunch& f, hipStream_t stream) {
    const int64_t blocks = tile_blocks(f.a) * f.parts.count;
    if (!grid_fits(blocks, kTileThreads)) return hipErrorInvalidConfiguration;
    if (f.a.f16) launch_type<true>(f, dim3((unsigned)blocks), stream);
    else launch_type<false>(f, dim3((unsigned)blocks), stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || f.parts.count == 1) return e;
    const int64_t joins = tile_slots(f.a) / kTileWaves;
    if (!grid_fits(joins, kTileThreads)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)joins), block(kTileThreads);
    if (f.a.f16) hipLaunchKernelGGL((join_tiles_kernel<true>), grid, block, 0, stream, f);
    else hipLaunchKernelGGL((join_tiles_kernel<false>), grid, block, 0, stream, f);
    return hipGetLastError();
}

}  // namespace tl
