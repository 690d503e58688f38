// Attention of new tokens over the pages that a list names for each of them and
// KV head (tl_attend_pages).
//
// Rows of a workgroup are up to 16, or 32: the query heads that share the KV head,
// of one token or of several neighbouring ones of a sequence, whose lists are mostly
// alike; it reads every page that one of them names once.  The products are
// few_rows': a step is 32 tokens a wavefront, K Q^T and V^T P^T, and a lane keeps one
// row.
//
// Single tokens are bound by reading: 64 of them, 64 pages of 16 tokens for each of 8
// KV heads (268 MB), take 48 us, 5.6 TB/s, past the caches.  Through them it is 45 us call
// after call, but 107 in place of 56 behind other work that left its writes there, as an
// iteration's other layers do.  Chunks are bound by the vector
// instructions around the products (half of the cycles) and the waits between them.
#include <hip/hip_runtime.h>

#include <float.h>

#include <algorithm>

#include "attend_common.h"
#include "attend_few.h"
#include "cache.h"
#include "cache_rows.h"
#include "device_util.h"
#include "tl.h"
#include "tl_internal.h"

namespace tl {
namespace {

constexpr int kPagesWaves = 4, kPagesThreads = kPagesWaves * kWave;
// Page indices that the lists' bits hold at once (a longer table goes window by
// window), for all of a workgroup's tokens.
constexpr int kMostWords = 4096;

struct PagesLaunch {
    AttendLaunch f;         // few: a slot per token and head
    const int32_t* selected;
    int32_t n_select;
    int32_t slots;          // tokens of a workgroup
    int32_t row_tiles;      // ... or workgroups of a token's heads
    int32_t words;          // of 32 pages each, of a token in a window
    int32_t list;           // entries that the list has room for
};

// A page that some row sees: its number, its place in the sequence, and the
// tokens (bits) whose lists name it.
struct Entry {
    int32_t page, index;
    uint32_t who;
};

__host__ __device__ inline size_t list_bytes(const PagesLaunch& L) {
    return (size_t)L.slots * L.words * sizeof(uint32_t) + (size_t)L.list * sizeof(Entry);
}

// The tokens' lists in the window of pages [w0, w0 + 32 words) as `list`, in
// ascending order, without entries that have no page; returns their number.  A list is
// a set: the order of its entries and repetitions do not matter.
__device__ __forceinline__ int32_t build_list(const PagesLaunch& L, int64_t b, int64_t token, int32_t kvh, int32_t many,
                                              int32_t w0, int32_t pages, uint32_t* bits, Entry* list, int32_t* wave_sum) {
    const CacheView& c = L.f.a.c;
    const int wave = wave_number();
    const int32_t words = min(L.words, (pages - w0 + 31) / 32);
    for (int32_t k = threadIdx.x; k < many * words; k += kPagesThreads) bits[k] = 0;
    __syncthreads();
    for (int32_t k = threadIdx.x; k < many * L.n_select; k += kPagesThreads) {
        const int32_t s = k / L.n_select;
        const int32_t j = L.selected[((token + s) * c.n_kv_heads + kvh) * L.n_select + (k - s * L.n_select)];
        if (j >= w0 && j < pages && j - w0 < words * 32) atomicOr(&bits[s * words + (j - w0) / 32], 1u << (j & 31));
    }
    __syncthreads();
    int32_t n = 0;
    for (int32_t k0 = 0; k0 < words; k0 += kPagesThreads) {
        const int32_t k = k0 + threadIdx.x;
        uint32_t any = 0;
        if (k < words)
            for (int32_t s = 0; s < many; ++s) any |= bits[s * words + k];
        const int32_t own = __popc(any), incl = wave_incl_scan(own);
        if (lane_id() == kWave - 1) wave_sum[wave] = incl;
        __syncthreads();
        int32_t at = n + incl - own;
        for (int w = 0; w < kPagesWaves; ++w) {
            if (w < wave) at += wave_sum[w];
            n += wave_sum[w];
        }
        for (uint32_t left = any; left; left &= left - 1, ++at) {
            const int bit = __builtin_ctz(left);
            uint32_t who = 0;
            for (int32_t s = 0; s < many; ++s) who |= (bits[s * words + k] >> bit & 1) << s;
            if (at < L.list) list[at] = Entry{-1, w0 + k * 32 + bit, who};
        }
        __syncthreads();
    }
    n = min(n, L.list);
    // (the table by all lanes: not one behind the other)
    for (int32_t k = threadIdx.x; k < n; k += kPagesThreads) {
        const int32_t page = c.table[b * c.table_width + list[k].index];
        list[k].page = page >= 0 && page < c.n_pages ? page : -1;
    }
    __syncthreads();
    return n;
}

// Token u of the list: where it lies (-1: nowhere), its position and who names it.
struct Place {
    int64_t at;
    int32_t t;
    uint32_t who;
};
__device__ __forceinline__ Place place_of(const CacheView& c, const Entry* list, int32_t n, int64_t u) {
    Place r = {-1, 0, 0};
    if (u >= (int64_t)n * c.page_tokens) return r;
    const uint32_t e = div_u32((uint32_t)u, c.div_page), row = (uint32_t)u - e * (uint32_t)c.page_tokens;
    const Entry x = list[e];
    r.t = (int32_t)min((int64_t)x.index * c.page_tokens + row, (int64_t)INT32_MAX);      // (no position)
    if (x.page < 0) return r;
    r.who = x.who;
    r.at = (int64_t)x.page * c.page_stride + (int64_t)row * c.token_stride;
    return r;
}

// One row by itself over the list's tokens u0 .. u1 - 1, as the definition has
// it (row_alone's way), added to `r`.
template <bool F16>
__device__ void row_alone_pages(const AttendParams& P, int64_t token, int32_t head, int32_t pos, uint32_t bit,
                                const Entry* list, int32_t n, int64_t u0, int64_t u1, float score_scale, RowSums& r) {
    const CacheView& c = P.c;
    const int lane = lane_id(), half = lane / 32, d = (lane & 31) * 8;
    const bool in = d < c.head_dim;
    float q[8] = {};
    if (in) load8<F16>(P.query + token * P.query_token_stride + (int64_t)head * P.query_head_stride + d, q);
    const int64_t at0 = (int64_t)(head / P.group) * c.head_stride + d;
#pragma unroll 1
    for (int64_t u = u0 + half; u < u1 + half; u += 2) {
        const Place y = place_of(c, list, n, u < u1 ? u : INT64_MAX);
        const int64_t at = (y.who & bit) && y.t <= pos ? y.at : -1;
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

// The wavefronts' sums of a workgroup.
template <int DP, int TILES>
struct PagesLds {
    float sums[kPagesWaves][TILES * kFewRows][DP + 4];
    float stats[kPagesWaves][TILES * kFewRows][2];
};

// TILES: of 16 rows, which share what is read and turned.  Two tiles where sequences
// have many new tokens: 512 of two sequences, each with 48 of up to 683 pages of 24
// tokens, 32 heads on 8, 88 us, and 117 with one.
// Workgroups: part fastest, then the heads' tile, then the KV head, then the
// tokens' tile (numbered through the batch with gaps: those of sequence b begin at
// floor(q_offset[b] / slots) + b).
template <bool F16, int DP, bool EXACT, int TILES, bool STREAM>
__global__ __launch_bounds__(kPagesThreads, DP > 128 ? 1 : TILES > 1 ? 2 : 3) void attend_pages_kernel(PagesLaunch L, int64_t first) {
    extern __shared__ __attribute__((aligned(16))) unsigned char lds_bytes[];
    __shared__ int32_t wave_sum[kPagesWaves];
    constexpr int WAVES = kPagesWaves;
    constexpr int kSteps = DP / 32, kPer = DP / 16, kRows = TILES * kFewRows;
    const AttendLaunch& F = L.f;
    const AttendParams& P = F.a;
    const CacheView& c = P.c;
    const int D = EXACT ? DP : c.head_dim;
    const int wave = wave_number(), lane = lane_id(), n = lane & 15, g = lane >> 4;

    int64_t x = blockIdx.x + first;
    const int32_t part = (int32_t)(x % F.few.count);
    x /= F.few.count;
    const int32_t row_tile = (int32_t)(x % L.row_tiles);
    x /= L.row_tiles;
    const int32_t kvh = (int32_t)(x % c.n_kv_heads);
    x /= c.n_kv_heads;
    int64_t b = x, tile0 = x;
    if (c.q_offset) {
        auto first_tile = [&](int64_t at) { return clamp_offset(c, c.q_offset[at]) / L.slots + at; };
        int64_t lo = 0, hi = c.n_seqs;
        while (hi - lo > 1) {
            const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
            const bool below = at < hi && first_tile(at) <= x;
            const int k = max((int)__popcll(__ballot(below)) - 1, 0);
            lo += k * step;
            hi = min(lo + step, hi);
        }
        b = lo;
        tile0 = first_tile(b);
    }
    const SeqRows s = seq_rows(c, b);
    const int64_t s0 = (x - tile0) * L.slots;               // the first of its tokens here
    if (x < tile0 || s0 >= s.n) return;
    const int32_t many = (int32_t)min((int64_t)L.slots, s.n - s0);
    const int64_t token0 = s.first + s0;
    const int32_t pos0 = (int32_t)(s.length - s.n + s0);
    const int32_t here = min(L.slots > 1 ? many * P.group : P.group - row_tile * kRows, kRows);
    bool real[TILES];
    int32_t slot[TILES];
#pragma unroll
    for (int y = 0; y < TILES; ++y) {
        real[y] = y * kFewRows + n < here;
        slot[y] = real[y] && L.slots > 1 ? (y * kFewRows + n) / P.group : 0;
    }
    const int64_t last = min((int64_t)pos0 + many - 1, table_tokens(c) - 1);
    const int32_t pages = last < 0 ? 0 : (int32_t)(div_u32((uint32_t)last, c.div_page) + 1);

    uint32_t* const bits = (uint32_t*)lds_bytes;
    Entry* const list = (Entry*)(lds_bytes + (size_t)L.slots * L.words * sizeof(uint32_t));

    f32x4 acc[TILES][kPer];
    float m[TILES], l[TILES];
    u32x4 q[TILES][kSteps];
#pragma unroll
    for (int y = 0; y < TILES; ++y) {
        m[y] = kNone;
        l[y] = 0.0f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) acc[y][j] = f32x4{0, 0, 0, 0};
        const int32_t head = kvh * P.group + row_tile * kRows + y * kFewRows + n - slot[y] * P.group;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int d = 32 * k + 8 * g;
            q[y][k] = u32x4{0, 0, 0, 0};
            if (real[y] && (EXACT || d < D))
                q[y][k] = *(const u32x4*)(P.query + (token0 + slot[y]) * P.query_token_stride +
                                          (int64_t)head * P.query_head_stride + d);
        }
    }
    const uint16_t* const keys = c.key + (int64_t)kvh * c.head_stride;
    const uint16_t* const values = c.value + (int64_t)kvh * c.head_stride;

    // this part's steps of a window's list
    auto steps_of = [&](int32_t entries, int32_t* from, int32_t* to) {
        const int32_t tiles = (int32_t)(((int64_t)entries * c.page_tokens + kFewTile - 1) / kFewTile);
        const int32_t per = max(F.few.tokens / kFewTile, (tiles + F.few.count - 1) / F.few.count);
        *from = (int32_t)min((int64_t)tiles, (int64_t)part * per);
        *to = (int32_t)min((int64_t)tiles, (int64_t)(part + 1) * per);
    };

    for (int64_t w0 = 0; w0 < pages; w0 += (int64_t)L.words * 32) {
        const int32_t entries = build_list(L, b, token0, kvh, many, (int32_t)w0, pages, bits, list, wave_sum);
        int32_t v_first, v_end;
        steps_of(entries, &v_first, &v_end);
        Place at = place_of(c, list, entries, (int64_t)(v_first + wave) * kFewTile + (lane & 31));
        for (int32_t v = v_first + wave; v < v_end; v += WAVES) {
            const int64_t at0 = max(at.at, (int64_t)0);
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
            // the step's tokens that each row sees, by the row's token
            uint32_t sees[TILES] = {}, any = 0, all = ~0u;
            for (int32_t t = 0; t < many; ++t) {
                const uint32_t y = (uint32_t)__ballot((at.who >> t & 1) && at.t <= pos0 + t);
#pragma unroll
                for (int z = 0; z < TILES; ++z) sees[z] = t == slot[z] ? y : sees[z];
                any |= y;
                all &= y;
            }
            if (v + WAVES < v_end) at = place_of(c, list, entries, (int64_t)(v + WAVES) * kFewTile + (lane & 31));

            u32x4 pw[TILES];
#pragma unroll
            for (int y = 0; y < TILES; ++y) {
                f32x4 sc[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    sc[h] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < kSteps; ++e) sc[h] = mfma16<F16>(k[h][e], q[y][e], sc[h]);
                }
                if (all != ~0u)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!(sees[y] >> (16 * h + 4 * g + i) & 1)) sc[h][i] = -INFINITY;
                // the softmax's step: lanes n, n + 16, n + 32 and n + 48 hold row n
                float top = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                                  fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if (__any(top > m[y])) {
                    const float m2 = fmaxf(m[y], top);
                    const float keep = weight(m[y], m2, F.score_scale);
                    m[y] = m2;
                    l[y] *= keep;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) acc[y][j] *= keep;
                }
                float p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = weight(sc[e / 4][e % 4], m[y], F.score_scale, kLiftFew<F16>);
                l[y] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));     // of this lane's tokens
                pw[y] = u32x4{pack2<F16>(p[0], p[1]), pack2<F16>(p[2], p[3]), pack2<F16>(p[4], p[5]),
                              pack2<F16>(p[6], p[7])};
            }
            // values that no row sees are not used, whatever they are
            if (any != ~0u)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (!(any >> (16 * (e / 4) + 4 * g + e % 4) & 1))
#pragma unroll
                        for (int y = 0; y < kPer / 2; ++y) w[e][y] = 0;
                }
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
                u32x4 a;
#pragma unroll
                for (int y = 0; y < 4; ++y) a[y] = __builtin_amdgcn_perm(w[2 * y + 1][j / 2], w[2 * y][j / 2], sel);
#pragma unroll
                for (int y = 0; y < TILES; ++y) acc[y][j] = mfma16<F16>(a, pw[y], acc[y][j]);
            }
        }
        __syncthreads();                // the list is read
    }
    bool special = false;
#pragma unroll
    for (int y = 0; y < TILES; ++y) {
        l[y] += __shfl_xor(l[y], 16);
        l[y] += __shfl_xor(l[y], 32);
        constexpr float kBack = F16 ? 1.0f / 32768.0f : 1.0f;       // 2^-lift
        l[y] *= kBack;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            acc[y][j] *= kBack;
            // Values that some rows see and others do not reach the others as 0 x value,
            // which is NaN where they are not finite.  Where sums are, the rows are
            // computed one by one instead, a wavefront takes every fourth.
#pragma unroll
            for (int i = 0; i < 4; ++i) special |= L.slots > 1 && !__builtin_isfinite(acc[y][j][i]);
        }
    }
    const bool one_by_one = __syncthreads_or(special);
    PagesLds<DP, TILES>& lds = *(PagesLds<DP, TILES>*)lds_bytes;
    auto& sums = lds.sums;
    auto& stats = lds.stats;
    if (one_by_one) {
        // (the list and the sums share their memory: all rows before any sums)
        RowSums alone[kRows / WAVES];
#pragma unroll
        for (int k = 0; k < kRows / WAVES; ++k) alone[k] = RowSums{{}, kNone, 0.0f};
        for (int64_t w0 = 0; w0 < pages; w0 += (int64_t)L.words * 32) {
            const int32_t entries = build_list(L, b, token0, kvh, many, (int32_t)w0, pages, bits, list, wave_sum);
            int32_t v_first, v_end;
            steps_of(entries, &v_first, &v_end);
#pragma unroll
            for (int k = 0; k < kRows / WAVES; ++k) {
                const int r = k * WAVES + wave, sl = L.slots > 1 ? r / P.group : 0;
                if (r < here)
                    row_alone_pages<F16>(P, token0 + sl, kvh * P.group + row_tile * kRows + r - sl * P.group, pos0 + sl,
                                         1u << sl, list, entries, (int64_t)v_first * kFewTile, (int64_t)v_end * kFewTile,
                                         F.score_scale, alone[k]);
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < kRows / WAVES; ++k) {
            const int r = k * WAVES + wave;
            RowSums y = alone[k];
            // the halves' tokens
            const float mo = __shfl_xor(y.m, 32), lo = __shfl_xor(y.l, 32), top = fmaxf(y.m, mo);
            const float a = weight(y.m, top, F.score_scale), z = weight(mo, top, F.score_scale);
#pragma unroll
            for (int e = 0; e < 8; ++e) y.acc[e] = y.acc[e] * a + __shfl_xor(y.acc[e], 32) * z;
            if (r >= here) continue;
            for (int o = 0; o < WAVES; ++o) {
                const int d = (lane & 31) * 8;
                if (lane < 32 && d < DP) {
                    f32x4 u = {y.acc[0], y.acc[1], y.acc[2], y.acc[3]}, t = {y.acc[4], y.acc[5], y.acc[6], y.acc[7]};
                    if (o > 0) u = t = f32x4{0, 0, 0, 0};
                    *(f32x4*)&sums[o][r][d] = u;
                    *(f32x4*)&sums[o][r][d + 4] = t;
                }
                if (lane == 0) {
                    stats[o][r][0] = o == 0 ? top : kNone;
                    stats[o][r][1] = o == 0 ? y.l * a + lo * z : 0.0f;
                }
            }
        }
    } else {
        // acc[y][j][i] is element kPer * (4 g + i) + j of row 16 y + n
#pragma unroll
        for (int y = 0; y < TILES; ++y) {
            if (!real[y]) continue;
            const int r = y * kFewRows + n;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kPer; j += 4)
                    *(f32x4*)&sums[wave][r][kPer * (4 * g + i) + j] =
                        f32x4{acc[y][j][i], acc[y][j + 1][i], acc[y][j + 2][i], acc[y][j + 3][i]};
            if (g == 0) {
                stats[wave][r][0] = m[y];
                stats[wave][r][1] = l[y];
            }
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < here * (DP / 4); e += kPagesThreads) {
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
        const int32_t sl = L.slots > 1 ? r / P.group : 0;
        const int64_t to = (token0 + sl) * P.n_heads + kvh * P.group + row_tile * kRows + r - sl * P.group;
        if (F.few.count > 1) {
            const int64_t at = to * F.few.count + part;
            if (d < D && all != 0.0f) *(f32x4*)(F.few.sums + at * D + d) = o;
            if (d == 0) *(float2*)(F.few.stats + at * 2) = make_float2(top, all);
        } else {
            const float f = all == 0.0f ? 0.0f : 1.0f / all;
            if (all == 0.0f) o = f32x4{0, 0, 0, 0};
            if (d < D)
                *(uint2*)(P.out + to * D + d) = make_uint2(pack2<F16>(o[0] * f, o[1] * f), pack2<F16>(o[2] * f, o[3] * f));
            if (d == 0 && P.lse) P.lse[to] = log_sum(top, all, F.score_scale);
        }
    }
}

template <bool F16, int LANES>
__global__ __launch_bounds__(kPagesThreads) void join_pages_kernel(AttendLaunch F, int64_t first) {
    const AttendParams& P = F.a;
    const int64_t to = (blockIdx.x + first) * kPagesWaves + wave_number(), i = to / P.n_heads;
    int64_t b;
    if (i >= P.c.n_tokens || !find_seq(P.c, i, &b)) return;
    const SeqRows s = seq_rows(P.c, b);
    if (i < s.first || i - s.first >= s.n) return;
    join_row<F16, LANES, 1>(F, F.few, to, to, 1.0f);
}

// Workgroups of two tiles from which on they are taken: 512 tokens of one sequence with 48
// pages each take 61 us so and 79 with one, 4 times 64 with 128 pages 71 and 106; 32 tokens
// take 22 with one tile and 26 with two.
constexpr int64_t kTwoTiles = 256;

int64_t out_slots(const AttendParams& p) { return p.c.n_tokens * p.n_heads; }

// Rows of a workgroup, and its tokens: several where sequences have several and
// their heads leave room; twice as many where there are workgroups enough.
struct RowTiles {
    int32_t tiles, slots;
};
RowTiles tiles_of(const AttendPagesParams& q) {
    const AttendParams& p = q.a;
    const bool share = p.c.q_offset && p.c.n_tokens > 2 * p.c.n_seqs;
    auto slots = [&](int32_t tiles) {
        return std::max(1, std::min(tiles * kFewRows / p.group, TL_MAX_SELECTED / std::max(q.n_select, 1)));
    };
    if (!share || p.group > kFewRows) return {1, 1};
    if (p.c.head_dim <= 128 && slots(2) > slots(1) && p.c.n_tokens / slots(2) * p.c.n_kv_heads >= kTwoTiles) return {2, slots(2)};
    return {1, slots(1)};
}
int64_t workgroups(const AttendPagesParams& q, const RowTiles& r) {
    const AttendParams& p = q.a;
    const int64_t tiles = p.c.q_offset ? p.c.n_tokens / r.slots + p.c.n_seqs : p.c.n_seqs;
    return tiles * p.c.n_kv_heads * ((p.group + r.tiles * kFewRows - 1) / (r.tiles * kFewRows));
}

constexpr int kLeastTokens = kPagesWaves * kFewTile;
int64_t wanted(const AttendPagesParams& q) {
    const RowTiles r = tiles_of(q);
    const int64_t blocks = workgroups(q, r), tokens = (int64_t)q.n_select * q.a.c.page_tokens;
    // workgroups that the chip holds: three a CU, of two tiles two.  Single tokens take
    // one a CU, as fewer parts are joined (8 sequences of 128 pages 22 us, 26 with three;
    // 32 of them 54 and 60), and tokens that share their lists more, as a workgroup's union is
    // longer than a list (4 times 8 tokens of 128 pages 31 us, 41 with one).
    const int64_t fill = r.tiles > 1 ? 512 : r.slots > 1 ? 768 : 256;
    if (tokens <= 2 * kLeastTokens || (3 * blocks >= 2 * fill && tokens <= 16 * kLeastTokens)) return 1;
    int64_t n = std::min((fill + blocks - 1) / std::max<int64_t>(blocks, 1), (tokens + kLeastTokens - 1) / kLeastTokens);
    while (n > 1 && 5 * n * n > 2 * tokens) --n;
    return n;
}

constexpr int64_t kAlign = 256;
int64_t aligned(int64_t bytes) { return (bytes + kAlign - 1) / kAlign * kAlign; }
int64_t sums_bytes(const AttendParams& p, int64_t parts) {
    return aligned(out_slots(p) * parts * p.c.head_dim * (int64_t)sizeof(float));
}
int64_t parts_bytes(const AttendParams& p, int64_t parts) {
    return parts > 1 ? sums_bytes(p, parts) + aligned(out_slots(p) * parts * 2 * (int64_t)sizeof(float)) : 0;
}

template <bool F16, int DP, int TILES, bool STREAM>
hipError_t launch_tiles(const PagesLaunch& l, int64_t blocks, hipStream_t stream) {
    const size_t lds = std::max(sizeof(PagesLds<DP, TILES>), list_bytes(l));
    return launch_all(blocks * l.f.few.count, kPagesThreads, [&](dim3 grid, int64_t first) {
        const dim3 block(kPagesThreads);
        if (l.f.a.c.head_dim == DP)
            hipLaunchKernelGGL((attend_pages_kernel<F16, DP, true, TILES, STREAM>), grid, block, lds, stream, l, first);
        else hipLaunchKernelGGL((attend_pages_kernel<F16, DP, false, TILES, STREAM>), grid, block, lds, stream, l, first);
    });
}

template <bool F16, int DP>
hipError_t launch_dim(const PagesLaunch& l, int32_t tiles, int64_t blocks, hipStream_t stream) {
    const AttendParams& p = l.f.a;
    hipError_t e = hipSuccess;
    if (l.slots == 1) e = launch_tiles<F16, DP, 1, true>(l, blocks, stream);
    else if (tiles == 1) e = launch_tiles<F16, DP, 1, false>(l, blocks, stream);
    else if constexpr (DP <= 128) e = launch_tiles<F16, DP, 2, false>(l, blocks, stream);
    if (e != hipSuccess || l.f.few.count == 1) return e;
    return launch_all((out_slots(p) + kPagesWaves - 1) / kPagesWaves, kPagesThreads, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((join_pages_kernel<F16, DP / 4>), grid, dim3(kPagesThreads), 0, stream, l.f, first);
    });
}

template <bool F16>
hipError_t launch_type(const PagesLaunch& l, int32_t tiles, int64_t blocks, hipStream_t stream) {
    if (l.f.a.c.head_dim <= 64) return launch_dim<F16, 64>(l, tiles, blocks, stream);
    if (l.f.a.c.head_dim <= 128) return launch_dim<F16, 128>(l, tiles, blocks, stream);
    return launch_dim<F16, 256>(l, tiles, blocks, stream);
}

}  // namespace

uint64_t attend_pages_workspace_bytes(const AttendPagesParams& q) {
    if (q.a.c.n_tokens == 0 || q.a.c.n_seqs == 0) return 0;
    return (uint64_t)parts_bytes(q.a, wanted(q));
}

hipError_t launch_attend_pages(const AttendPagesParams& q, hipStream_t stream) {
    PagesLaunch l{};
    l.f.a = q.a;
    l.f.score_scale = q.a.scale * kLog2e;
    l.selected = q.selected;
    l.n_select = q.n_select;
    const RowTiles r = tiles_of(q);
    l.slots = r.slots;
    l.row_tiles = (q.a.group + r.tiles * kFewRows - 1) / (r.tiles * kFewRows);
    l.words = (int32_t)std::max<int64_t>(1, std::min<int64_t>(((int64_t)q.a.c.table_width + 31) / 32, kMostWords / l.slots));
    l.list = (int32_t)std::max<int64_t>(1, std::min<int64_t>((int64_t)l.slots * q.n_select, (int64_t)l.words * 32));
    int64_t want = wanted(q);
    while (want > 1 && (uint64_t)parts_bytes(q.a, want) > q.a.workspace_bytes) --want;
    l.f.few = Parts{(int32_t)want, kLeastTokens, nullptr, nullptr};
    if (want > 1) {
        l.f.few.sums = (float*)q.a.workspace;
        l.f.few.stats = (float*)((unsigned char*)q.a.workspace + sums_bytes(q.a, want));
    }
    const int64_t blocks = workgroups(q, r);
    // (sequences without rows count here, which no check before has bounded)
    if (q.a.c.n_seqs > INT32_MAX / q.a.c.n_kv_heads || blocks > INT32_MAX) return hipErrorInvalidConfiguration;
    return q.a.f16 ? launch_type<true>(l, r.tiles, blocks, stream) : launch_type<false>(l, r.tiles, blocks, stream);
}

}  // namespace tl
