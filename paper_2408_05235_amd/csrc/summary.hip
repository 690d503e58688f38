// Summaries of the cache's pages (tl_page_bounds) and the pages that score best
// for new tokens (tl_select_pages).
//
// A page's summary of a KV head is, per element, the least and the largest of its
// keys in 127ths of the largest absolute value.  For a query q in 127ths of its own,
// sum_d max(q_d lo_d, q_d hi_d) bounds its product with any key of the page; it is a
// sum of whole numbers below 2^23, so that scores, ties and the pages taken do not
// depend on how the work is cut.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_common.h"
#include "cache.h"
#include "cache_rows.h"
#include "device_util.h"
#include "tl_internal.h"

namespace tl {
namespace {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;

constexpr int kBoundsThreads = 256, kBoundsWaves = kBoundsThreads / kWave;
constexpr float kInv127 = 1.0f / 127.0f;

// Pages that a sequence's new tokens lie in are numbered through the batch with
// gaps, which needs no sum over the batch: n tokens touch at most floor(n / N) + 2
// pages, and those of sequence b begin at floor(q_offset[b] / N) + 2 b.
__device__ __forceinline__ int64_t first_slot(const CacheView& c, int64_t b) {
    return div_u32((uint32_t)clamp_offset(c, c.q_offset[b]), c.div_page) + 2 * b;
}

// The last sequence whose first slot is at most `slot`: 64 ways at a time.
__device__ __forceinline__ int64_t slot_seq(const CacheView& c, int64_t slot) {
    int64_t lo = 0, hi = c.n_seqs;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane_id() * step;
        const bool below = at < hi && first_slot(c, at) <= slot;
        const int k = max((int)__popcll(__ballot(below)) - 1, 0);
        lo += k * step;
        hi = min(lo + step, hi);
    }
    return lo;
}

__device__ __forceinline__ uint32_t pack_bytes(const float (&x)[8], int from) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int32_t)x[from + i] & 0xffu) << (8 * i);
    return w;
}

typedef __attribute__((ext_vector_type(2))) short s16x2;

// The other bits of negative values turned round; its own inverse.
__device__ __forceinline__ s16x2 turned(s16x2 x) { return x ^ ((x >> 15) & s16x2{0x7fff, 0x7fff}); }
__device__ __forceinline__ s16x2 shuffled(s16x2 x, int o) {
    return __builtin_bit_cast(s16x2, __shfl_xor(__builtin_bit_cast(int, x), o));
}

// A wavefront per slot and KV head.  Bound by reading the keys once: those of 32
// prompts, 128 MB, take 23 us, 5.6 TB/s (32 with the floats' own maxima and every lane's
// quotients, when 78% of the cycles went to them).  `lanes` lanes (a power of two of at least
// head_dim / 8) take 8 elements each of a token, the others other tokens.
template <bool F16, int BATCH>
__global__ __launch_bounds__(kBoundsThreads) void bounds_kernel(BoundsParams P, int lanes, int64_t first) {
    const CacheView& c = P.c;
    const int64_t item = (blockIdx.x + first) * kBoundsWaves + wave_number();
    const int64_t slot = item / c.n_kv_heads;
    const int32_t kvh = (int32_t)(item - slot * c.n_kv_heads);
    if (slot >= P.slots) return;
    const int64_t b = c.q_offset ? slot_seq(c, slot) : slot;
    const SeqRows s = seq_rows(c, b);
    const int32_t from = max(s.length - s.n, 0), end = (int32_t)min((int64_t)s.length, table_tokens(c));
    if (s.n == 0 || from >= end) return;
    const int64_t nth = c.q_offset ? slot - first_slot(c, b) : 0;
    const int64_t j = (int64_t)div_u32((uint32_t)from, c.div_page) + nth;
    if (nth < 0 || j * c.page_tokens >= end) return;
    const int32_t page = c.table[b * c.table_width + j];
    if (page < 0 || page >= c.n_pages) return;
    const int count = (int)min((int64_t)c.page_tokens, end - j * c.page_tokens);

    const int piece = lane_id() & (lanes - 1), sub = lane_id() / lanes, per = kWave / lanes;
    const bool in = piece * 8 < c.head_dim;
    const uint16_t* const keys = c.key + (int64_t)page * c.page_stride + (int64_t)kvh * c.head_stride + piece * 8;
    // Two elements a word, as 16-bit whole numbers that order as the floats do (a
    // negative one's other bits turned round), whose packed maxima and minima take half
    // the instructions of the floats'.  Infinities and NaN are beyond all others.
    s16x2 hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) hi[i] = s16x2{-32768, -32768}, lo[i] = s16x2{32767, 32767};
    if (in) {
        // (the last token again in the place of those behind it, which changes nothing)
        for (int r0 = sub; r0 < count; r0 += BATCH * per) {
            u32x4 v[BATCH];
#pragma unroll
            for (int y = 0; y < BATCH; ++y)
                v[y] = __builtin_nontemporal_load((const u32x4*)(keys + (int64_t)min(r0 + y * per, count - 1) * c.token_stride));
#pragma unroll
            for (int y = 0; y < BATCH; ++y)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = v[y][i];
                    const s16x2 x = turned(__builtin_bit_cast(s16x2, w));
                    hi[i] = __builtin_elementwise_max(hi[i], x);
                    lo[i] = __builtin_elementwise_min(lo[i], x);
                }
        }
    }
    for (int o = lanes; o < kWave; o <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            hi[i] = __builtin_elementwise_max(hi[i], shuffled(hi[i], o));
            lo[i] = __builtin_elementwise_min(lo[i], shuffled(lo[i], o));
        }
    // the largest absolute value: of two's complements, -x - 1 orders as a negative's
    // magnitude does
    s16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_elementwise_max(hi[i], ~lo[i]));
    int32_t bits = in ? max((int32_t)top[0], (int32_t)top[1]) : 0;
    for (int o = 1; o < lanes; o <<= 1) bits = max(bits, __shfl_xor(bits, o));
    const bool bad = bits >= (F16 ? 0x7c00 : 0x7f80);
    const float most = to_float<F16>((uint16_t)bits);
    // (a product and not a quotient, as stated in tl.h)
    const float scale = bad ? INFINITY : most * kInv127;
    // (a largest value so small that its 127th is 0 counts as 0)
    const bool none = bad || scale == 0.0f;
    const int64_t at = (int64_t)page * c.n_kv_heads + kvh;
    int8_t* const to = P.bounds + at * 2 * c.head_dim + piece * 8;
    // the quotients by the lanes that have the same elements: a word each, or two
    const int words = per >= 4 ? 1 : 2;
    for (int k = 0; k < words; ++k) {
        const int word = sub * words + k;
        s16x2 h = hi[0], l = lo[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            h = word == i ? hi[i] : h;
            l = word == i ? lo[i] : l;
        }
        h = turned(h);
        l = turned(l);
        uint32_t low = 0, high = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float x = to_float<F16>((uint16_t)h[e]), y = to_float<F16>((uint16_t)l[e]);
            const float a = none ? 0.0f : fminf(fmaxf(ceilf(x / scale), -127.0f), 127.0f);
            const float z = none ? 0.0f : fminf(fmaxf(floorf(y / scale), -127.0f), 127.0f);
            high |= ((uint32_t)(int32_t)a & 0xffu) << (8 * e);
            low |= ((uint32_t)(int32_t)z & 0xffu) << (8 * e);
        }
        if (in && word < 4) {
            *(uint16_t*)(to + 2 * word) = (uint16_t)low;
            *(uint16_t*)(to + c.head_dim + 2 * word) = (uint16_t)high;
        }
    }
    if (lane_id() == 0) P.scale[(int64_t)page * P.scale_stride + kvh] = scale;
}

// ---------------------------------------------------------------- scores

// Orders as the floats do; above all of them a page that is always taken, at the
// bottom a NaN and then a page that is no candidate.
constexpr uint32_t kAlways = 0xffffffffu, kNan = 1u, kNoPage = 0u;
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return kNan;
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);      // one zero
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kScoreWaves = 4, kScoreThreads = kScoreWaves * kWave;

// Bound by how many round trips are under way: a token's length, its table, then the
// pages.  64 single tokens of up to 36864 cached ones (136 MB of summaries) take 35 us,
// 3.9 TB/s, with 4096 workgroups or more (57 with 2048, 37 with 8192, whose rows are
// made more often), two chunks of 512 tokens 32 us with eight tiles a workgroup (36 with
// four, 46 with two).
// A workgroup scores a range of pages for rows of one KV head, 16 rows (query heads)
// a tile: `tiles` tiles of `slots` tokens of `per` rows each (the next power of two of
// the heads that share the KV head), or the more than 16 heads of one token.  Lane (n =
// lane % 16, g = lane / 16) holds the bytes 64 k + 16 g .. of row n and of page n (K =
// 64 bytes a matrix instruction), and of the result the rows 4 g .. 4 g + 3 of page n.
struct ScoreLaunch {
    SelectPagesParams s;
    int32_t per, per_bits, slots, tiles;    // per = 1 << per_bits
    int32_t tokens_of;      // tokens of a workgroup: slots x tiles, or 1
    int32_t span;           // pages of a workgroup
    int32_t spans;          // workgroups of a row tile
    int64_t token0, tokens; // the tokens of this launch
    uint32_t* keys;         // [tokens][n_kv_heads][table_width]
};

// Bytes of a row in LDS: the least elements' share (min(i, 0)), the largest's
// (max(i, 0)), zeros; a piece more, so that rows do not begin in one bank.
template <int STEPS>
constexpr int kRowBytes = STEPS * 64 + 16;

// Pages that a wavefront has on their way at once: 16 KB of them.
template <int STEPS>
constexpr int kPagesOfStep = STEPS > 4 ? 32 : 64;

// V: values that a lane keeps of a tile's column (4 of 1 row each, 2 of 2, else 1).
template <bool F16, int STEPS, int V>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(ScoreLaunch F, int64_t first) {
    constexpr int kSub = kPagesOfStep<STEPS> / 16, kStep = kPagesOfStep<STEPS>;
    extern __shared__ __attribute__((aligned(16))) unsigned char rows_lds[];
    const SelectPagesParams& P = F.s;
    const CacheView& c = P.c;
    const int wave = wave_number(), lane = lane_id(), n = lane & 15, g = lane >> 4;
    const int D = c.head_dim, n_rows = F.tiles * 16;
    float* const unit = (float*)(rows_lds + n_rows * kRowBytes<STEPS>);
    int64_t x = blockIdx.x + first;
    const int32_t span = (int32_t)(x % F.spans);
    x /= F.spans;
    const int32_t kvh = (int32_t)(x % c.n_kv_heads);
    const int64_t t0 = x / c.n_kv_heads * F.tokens_of;      // of this launch
    const bool one = P.group > 16;                          // one token's heads

    // A run of the tokens from s0 on that are one sequence's: up to s_end, the
    // first at position pos0, and the pages of this workgroup that the last one sees
    // (s_end = s0: the token is nobody's).
    struct Run {
        int32_t s_end, p_end;
        int64_t pos0;
        const int32_t* table_row;
    };
    auto run_from = [&](int32_t s0) {
        const int64_t i0 = F.token0 + t0 + s0;
        int64_t b;
        const bool of_one = find_seq(c, i0, &b);
        const SeqRows s = of_one ? seq_rows(c, b) : SeqRows{};
        Run r = {s0, 0, 0, nullptr};
        if (!of_one || i0 < s.first || i0 - s.first >= s.n) return r;
        const int32_t many = (int32_t)min(min((int64_t)(F.tokens_of - s0), s.first + s.n - i0), F.tokens - t0 - s0);
        r.s_end = s0 + many;
        r.pos0 = (int64_t)s.length - s.n + (i0 - s.first);
        const int64_t last = min(r.pos0 + many - 1, table_tokens(c) - 1);
        const int32_t pages = last < 0 ? 0 : (int32_t)(div_u32((uint32_t)last, c.div_page) + 1);
        r.p_end = (int32_t)min((int64_t)pages, (int64_t)(span + 1) * F.span);
        r.table_row = c.table + b * c.table_width;
        return r;
    };
    const int32_t p_span = (int32_t)min((int64_t)span * F.span, (int64_t)INT32_MAX);
    Run run = run_from(0);
    if (F.tokens_of == 1 && run.p_end <= p_span) return;

    // The rows in 127ths of their largest value, kRowsAtOnce a wavefront, 8 elements
    // a lane.  (Rows behind the last head are that head's again, which changes no
    // maximum; what is in no token's row is not used.)
    constexpr int kLanes = STEPS * 4, kRowsAtOnce = kWave / kLanes;
    const int used = one || F.tokens_of > 1 ? n_rows : F.per, d = lane % kLanes * 8;
    for (int r0 = wave * kRowsAtOnce; r0 < used; r0 += kScoreWaves * kRowsAtOnce) {
        const int row = r0 + lane / kLanes;
        const int32_t slot = one ? 0 : row / 16 * F.slots + ((row & 15) >> F.per_bits);
        const int32_t head = min(one ? row : row & (F.per - 1), P.group - 1);
        const bool real = row < used && t0 + slot < F.tokens;
        float q[8] = {}, most = 0.0f;
        if (real && d < D) {
            const u32x4 v = *(const u32x4*)(P.query + (F.token0 + t0 + slot) * P.query_token_stride +
                                            (int64_t)(kvh * P.group + head) * P.query_head_stride + d);
            bool special = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                special |= not_finite2<F16>(v[i]);
                q[2 * i] = to_float<F16>((uint16_t)v[i]);
                q[2 * i + 1] = to_float<F16>((uint16_t)(v[i] >> 16));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(q[i]));
            if (special) most = INFINITY;
        }
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
        const float z = most < INFINITY ? most * kInv127 : 0.0f;
        // rint(q / z): by the reciprocal, whose product is off by less than 2^-14, and
        // divided where that could round the other way
        const float inverse = 1.0f / z;
        float y[8];
        bool near = !(z > 1e-30f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = q[i] * inverse;
            near |= fabsf(fabsf(y[i] - rintf(y[i])) - 0.5f) < 0x1p-13f;
        }
        if (near)
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = z > 0.0f ? q[i] / z : 0.0f;
        float low[8], high[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = rintf(y[i]);
            low[i] = fminf(y[i], 0.0f);
            high[i] = fmaxf(y[i], 0.0f);
        }
        if (row < used) {
            unsigned char* const to = rows_lds + row * kRowBytes<STEPS>;
            if (d < D) {
                *(uint2*)(to + d) = make_uint2(pack_bytes(low, 0), pack_bytes(low, 4));
                *(uint2*)(to + D + d) = make_uint2(pack_bytes(high, 0), pack_bytes(high, 4));
            } else {
                *(uint2*)(to + 2 * d) = make_uint2(0, 0);
                *(uint2*)(to + 2 * d + 8) = make_uint2(0, 0);
            }
            if (d == 0) unit[row] = z;
        }
    }
    __syncthreads();

    // The tokens can be of several sequences, whose pages differ: each sequence
    // in its turn.
    for (int32_t s0 = 0; s0 < F.tokens_of && t0 + s0 < F.tokens;) {
        if (s0 > 0) run = run_from(s0);
        if (run.s_end == s0) {
            ++s0;
            continue;
        }
        const int32_t s_end = run.s_end, p_end = run.p_end;
        const int64_t pos0 = run.pos0;
        const int32_t* const table_row = run.table_row;
        const int32_t tile0 = one ? 0 : s0 / F.slots, tile1 = one ? F.tiles : (s_end - 1) / F.slots + 1;
        const int64_t p_first = (int64_t)p_span + wave * kStep;
        // a step of kStep pages, whose bytes come at once; lane l has page l of it
        int32_t next = p_first + lane < p_end && lane < kStep ? table_row[p_first + lane] : -1;
        for (int64_t p0 = p_first; p0 < p_end; p0 += kScoreWaves * kStep) {
            const bool is_page = next >= 0 && next < c.n_pages;
            const uint32_t is_there = (uint32_t)is_page;
            const int32_t mine = is_page ? next : 0;
            const float scale_of_lane = is_page ? P.scale[(int64_t)mine * P.scale_stride + kvh] : 0.0f;
            i32x4 a[kSub][STEPS];
            float scale[kSub];
            bool there[kSub];
#pragma unroll
            for (int u = 0; u < kSub; ++u) {
                const int32_t page = __shfl(mine, u * 16 + n);
                there[u] = __shfl((int)is_there, u * 16 + n) != 0;
                const int8_t* const at = P.bounds + ((int64_t)page * c.n_kv_heads + kvh) * 2 * D + 16 * g;
#pragma unroll
                for (int k = 0; k < STEPS; ++k) {
                    a[u][k] = i32x4{0, 0, 0, 0};
                    // (Through the caches: past them 64 single tokens' 153 MB take 60 us
                    // where other data in the caches has to be written back first, and 74
                    // so, but 55 and 51 where the last cache has them, and chunks 3% more.)
                    if (there[u] && 64 * k + 16 * g < 2 * D) a[u][k] = *(const i32x4*)(at + 64 * k);
                }
            }
#pragma unroll
            for (int u = 0; u < kSub; ++u) scale[u] = __shfl(scale_of_lane, u * 16 + n);
            const int64_t p_next = p0 + kScoreWaves * kStep + lane;
            next = p_next < p_end && lane < kStep ? table_row[p_next] : -1;

            float top[kSub][V];
            for (int tile = tile0; tile < tile1; ++tile) {
                const unsigned char* const row_at = rows_lds + (tile * 16 + n) * kRowBytes<STEPS> + 16 * g;
                i32x4 q[STEPS];
                float z[4];
#pragma unroll
                for (int k = 0; k < STEPS; ++k) q[k] = *(const i32x4*)(row_at + 64 * k);
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = unit[tile * 16 + 4 * g + i];
                // the page that each value's token is in (below 0: the lane writes no key)
                int32_t cur[V];
                int64_t to[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int32_t row = 4 * g + v * (4 / V), at = row >> F.per_bits;
                    const int32_t slot = one ? 0 : tile * F.slots + at;
                    const int64_t pos = pos0 + (slot - s0);
                    const bool writes = (row & (F.per - 1)) == 0 && at < F.slots && slot >= s0 && slot < s_end;
                    cur[v] = !writes ? -2 : pos < 0 ? -1 : (int32_t)div_u32((uint32_t)pos, c.div_page);
                    to[v] = ((t0 + slot) * c.n_kv_heads + kvh) * c.table_width + p0 + n;
                }
#pragma unroll
                for (int u = 0; u < kSub; ++u) {
                    i32x4 acc = {0, 0, 0, 0};
#pragma unroll
                    for (int k = 0; k < STEPS; ++k)
                        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[k], a[u][k], acc, 0, 0, 0);
                    float m[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) m[i] = z[i] * (float)acc[i];
                    if constexpr (V == 2) {
                        m[0] = fmaxf(m[0], m[1]);
                        m[1] = fmaxf(m[2], m[3]);
                    }
                    if constexpr (V == 1) {
                        m[0] = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
                        if (F.per >= 8) m[0] = fmaxf(m[0], __shfl_xor(m[0], 16));
                        if (F.per >= 16) m[0] = fmaxf(m[0], __shfl_xor(m[0], 32));
                    }
#pragma unroll
                    for (int v = 0; v < V; ++v) top[u][v] = one && tile > 0 ? fmaxf(top[u][v], m[v]) : m[v];
                    const int32_t j = (int32_t)p0 + u * 16 + n;
                    if ((one && tile + 1 < tile1) || j >= p_end) continue;
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if (cur[v] < -1) continue;
                        uint32_t key = kNoPage;
                        if (there[u] && j <= cur[v]) {
                            if (j < P.first || j > cur[v] - P.last) key = kAlways;
                            else key = order_of(__builtin_isfinite(scale[u]) ? top[u][v] * scale[u] : INFINITY);
                        }
                        F.keys[to[v] + u * 16] = key;
                    }
                }
            }
        }
        s0 = s_end;
    }
}

// ---------------------------------------------------------------- the choice

// The K best pages of one token and KV head, in ascending order: the K-th
// largest key by digits of 8 bits, from the top bit in which the keys differ, then the
// pages above it and as many of those equal to it, lowest first, as are left.  Bound
// by latency: WAVES wavefronts keep HELD keys a lane in registers, the others are read
// again for each digit.  512 choices of up to 2305 pages take 8.3 us, 8192 of up to 683 21.
template <int WAVES, int HELD>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void pick_kernel(ScoreLaunch F, int64_t first) {
    constexpr int kThreads = WAVES * kWave, kItems = WAVES == 1 ? 4 : 1;
    struct Lds {
        int32_t count[256];
        uint32_t found[3];
        uint32_t low[WAVES], high[WAVES];
        int32_t above[WAVES], ties[WAVES];
    };
    __shared__ Lds all[kItems];
    const SelectPagesParams& P = F.s;
    const CacheView& c = P.c;
    const int w = wave_number(), lane = lane_id();
    const int wave = WAVES == 1 ? 0 : w, tid = wave * kWave + lane;
    Lds& lds = all[WAVES == 1 ? w : 0];
    auto sync = [] {
        if constexpr (WAVES > 1) {
            __syncthreads();
        } else {
            // (a wavefront's own LDS operations are in order; the compiler keeps them so)
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    };
    const int64_t x = (blockIdx.x + first) * kItems + (WAVES == 1 ? w : 0);
    const int64_t i = F.token0 + x / c.n_kv_heads;
    int64_t b;
    if (x >= F.tokens * c.n_kv_heads || !find_seq(c, i, &b)) return;
    const SeqRows s = seq_rows(c, b);
    if (i < s.first || i - s.first >= s.n) return;
    const int64_t pos = (int64_t)s.length - s.n + (i - s.first);
    const int64_t last = min(pos, table_tokens(c) - 1);
    const int32_t n = last < 0 ? 0 : (int32_t)(div_u32((uint32_t)last, c.div_page) + 1);
    const uint32_t* const keys = F.keys + x * c.table_width;
    int32_t* const out = P.selected + (F.token0 * c.n_kv_heads + x) * P.n_select;

    // a wavefront's keys are consecutive: key p0 + 64 e + lane
    const int32_t chunk = ((n + WAVES - 1) / WAVES + kWave - 1) / kWave * kWave;
    const int32_t p0 = min(wave * chunk, n), p1 = min(p0 + chunk, n);
    uint32_t held[HELD];
#pragma unroll
    for (int e = 0; e < HELD; ++e) held[e] = p0 + e * kWave + lane < p1 ? keys[p0 + e * kWave + lane] : kNoPage;
    auto each = [&](auto f) {
#pragma unroll
        for (int e = 0; e < HELD; ++e)
            if (e * kWave < p1 - p0) f(p0 + e * kWave + lane, held[e]);
        for (int32_t p = p0 + HELD * kWave; p < p1; p += kWave) f(p + lane, p + lane < p1 ? keys[p + lane] : kNoPage);
    };

    uint32_t threshold = 0;
    int32_t left = 0;                       // of the keys equal to the threshold
    if (n > P.n_select) {
        // the keys that are not taken anyway lie in [low, high]
        uint32_t low = kAlways, high = 0;
        int32_t always = 0, real = 0;
        each([&](int32_t, uint32_t k) {
            always += __popcll(__ballot(k == kAlways));
            real += __popcll(__ballot(k != kNoPage));
            if (k != kNoPage && k != kAlways) {
                low = min(low, k);
                high = max(high, k);
            }
        });
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            low = min(low, (uint32_t)__shfl_xor((int)low, o));
            high = max(high, (uint32_t)__shfl_xor((int)high, o));
        }
        if constexpr (WAVES > 1) {
            if (lane == 0) {
                lds.low[wave] = low;
                lds.high[wave] = high;
                lds.above[wave] = always;
                lds.ties[wave] = real;
            }
            __syncthreads();
            always = real = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                low = min(low, lds.low[w]);
                high = max(high, lds.high[w]);
                always += lds.above[w];
                real += lds.ties[w];
            }
            __syncthreads();
        }
        left = P.n_select - always;
        if (real <= P.n_select) {
            left = 0;                       // all candidates
        } else if (left <= 0) {
            threshold = kAlways;
            left = P.n_select;
        } else {
            // digits from the highest bit in which low and high differ
            int bits = low == high ? 0 : 32 - __builtin_clz(low ^ high);
            uint32_t mask = bits >= 32 ? 0 : ~0u << bits;
            threshold = high & mask;
            while (bits > 0) {
                const int take = min(bits, 8), shift = bits - take;
                const uint32_t digits = (1u << take) - 1;
                for (int k = tid; k < 256; k += kThreads) lds.count[k] = 0;
                sync();
                each([&](int32_t, uint32_t k) {
                    if (k != kNoPage && k != kAlways && (k & mask) == threshold) atomicAdd(&lds.count[k >> shift & digits], 1);
                });
                sync();
                if (wave == 0) {
                    // lane l has the digits 255 - 4 l .. 252 - 4 l
                    int32_t d[4], sum = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        d[e] = lds.count[255 - 4 * lane - e];
                        sum += d[e];
                    }
                    int32_t at = wave_incl_scan(sum) - sum;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (at < left && at + d[e] >= left) {
                            lds.found[0] = (uint32_t)(255 - 4 * lane - e);
                            lds.found[1] = (uint32_t)(left - at);
                            lds.found[2] = (uint32_t)d[e];
                        }
                        at += d[e];
                    }
                }
                sync();
                threshold |= lds.found[0] << shift;
                mask |= digits << shift;
                left = (int32_t)lds.found[1];
                const bool done = lds.found[2] == (uint32_t)left;       // all keys of this prefix
                sync();
                if (done && shift > 0) {
                    // every key from here up is taken
                    left = 0;
                    threshold = threshold ? threshold - 1 : 0;
                    break;
                }
                bits = shift;
            }
        }
    }
    // a key above the threshold, or one equal to it among the first `left`; no
    // candidate (kNoPage) is never taken
    int32_t above = 0, ties = 0;
    each([&](int32_t, uint32_t k) {
        above += __popcll(__ballot(k > threshold));
        ties += __popcll(__ballot(k == threshold && k != kNoPage));
    });
    int32_t a0 = 0, e0 = 0, all_above = above, all_ties = ties;
    if constexpr (WAVES > 1) {
        if (lane == 0) {
            lds.above[wave] = above;
            lds.ties[wave] = ties;
        }
        __syncthreads();
        all_above = all_ties = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            a0 += w < wave ? lds.above[w] : 0;
            e0 += w < wave ? lds.ties[w] : 0;
            all_above += lds.above[w];
            all_ties += lds.ties[w];
        }
    }
    const uint64_t below = (1ull << lane) - 1;
    each([&](int32_t p, uint32_t k) {
        const bool is_above = k > threshold, is_tie = k == threshold && k != kNoPage;
        const uint64_t ma = __ballot(is_above), me = __ballot(is_tie);
        const int32_t ra = a0 + (int32_t)__popcll(ma & below), re = e0 + (int32_t)__popcll(me & below);
        if (is_above || (is_tie && re < left)) out[ra + min(re, left)] = p;
        a0 += __popcll(ma);
        e0 += __popcll(me);
    });
    for (int32_t k = all_above + min(all_ties, left) + tid; k < P.n_select; k += kThreads) out[k] = -1;
}

// One wavefront holds up to 1024 pages (8192 choices of 683: 41.8 us with four
// of them and digits from the top), four up to 4096.
template <int WAVES, int HELD>
hipError_t launch_pick(const ScoreLaunch& f, hipStream_t stream) {
    const int64_t items = f.tokens * f.s.c.n_kv_heads, blocks = WAVES == 1 ? (items + 3) / 4 : items;
    const int threads = WAVES == 1 ? 256 : WAVES * kWave;
    return launch_all(blocks, threads, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((pick_kernel<WAVES, HELD>), grid, dim3(threads), 0, stream, f, first);
    });
}

int64_t key_bytes(const SelectPagesParams& p, int64_t tokens) {
    return tokens * p.c.n_kv_heads * p.c.table_width * (int64_t)sizeof(uint32_t);
}

template <bool F16, int STEPS, int V>
hipError_t launch_values(const ScoreLaunch& f, int64_t blocks, hipStream_t stream) {
    const size_t lds = (size_t)f.tiles * 16 * (kRowBytes<STEPS> + sizeof(float));
    return launch_all(blocks, kScoreThreads, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((score_kernel<F16, STEPS, V>), grid, dim3(kScoreThreads), lds, stream, f, first);
    });
}

template <bool F16, int STEPS>
hipError_t launch_steps(const ScoreLaunch& f, int64_t blocks, hipStream_t stream) {
    if (f.per == 1) return launch_values<F16, STEPS, 4>(f, blocks, stream);
    if (f.per == 2) return launch_values<F16, STEPS, 2>(f, blocks, stream);
    return launch_values<F16, STEPS, 1>(f, blocks, stream);
}

template <bool F16>
hipError_t launch_scores(const ScoreLaunch& f, int64_t blocks, hipStream_t stream) {
    const int d = f.s.c.head_dim;
    if (d <= 32) return launch_steps<F16, 1>(f, blocks, stream);
    if (d <= 64) return launch_steps<F16, 2>(f, blocks, stream);
    if (d <= 128) return launch_steps<F16, 4>(f, blocks, stream);
    return launch_steps<F16, 8>(f, blocks, stream);
}

}  // namespace

// More than this no memory could back (sequences without rows count too).
constexpr int64_t kMostBlocks = INT32_MAX;

int64_t bounds_slots(const CacheView& c) {
    return c.q_offset ? c.n_tokens / c.page_tokens + 2 * c.n_seqs : c.n_seqs;
}

hipError_t launch_page_bounds(const BoundsParams& q, hipStream_t stream) {
    BoundsParams p = q;
    p.slots = bounds_slots(p.c);
    int lanes = 1;
    while (lanes * 8 < p.c.head_dim) lanes *= 2;
    if (p.slots > kMostBlocks / p.c.n_kv_heads) return hipErrorInvalidConfiguration;
    const int64_t blocks = (p.slots * p.c.n_kv_heads + kBoundsWaves - 1) / kBoundsWaves;
    const bool few = p.c.page_tokens <= 4 * (kWave / lanes);
    return launch_all(blocks, kBoundsThreads, [&](dim3 grid, int64_t first) {
        const dim3 block(kBoundsThreads);
        if (p.f16 && few) hipLaunchKernelGGL((bounds_kernel<true, 4>), grid, block, 0, stream, p, lanes, first);
        else if (p.f16) hipLaunchKernelGGL((bounds_kernel<true, 8>), grid, block, 0, stream, p, lanes, first);
        else if (few) hipLaunchKernelGGL((bounds_kernel<false, 4>), grid, block, 0, stream, p, lanes, first);
        else hipLaunchKernelGGL((bounds_kernel<false, 8>), grid, block, 0, stream, p, lanes, first);
    });
}

// Tiles of rows that a workgroup scores the pages that it reads for.
constexpr int kSharedTiles = 8;

// Scores of up to so many bytes at once; of more tokens in several launches.
constexpr int64_t kMostKeys = 256ll << 20;

uint64_t select_workspace_least(const SelectPagesParams& p) { return (uint64_t)key_bytes(p, 1); }
uint64_t select_workspace_bytes(const SelectPagesParams& p) {
    if (p.c.n_tokens == 0 || p.c.n_seqs == 0) return 0;
    return (uint64_t)std::max(key_bytes(p, 1), std::min(key_bytes(p, p.c.n_tokens), kMostKeys));
}

hipError_t launch_select_pages(const SelectPagesParams& p, hipStream_t stream) {
    ScoreLaunch f{};
    f.s = p;
    f.per = 1;
    while (f.per < p.group && f.per < 16) f.per *= 2, ++f.per_bits;
    // tokens of one sequence share what is read; single ones of several do not
    const bool share = p.c.q_offset && p.c.n_tokens > 2 * p.c.n_seqs;
    f.slots = share ? 16 / f.per : 1;
    f.tiles = p.group > 16 ? (p.group + 15) / 16 : share ? kSharedTiles : 1;
    f.tokens_of = p.group > 16 ? 1 : f.slots * f.tiles;
    f.keys = (uint32_t*)p.workspace;
    const int64_t one = key_bytes(p, 1);
    const int64_t slab = one ? std::min<int64_t>(p.c.n_tokens, (int64_t)(p.workspace_bytes / (uint64_t)one)) : p.c.n_tokens;
    for (f.token0 = 0; f.token0 < p.c.n_tokens; f.token0 += slab) {
        f.tokens = std::min(slab, p.c.n_tokens - f.token0);
        const int64_t row_tiles = (f.tokens + f.tokens_of - 1) / f.tokens_of * p.c.n_kv_heads;
        // spans of pages until the chip is full
        const int32_t round = kScoreWaves * (p.c.head_dim > 128 ? kPagesOfStep<8> : kPagesOfStep<4>);
        const int64_t steps = ((int64_t)p.c.table_width + round - 1) / round;
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>(steps, (4096 + row_tiles - 1) / std::max<int64_t>(row_tiles, 1)));
        f.span = (int32_t)std::min<int64_t>((steps + want - 1) / want * round, INT32_MAX);
        f.spans = f.span ? (int32_t)((p.c.table_width + (int64_t)f.span - 1) / f.span) : 0;
        hipError_t e = hipSuccess;
        if (f.spans > 0)
            e = p.f16 ? launch_scores<true>(f, row_tiles * f.spans, stream) : launch_scores<false>(f, row_tiles * f.spans, stream);
        if (e != hipSuccess) return e;
        e = p.c.table_width <= 1024 ? launch_pick<1, 16>(f, stream) : launch_pick<4, 16>(f, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tl
