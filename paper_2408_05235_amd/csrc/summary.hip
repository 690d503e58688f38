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

// A wavefront per slot and KV head: `lanes` lanes (a power of two of at least
// head_dim / 8) take 8 elements each of a token, the others other tokens.
template <bool F16>
__global__ __launch_bounds__(kBoundsThreads) void bounds_kernel(BoundsParams P, int lanes, int64_t first) {
    const CacheView& c = P.c;
    const int64_t item = (blockIdx.x + first) * kBoundsWaves + threadIdx.x / kWave;
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
    float hi[8], lo[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) hi[i] = -INFINITY, lo[i] = INFINITY;
    bool special = false;
    if (in) {
#pragma unroll 4
        for (int r = sub; r < count; r += per) {
            const u32x4 v = *(const u32x4*)(keys + (int64_t)r * c.token_stride);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                special |= not_finite2<F16>(v[i]);
                const float a = to_float<F16>((uint16_t)v[i]), z = to_float<F16>((uint16_t)(v[i] >> 16));
                hi[2 * i] = fmaxf(hi[2 * i], a);
                lo[2 * i] = fminf(lo[2 * i], a);
                hi[2 * i + 1] = fmaxf(hi[2 * i + 1], z);
                lo[2 * i + 1] = fminf(lo[2 * i + 1], z);
            }
        }
    }
    for (int o = lanes; o < kWave; o <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], o));
            lo[i] = fminf(lo[i], __shfl_xor(lo[i], o));
        }
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = in ? fmaxf(most, fmaxf(hi[i], -lo[i])) : most;
    for (int o = 1; o < lanes; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
    // (the same in every lane group; a product and not a quotient, as stated in tl.h)
    const bool bad = __any(special);
    const float scale = bad ? INFINITY : most * kInv127;
    // (a largest value so small that its 127th is 0 counts as 0)
    const bool none = bad || scale == 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hi[i] = none ? 0.0f : fminf(fmaxf(ceilf(hi[i] / scale), -127.0f), 127.0f);
        lo[i] = none ? 0.0f : fminf(fmaxf(floorf(lo[i] / scale), -127.0f), 127.0f);
    }
    const int64_t at = (int64_t)page * c.n_kv_heads + kvh;
    if (sub == 0 && in) {
        int8_t* const to = P.bounds + at * 2 * c.head_dim + piece * 8;
        *(uint2*)to = make_uint2(pack_bytes(lo, 0), pack_bytes(lo, 4));
        *(uint2*)(to + c.head_dim) = make_uint2(pack_bytes(hi, 0), pack_bytes(hi, 4));
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

// A workgroup scores a range of pages for a tile of rows of one KV head.  A tile
// is `slots` tokens of `per` rows each (query heads of the KV head; per: the next
// power of two of them), or a token's heads in `tiles` times 16 rows.  Lane (n =
// lane % 16, g = lane / 16) holds the bytes 64 k + 16 g .. of row n and of page n (K =
// 64 bytes a matrix instruction), and of the result the rows 4 g .. 4 g + 3 of page n.
struct ScoreLaunch {
    SelectPagesParams s;
    int32_t per, slots, tiles;
    int32_t span;           // pages of a workgroup
    int32_t spans;          // workgroups of a row tile
    int64_t token0, tokens; // the tokens of this launch
    uint32_t* keys;         // [tokens][n_kv_heads][table_width]
};

// Bytes of a row in LDS: the least elements' share (min(i, 0)), the largest's
// (max(i, 0)), zeros; a piece more, so that rows do not begin in one bank.
template <int STEPS>
constexpr int kRowBytes = STEPS * 64 + 16;

template <bool F16, int STEPS>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(ScoreLaunch F, int64_t first) {
    extern __shared__ __attribute__((aligned(16))) unsigned char rows_lds[];
    const SelectPagesParams& P = F.s;
    const CacheView& c = P.c;
    const int wave = threadIdx.x / kWave, lane = lane_id(), n = lane & 15, g = lane >> 4;
    const int D = c.head_dim, n_rows = F.tiles * 16;
    float* const unit = (float*)(rows_lds + n_rows * kRowBytes<STEPS>);
    int64_t x = blockIdx.x + first;
    const int32_t span = (int32_t)(x % F.spans);
    x /= F.spans;
    const int32_t kvh = (int32_t)(x % c.n_kv_heads);
    const int64_t t0 = x / c.n_kv_heads * F.slots;          // of this launch

    // the rows in 127ths of their largest value
    for (int row = wave; row < n_rows; row += kScoreWaves) {
        const int32_t slot = F.tiles > 1 ? 0 : row / F.per, head = F.tiles > 1 ? row : row % F.per;
        const bool real = slot < F.slots && t0 + slot < F.tokens && head < P.group;
        const int d = lane * 8;
        float q[8] = {};
        bool special = false;
        if (real && d < D) {
            const u32x4 v = *(const u32x4*)(P.query + (F.token0 + t0 + slot) * P.query_token_stride +
                                            (int64_t)(kvh * P.group + head) * P.query_head_stride + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                special |= not_finite2<F16>(v[i]);
                q[2 * i] = to_float<F16>((uint16_t)v[i]);
                q[2 * i + 1] = to_float<F16>((uint16_t)(v[i] >> 16));
            }
        }
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(q[i]));
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
        most = __shfl(most, 0);                             // (lanes 32 and up hold no elements)
        const float z = __any(special) ? 0.0f : most * kInv127;
        float low[8], high[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float r = z > 0.0f ? rintf(q[i] / z) : 0.0f;
            low[i] = fminf(r, 0.0f);
            high[i] = fmaxf(r, 0.0f);
        }
        unsigned char* const to = rows_lds + row * kRowBytes<STEPS>;
        if (d < D) {
            *(uint2*)(to + d) = make_uint2(pack_bytes(low, 0), pack_bytes(low, 4));
            *(uint2*)(to + D + d) = make_uint2(pack_bytes(high, 0), pack_bytes(high, 4));
        }
        for (int o = 2 * D + lane * 8; o < STEPS * 64; o += kWave * 8) *(uint2*)(to + o) = make_uint2(0, 0);
        if (lane == 0) unit[row] = z;
    }
    __syncthreads();

    auto fragment = [&](int tile, int k) {
        return *(const i32x4*)(rows_lds + (tile * 16 + n) * kRowBytes<STEPS> + 64 * k + 16 * g);
    };
    i32x4 q[STEPS];
    float z[4];
#pragma unroll
    for (int k = 0; k < STEPS; ++k) q[k] = fragment(0, k);
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = unit[4 * g + i];

    // The tile's tokens can be of several sequences, whose pages differ: each
    // sequence in its turn.
    for (int32_t s0 = 0; s0 < F.slots;) {
        const int64_t i0 = F.token0 + t0 + s0;
        if (t0 + s0 >= F.tokens) return;
        int64_t b;
        const bool of_one = find_seq(c, i0, &b);
        const SeqRows s = of_one ? seq_rows(c, b) : SeqRows{};
        if (!of_one || i0 < s.first || i0 - s.first >= s.n) {
            ++s0;
            continue;
        }
        const int32_t many = (int32_t)min(min((int64_t)(F.slots - s0), s.first + s.n - i0), F.tokens - t0 - s0);
        const int32_t s_end = s0 + many;
        const int64_t pos0 = (int64_t)s.length - s.n + (i0 - s.first);
        // pages that the last of these tokens sees
        const int64_t last = min(pos0 + many - 1, table_tokens(c) - 1);
        const int32_t pages = last < 0 ? 0 : (int32_t)(div_u32((uint32_t)last, c.div_page) + 1);
        const int32_t p_end = (int32_t)min((int64_t)pages, (int64_t)(span + 1) * F.span);
        const int32_t* const table_row = c.table + b * c.table_width;
        for (int64_t p0 = (int64_t)span * F.span + wave * 16; p0 < p_end; p0 += kScoreWaves * 16) {
            const int32_t j = (int32_t)p0 + n;
            const int32_t page = j < p_end ? table_row[j] : -1;
            const bool there = page >= 0 && page < c.n_pages;
            const int64_t at = ((int64_t)(there ? page : 0) * c.n_kv_heads + kvh) * 2 * D;
            i32x4 a[STEPS];
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                const int d = 64 * k + 16 * g;
                a[k] = i32x4{0, 0, 0, 0};
                if (there && d < 2 * D) a[k] = *(const i32x4*)(P.bounds + at + d);
            }
            const float scale = there ? P.scale[(int64_t)page * P.scale_stride + kvh] : 0.0f;
            float top[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) top[i] = -INFINITY;
            for (int tile = 0; tile < F.tiles; ++tile) {
                if (F.tiles > 1) {
#pragma unroll
                    for (int k = 0; k < STEPS; ++k) q[k] = fragment(tile, k);
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = unit[tile * 16 + 4 * g + i];
                }
                i32x4 acc = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < STEPS; ++k) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[k], a[k], acc, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 4 * g + i, head = F.tiles > 1 ? tile * 16 + row : row % F.per;
                    if (head < P.group) top[i] = fmaxf(top[i], z[i] * (float)acc[i]);
                }
            }
            if (F.per >= 2) {
                top[0] = fmaxf(top[0], top[1]);
                top[2] = fmaxf(top[2], top[3]);
            }
            if (F.per >= 4) top[0] = fmaxf(top[0], top[2]);
            if (F.per >= 8) top[0] = fmaxf(top[0], __shfl_xor(top[0], 16));
            if (F.per >= 16) top[0] = fmaxf(top[0], __shfl_xor(top[0], 32));
            if (j < p_end) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t slot = (4 * g + i) / F.per;
                    if ((4 * g + i) % F.per != 0 || slot < s0 || slot >= s_end) continue;
                    const int64_t pos = pos0 + (slot - s0);
                    uint32_t key = kNoPage;
                    if (there && pos >= 0 && (int64_t)j * c.page_tokens <= pos) {
                        const int32_t cur = (int32_t)div_u32((uint32_t)pos, c.div_page);
                        if (j < P.first || j > cur - P.last) key = kAlways;
                        else key = order_of(__builtin_isfinite(scale) ? top[i] * scale : INFINITY);
                    }
                    F.keys[((t0 + slot) * c.n_kv_heads + kvh) * c.table_width + j] = key;
                }
            }
        }
        s0 = s_end;
    }
}

// ---------------------------------------------------------------- the choice

constexpr int kPickThreads = 256, kPickWaves = kPickThreads / kWave;

// The K best pages of one token and KV head, in ascending order: the K-th
// largest key by its digits of 8 bits, from the top, then the pages above it and as
// many of those equal to it, lowest first, as are left.
__global__ __launch_bounds__(kPickThreads) void pick_kernel(ScoreLaunch F, int64_t first) {
    const SelectPagesParams& P = F.s;
    const CacheView& c = P.c;
    const int64_t x = blockIdx.x + first;
    const int64_t i = F.token0 + x / c.n_kv_heads;
    int64_t b;
    if (!find_seq(c, i, &b)) return;
    const SeqRows s = seq_rows(c, b);
    if (i < s.first || i - s.first >= s.n) return;
    const int64_t pos = (int64_t)s.length - s.n + (i - s.first);
    const int64_t last = min(pos, table_tokens(c) - 1);
    const int32_t n = last < 0 ? 0 : (int32_t)(div_u32((uint32_t)last, c.div_page) + 1);
    const uint32_t* const keys = F.keys + x * c.table_width;
    int32_t* const out = P.selected + (F.token0 * c.n_kv_heads + x) * P.n_select;

    __shared__ int32_t count[256];
    __shared__ uint32_t found[2];
    __shared__ int32_t wave_above[kPickWaves], wave_ties[kPickWaves];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    uint32_t prefix = 0, mask = 0;
    int32_t left = P.n_select;              // rank of the K-th among those that match the prefix
    if (n <= P.n_select) {
        // all that are candidates: keys above kNoPage
        left = 0;
    } else {
        for (int shift = 24; shift >= 0; shift -= 8) {
            count[threadIdx.x] = 0;
            __syncthreads();
            for (int32_t p = threadIdx.x; p < n; p += kPickThreads) {
                const uint32_t k = keys[p];
                if ((k & mask) == prefix) atomicAdd(&count[k >> shift & 255], 1);
            }
            __syncthreads();
            if (wave == 0) {
                // lane l has the digits 255 - 4 l .. 252 - 4 l
                int32_t d[4], sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    d[e] = count[255 - 4 * lane - e];
                    sum += d[e];
                }
                const int32_t before = wave_incl_scan(sum) - sum;
                int32_t at = before;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (at < left && at + d[e] >= left) {
                        found[0] = (uint32_t)(255 - 4 * lane - e);
                        found[1] = (uint32_t)(left - at);
                    }
                    at += d[e];
                }
            }
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= 255u << shift;
            left = (int32_t)found[1];
        }
    }
    // a key above `prefix`, or one equal to it among the first `left`; no
    // candidate (kNoPage) is never taken
    const int32_t chunk = (n + kPickWaves - 1) / kPickWaves, p0 = wave * chunk, p1 = min(p0 + chunk, n);
    int32_t above = 0, ties = 0;
    for (int32_t p = p0; p < p1; p += kWave) {
        const uint32_t k = p + lane < p1 ? keys[p + lane] : kNoPage;
        above += __popcll(__ballot(k > prefix));
        ties += __popcll(__ballot(k == prefix && k != kNoPage));
    }
    if (lane == 0) {
        wave_above[wave] = above;
        wave_ties[wave] = ties;
    }
    __syncthreads();
    int32_t a0 = 0, e0 = 0;
    for (int w = 0; w < wave; ++w) {
        a0 += wave_above[w];
        e0 += wave_ties[w];
    }
    const uint64_t below = (1ull << lane) - 1;
    for (int32_t p = p0; p < p1; p += kWave) {
        const uint32_t k = p + lane < p1 ? keys[p + lane] : kNoPage;
        const uint64_t ma = __ballot(k > prefix), me = __ballot(k == prefix && k != kNoPage);
        const int32_t ra = a0 + __popcll(ma & below), re = e0 + __popcll(me & below);
        if (k > prefix || (k == prefix && k != kNoPage && re < left)) out[ra + min(re, left)] = p + lane;
        a0 += __popcll(ma);
        e0 += __popcll(me);
    }
    int32_t all_above = 0, all_ties = 0;
    for (int w = 0; w < kPickWaves; ++w) {
        all_above += wave_above[w];
        all_ties += wave_ties[w];
    }
    for (int32_t k = all_above + min(all_ties, left) + (int32_t)threadIdx.x; k < P.n_select; k += kPickThreads) out[k] = -1;
}

int64_t key_bytes(const SelectPagesParams& p, int64_t tokens) {
    return tokens * p.c.n_kv_heads * p.c.table_width * (int64_t)sizeof(uint32_t);
}

template <bool F16, int STEPS>
hipError_t launch_steps(const ScoreLaunch& f, int64_t blocks, hipStream_t stream) {
    const size_t lds = (size_t)f.tiles * 16 * (kRowBytes<STEPS> + sizeof(float));
    return launch_all(blocks, kScoreThreads, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((score_kernel<F16, STEPS>), grid, dim3(kScoreThreads), lds, stream, f, first);
    });
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

int64_t bounds_slots(const CacheView& c) {
    return c.q_offset ? c.n_tokens / c.page_tokens + 2 * c.n_seqs : c.n_seqs;
}

hipError_t launch_page_bounds(const BoundsParams& q, hipStream_t stream) {
    BoundsParams p = q;
    p.slots = bounds_slots(p.c);
    int lanes = 1;
    while (lanes * 8 < p.c.head_dim) lanes *= 2;
    const int64_t blocks = (p.slots * p.c.n_kv_heads + kBoundsWaves - 1) / kBoundsWaves;
    return launch_all(blocks, kBoundsThreads, [&](dim3 grid, int64_t first) {
        if (p.f16) hipLaunchKernelGGL((bounds_kernel<true>), grid, dim3(kBoundsThreads), 0, stream, p, lanes, first);
        else hipLaunchKernelGGL((bounds_kernel<false>), grid, dim3(kBoundsThreads), 0, stream, p, lanes, first);
    });
}

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
    while (f.per < p.group && f.per < 16) f.per *= 2;
    f.tiles = (p.group + 15) / 16;
    // tokens of one sequence share what is read; single ones of several do not
    f.slots = p.c.q_offset && p.c.n_tokens > 2 * p.c.n_seqs ? 16 / f.per : 1;
    f.keys = (uint32_t*)p.workspace;
    const int64_t one = key_bytes(p, 1);
    const int64_t slab = one ? std::min<int64_t>(p.c.n_tokens, (int64_t)(p.workspace_bytes / (uint64_t)one)) : p.c.n_tokens;
    for (f.token0 = 0; f.token0 < p.c.n_tokens; f.token0 += slab) {
        f.tokens = std::min(slab, p.c.n_tokens - f.token0);
        const int64_t row_tiles = (f.tokens + f.slots - 1) / f.slots * p.c.n_kv_heads;
        // spans of pages until the chip is full
        const int64_t steps = ((int64_t)p.c.table_width + 63) / 64;
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>(steps, (2048 + row_tiles - 1) / std::max<int64_t>(row_tiles, 1)));
        f.span = (int32_t)((steps + want - 1) / std::max<int64_t>(want, 1) * 64);
        f.spans = f.span ? (int32_t)((p.c.table_width + (int64_t)f.span - 1) / f.span) : 0;
        hipError_t e = hipSuccess;
        if (f.spans > 0)
            e = p.f16 ? launch_scores<true>(f, row_tiles * f.spans, stream) : launch_scores<false>(f, row_tiles * f.spans, stream);
        if (e != hipSuccess) return e;
        e = launch_all(f.tokens * p.c.n_kv_heads, kPickThreads, [&](dim3 grid, int64_t first) {
            hipLaunchKernelGGL(pick_kernel, grid, dim3(kPickThreads), 0, stream, f, first);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tl
