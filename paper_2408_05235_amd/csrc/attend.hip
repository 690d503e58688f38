// Attention of new tokens over the paged cache (tl_attend): the launch where
// every sequence has one new token (or all few), the join of split sequences, and
// the dispatch.
//
// Rows of a sequence and a KV head are its new tokens times the query heads
// that share the head.  Sequences of up to 16 rows (one new token, or a few) are
// bound by reading their keys and values once (few_rows), long prompts by the
// matrix products (tile_rows, which takes all sequences of more than 16 rows that
// offsets are given for).  Without offsets, one new token each, every sequence is
// few_rows': for more than 16 heads on a KV head in as many workgroups of 16 rows as it
// takes, each of which reads the keys and values.
#include <hip/hip_runtime.h>

#include <float.h>

#include <algorithm>

#include "attend_common.h"
#include "attend_few.h"
#include "cache.h"
#include "cache_rows.h"
#include "device_util.h"
#include "tl_internal.h"

namespace tl {
namespace {

constexpr int kFewWaves = 4, kFewThreads = kFewWaves * kWave;

// Bound by reading: 256 sequences of up to 4352 tokens, 20 heads with their
// own keys, take 0.90 ms, 6.3 TB/s (reading 4 GiB with such loads and nothing
// else reaches 7.1, a copy of 2 GiB 4.95).  Three
// wavefronts a SIMD (12 steps of 16 KB on their way in a CU): 0.93 ms with two, and
// 97 and 108 us for 4 sequences of 20011 to 36864 tokens.  (Two of a workgroup of
// eight: wide_few.)
template <bool F16, int DP, bool EXACT, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, DP > 128 ? 1 : WAVES > 4 ? 2 : 3) void few_rows_kernel(AttendLaunch F,
                                                                                                  int64_t first) {
    __shared__ FewLds<WAVES, DP> lds;
    few_rows<F16, DP, EXACT, WAVES, true>(F, blockIdx.x + first, lds);
}

// Four wavefronts per slot where there are many parts, else one: first the
// slots of few_rows, then those of tile_rows.  4 us with its launch where there is
// little to join.  With four: 8 heads of 36864 tokens, 96 parts, attention and
// join 37.3 us, 47.9 with one; 1 head of 131072, 229 parts, 32.8 and 61.2.  Of a few parts
// each one is better (384 rows of 2: 76.9 and 78.3 us; 1024 of 9, with tile_rows: 19.2 and
// 20.6).
template <bool F16, int LANES, int WAVES>
__global__ __launch_bounds__(kFewThreads) void join_kernel(AttendLaunch F, int64_t few_slots, int64_t first) {
    const AttendParams& P = F.a;
    const CacheView& c = P.c;
    const int64_t block = blockIdx.x + first;
    const int64_t slot = WAVES > 1 ? block : block * kFewWaves + threadIdx.x / kWave;
    if (slot < few_slots) {
        const int64_t x = slot / F.slot_rows, row = slot % F.slot_rows;
        const int32_t kvh = (int32_t)(x % c.n_kv_heads);
        const int64_t b = x / c.n_kv_heads;
        const SeqRows s = seq_rows(c, b);
        const int64_t rows = (int64_t)s.n * P.group;
        if ((c.q_offset && rows > kFewRows) || row >= rows) return;
        const int64_t token = row / P.group;
        join_row<F16, LANES, WAVES>(F, F.few, slot,
                                    (s.first + token) * P.n_heads + kvh * P.group + (row - token * P.group), 1.0f);
        return;
    }
    const int64_t to = slot - few_slots, i = to / P.n_heads;
    int64_t b;
    if (i >= c.n_tokens || !find_seq(c, i, &b)) return;
    const SeqRows s = seq_rows(c, b);
    if (i < s.first || i - s.first >= s.n || (int64_t)s.n * P.group <= kFewRows) return;
    join_row<F16, LANES, WAVES>(F, F.tiles, to, to, kUnliftTiles<F16>);
}

template <bool F16, int DP, int WAVES>
hipError_t launch_waves(const AttendLaunch& f, int64_t blocks, hipStream_t stream) {
    return launch_all(blocks * f.few.count, WAVES * kWave, [&](dim3 grid, int64_t first) {
        const dim3 block(WAVES * kWave);
        if (f.a.c.head_dim == DP)
            hipLaunchKernelGGL((few_rows_kernel<F16, DP, true, WAVES>), grid, block, 0, stream, f, first);
        else hipLaunchKernelGGL((few_rows_kernel<F16, DP, false, WAVES>), grid, block, 0, stream, f, first);
    });
}

template <bool F16, int DP>
hipError_t launch_few(const AttendLaunch& f, int64_t blocks, hipStream_t stream) {
    if constexpr (DP <= 128)
        if (f.wide) return launch_waves<F16, DP, 2 * kFewWaves>(f, blocks, stream);
    return launch_waves<F16, DP, kFewWaves>(f, blocks, stream);
}

template <bool F16, int DP>
hipError_t launch_join(const AttendLaunch& f, int64_t few_slots, int64_t tile_slots, hipStream_t stream) {
    const int64_t slots = few_slots + tile_slots;
    if (std::max(f.few.count, f.tiles.count) > 16)
        return launch_all(slots, kFewThreads, [&](dim3 grid, int64_t first) {
            hipLaunchKernelGGL((join_kernel<F16, DP / 4, kFewWaves>), grid, dim3(kFewThreads), 0, stream, f, few_slots,
                               first);
        });
    return launch_all((slots + kFewWaves - 1) / kFewWaves, kFewThreads, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((join_kernel<F16, DP / 4, 1>), grid, dim3(kFewThreads), 0, stream, f, few_slots, first);
    });
}

// Row tiles of a sequence and head for few_rows, its workgroups per part, and
// slots of a sequence and head, and of all.  (More than one row tile against
// tile_rows, which the same call with offsets gets, us: 64 sequences of 16 to 1280
// tokens with 32, 64 and 71 heads on one 21, 30, 37 and 28, 31, 34; 256 of 500 27, 50, 62
// and 39, 40, 41; 8 of 20000 34, 51, 79 and 42, 42, 43.  So few_rows is the better one
// up to 32 heads; beyond 48 it reads too often.)
int32_t few_row_tiles(const AttendParams& p) { return p.c.q_offset ? 1 : (p.group + kFewRows - 1) / kFewRows; }
int64_t few_blocks(const AttendParams& p) { return p.c.n_seqs * p.c.n_kv_heads * few_row_tiles(p); }
int32_t few_slot_rows(const AttendParams& p) { return p.c.q_offset ? kFewRows : p.group; }
int64_t few_slots(const AttendParams& p) { return p.c.n_seqs * p.c.n_kv_heads * few_slot_rows(p); }
int64_t tile_slots(const AttendParams& p) { return p.c.n_tokens * p.n_heads; }

// Which rows a call can have, from what the host knows.
bool needs_few(const AttendParams& p) { return p.group <= kFewRows || !p.c.q_offset; }
bool needs_tiles(const AttendParams& p) { return p.c.q_offset && p.c.n_tokens * p.group > kFewRows; }

// How far the tokens of a sequence are split: as long as there are fewer
// workgroups than `fill`, into parts of at least `least` tokens; and into parts of at
// most `most`.
struct SplitRule {
    int64_t fill, least, most;
};
// few_rows: three workgroups a CU (4 sequences of 20011 to 36864 tokens, 8
// heads: 96 us; with 512 workgroups 116, with 384 131); a step of each wavefront; and
// parts short enough that a long sequence does not end alone (96 of 16 to 36864
// tokens: 1.19 ms, unsplit 1.46).
constexpr SplitRule kSplitFew = {768, kFewWaves * kFewTile, 8192};
// few_rows beside tile_rows: a workgroup of up to 8 wavefronts a CU.
constexpr SplitRule kSplitMixed = {512, 8 * kFewTile, 8192};
// tile_rows: a workgroup a CU; of half the CUs in a batch of more sequences
// than row tiles, whose other sequences have few rows and read meanwhile (two
// chunks of 512 tokens with 62 single tokens: 712 us so, 869 us on all CUs; the only
// batch that was timed both ways).
constexpr SplitRule kSplitTiles = {256, 256, INT64_MAX}, kSplitHalf = {128, 256, INT64_MAX};
constexpr int64_t kMostParts = 256;
// Parts of `most` tokens, which even out a batch that has a long sequence, as
// long as their sums take no more than this: the host knows the table's width and not
// the lengths.  4096 sequences of 16 to 1000 tokens, 32 heads on 8, in a table for a
// million take 5.6 ms so, with all 128 parts 20 ms and 34 GB, with 256 MiB 2.1 ms; with one
// of 500000 tokens among them (and offsets) 4.9, 23 and 11.7.
constexpr int64_t kEvenBytes = 1ll << 30;
constexpr int64_t kApartBytes = 192 << 20;

// Tokens that a sequence's rows see at most, from what the host knows.
int64_t most_tokens(const AttendParams& p) {
    int64_t tokens = (int64_t)p.c.table_width * p.c.page_tokens;
    if (p.max_length > 0) tokens = std::min<int64_t>(tokens, p.max_length);
    if (p.window > 0) tokens = std::min<int64_t>(tokens, (int64_t)p.window + p.sinks);
    return tokens;
}

// Whether few_rows takes each sequence in one part with eight wavefronts: up
// to three of their steps, on up to a workgroup a CU.  8 heads of 500 tokens:
// 10.1 us so, 13.3 in four parts and a join; of 700 12.1 and 13.2, of 1000 16.8 and
// 13.2; 256 of 500 15.4 and 19.8.  Heads of more than 128 elements leave no
// registers for two steps a SIMD (8 of 400 tokens 21.4 and 14.0).
bool wide_few(const AttendParams& p) {
    const int64_t tokens = most_tokens(p);
    return !needs_tiles(p) && p.c.head_dim <= 128 && few_blocks(p) <= 256 && tokens > 2 * kFewWaves * kFewTile &&
           tokens <= 6 * kFewWaves * kFewTile;
}

// Whether the sequences with few rows get a launch of their own before the
// others': where most can be such (as when every sequence has one token and the
// caller gives offsets all the same) and there is much to read.  In one launch
// tile_rows' LDS leaves them two wavefronts a SIMD: 32 sequences of 2000 tokens, 8
// heads (262 MB) take 55 us so and 61 in one launch, 64 of 500 (131 MB) 28.6 and 27.8.
bool apart(const AttendParams& p) {
    return needs_few(p) && needs_tiles(p) && p.c.n_tokens * p.group <= kFewRows * p.c.n_seqs &&
           most_tokens(p) * p.c.n_seqs * p.c.n_kv_heads * p.c.head_dim * 4 >= kApartBytes;
}

int64_t wanted_parts(const AttendParams& p, const SplitRule& rule, int64_t blocks, int64_t slots) {
    const int64_t tokens = most_tokens(p);
    // A join costs 4 to 5 us with its launch.  It does not pay for two parts'
    // tokens (8 heads of 250: 10.0 us in one, 14.1 in two), nor for short sequences
    // that nearly fill the chip (512 workgroups of 600: 29.9 and 34.8 us; of 16
    // to 1280, 48.9 and 46.3).
    int64_t fill = std::min((rule.fill + blocks - 1) / blocks, (tokens + rule.least - 1) / rule.least);
    if (tokens <= 2 * rule.least || (3 * blocks >= 2 * rule.fill && tokens < 8 * rule.least)) fill = 1;
    // Each further part makes the join longer by as much as it takes off the
    // parts when there are sqrt(0.4 tokens): 1 head of 20000 tokens in 64, 128 and
    // 157 parts 15.4, 16.3 and 17.2 us; 2 of 36864 in 64, 128 and 256 22.9, 20.6 and 24.9;
    // 1 of 131072 53.0, 36.3 and 32.8.
    while (fill > 1 && 5 * fill * fill > 2 * tokens) --fill;
    const int64_t even = std::min(tokens / rule.most + (tokens % rule.most != 0),
                                  kEvenBytes / (slots * p.c.head_dim * (int64_t)sizeof(float)));
    const int64_t n = std::max(fill, even);
    return std::max<int64_t>(1, std::min(n, kMostParts));
}
const SplitRule& few_rule(const AttendParams& p) {
    return needs_tiles(p) && !apart(p) ? kSplitMixed : kSplitFew;
}
// (a lone sequence with many rows leaves none to few_rows)
int64_t few_parts(const AttendParams& p) {
    if (!needs_few(p) || wide_few(p) || (needs_tiles(p) && p.c.n_seqs == 1)) return 1;
    return wanted_parts(p, few_rule(p), few_blocks(p), few_slots(p));
}
// How row tiles are numbered.  A sequence of r rows has ceil(r / ROWS), which
// is at most floor(r / ROWS) + 1, and none if r <= kFewRows, so at most
// floor(r / (kFewRows + 1)).  A number without a tile is a workgroup that finds out
// and ends, but holds a CU's LDS for it: 256 sequences with one new token each,
// 20 heads: 1.18 ms with 257 numbers a head, 0.99 with 15.
struct TileNumbers {
    int64_t count;
    int32_t per;
    bool each;
};
TileNumbers number_tiles(const AttendParams& p) {
    const int64_t rows = p.c.n_tokens * p.group;
    const int32_t tile = tile_rows_of(p.c.head_dim), few = kFewRows + 1;
    if (rows / few < rows / tile + p.c.n_seqs) return {rows / few, few, false};
    return {rows / tile + p.c.n_seqs, tile, true};
}

// The lengths are those that the host knows of: the table's width where the
// caller gives no bound, and a short prompt in a wide table is split for tokens that it
// has not (of 64, 500 and 1000 tokens, 32 heads on 8: 15, 25 and 38 us in a table of
// their own size or with the bound, 24, 31 and 43 in one for 36864).
// (Workgroups without those that a ragged batch adds: too many parts cost
// less than too few.)  Rows are many here, and so are the parts' sums, which are
// written and read in 32 bits: as many parts as make their time, 26 ns a token,
// and that of the join least.  A prompt of 1000 tokens, 32 heads on 8: 37 us in
// one part, 55 in three; 8 of up to 1916, 4 heads on one: 63 us in one, 75 in
// three; 512 new tokens behind 16384: 155 us in four, 439 in one; 64: 41 us in 32, 423
// in one.  (All of heads of 128; others were not timed apart.)
int64_t tile_parts(const AttendParams& p) {
    if (!needs_tiles(p)) return 1;
    const int64_t tiles = std::max<int64_t>(1, p.c.n_tokens * p.group / tile_rows_of(p.c.head_dim));
    const int64_t most = wanted_parts(p, p.c.n_seqs > tiles && !apart(p) ? kSplitHalf : kSplitTiles,
                                      tiles * p.c.n_kv_heads, tile_slots(p));
    const int64_t sums = tile_slots(p) * p.c.head_dim * 2 * (int64_t)sizeof(float);     // bytes, of a part
    // (ns: a round of a workgroup a CU takes 8 us to begin and end; the sums at
    // 4.5 TB/s; a number without a tile holds a CU for 1.5 us)
    const int64_t wgs = tiles * p.c.n_kv_heads, empty = std::max<int64_t>(number_tiles(p).count * p.c.n_kv_heads - wgs, 0);
    auto cost = [&](int64_t parts) {
        return (wgs * parts + 255) / 256 * (8000 + most_tokens(p) * 26 / parts) + empty * parts * 6 +
               (parts > 1 ? 5000 + sums * parts / 4500 : 0);
    };
    int64_t best = 1;
    for (int64_t n = 2; n <= most; ++n)
        if (cost(n) < cost(best)) best = n;
    return best;
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
Parts take_parts(AttendParams* p, int64_t least, int64_t slots, int64_t want) {
    while (want > 1 && (uint64_t)parts_bytes(*p, slots, want) > p->workspace_bytes) --want;
    Parts r = {(int32_t)want, (int32_t)least, nullptr, nullptr};
    if (want > 1) {
        unsigned char* const at = (unsigned char*)p->workspace;
        r.sums = (float*)at;
        r.stats = (float*)(at + sums_bytes(*p, slots, want));
        p->workspace = at + parts_bytes(*p, slots, want);
        p->workspace_bytes -= (uint64_t)parts_bytes(*p, slots, want);
    }
    return r;
}

template <bool F16, int DP>
hipError_t launch_dim(const AttendLaunch& f, hipStream_t stream) {
    const AttendParams& p = f.a;
    const int64_t blocks = needs_few(p) ? few_blocks(p) : 0;
    hipError_t e = hipSuccess;
    const bool alone = apart(p) || !needs_tiles(p);
    if (alone) e = launch_few<F16, DP>(f, blocks, stream);
    if (e == hipSuccess && needs_tiles(p)) e = launch_mixed(f, alone ? 0 : blocks, stream);
    const int64_t few = f.few.count > 1 ? few_slots(p) : 0, tiles = f.tiles.count > 1 ? tile_slots(p) : 0;
    if (e == hipSuccess && few + tiles > 0) e = launch_join<F16, DP>(f, few, tiles, stream);
    return e;
}

template <bool F16>
hipError_t launch_type(const AttendLaunch& f, hipStream_t stream) {
    if (f.a.c.head_dim <= 64) return launch_dim<F16, 64>(f, stream);
    if (f.a.c.head_dim <= 128) return launch_dim<F16, 128>(f, stream);
    return launch_dim<F16, 256>(f, stream);
}

}  // namespace

uint64_t attend_workspace_bytes(const AttendParams& p) {
    if (p.c.n_tokens == 0 || p.c.n_seqs == 0) return 0;
    return (uint64_t)(parts_bytes(p, few_slots(p), few_parts(p)) + parts_bytes(p, tile_slots(p), tile_parts(p)));
}

hipError_t launch_attend(const AttendParams& p, hipStream_t stream) {
    // (sequences without rows count here, which no check before has bounded)
    if (needs_few(p) && few_blocks(p) > INT32_MAX) return hipErrorInvalidConfiguration;
    AttendLaunch f{};
    f.a = p;
    f.score_scale = p.scale * kLog2e;
    f.row_tiles = few_row_tiles(p);
    f.slot_rows = few_slot_rows(p);
    f.wide = wide_few(p);
    f.few = take_parts(&f.a, few_rule(p).least, few_slots(p), few_parts(p));
    f.tiles = take_parts(&f.a, kSplitTiles.least, tile_slots(p), tile_parts(p));
    const TileNumbers t = number_tiles(p);
    f.tile_count = t.count;
    f.tile_per = t.per;
    f.tile_each = t.each;
    return p.f16 ? launch_type<true>(f, stream) : launch_type<false>(f, stream);
}

}  // namespace tl
