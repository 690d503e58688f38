// The paged cache's pool: rows written to their pages, and pages given out,
// shared, freed, moved together and copied.
//
// All of it is memory traffic and latency: no call computes more than
// prefix sums of counts.  Free pages are listed by ballots in ascending order, so
// that the tables do not depend on timing; atomics add to page counts, take the least
// of the forks that claim a child and exchange a freed slot's length for 0, all of
// which come out the same in any order.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "cache.h"
#include "cache_rows.h"
#include "device_util.h"
#include "tl_internal.h"

namespace tl {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kAppendThreads = 256;
constexpr int kAppendTokens = 16;       // most tokens of a workgroup

// One workgroup moves `tokens` consecutive rows, 16 bytes per lane.  Bound by
// memory: 65415 tokens of 8 heads of 128 (536 MB) take 111 us, 4.8 TB/s; 64
// tokens 3 us, a launch and four round trips.
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendParams P, int tokens, int64_t block) {
    const CacheView& c = P.c;
    __shared__ int64_t dst[kAppendTokens];
    const int64_t first = (blockIdx.x + block) * tokens;
    if (P.appended && first == 0 && threadIdx.x == 0) *P.appended = 1;
    if ((int)threadIdx.x < tokens) {
        const int64_t i = first + threadIdx.x;
        int64_t at = -1, b;
        if (i < c.n_tokens && find_seq(c, i, &b)) {
            const SeqRows s = seq_rows(c, b);
            const int64_t pos = (int64_t)s.length - s.n + (i - s.first);
            if (i >= s.first && i - s.first < s.n && pos >= 0 && pos < table_tokens(c))
                at = token_offset(c, c.table + b * c.table_width, (int32_t)pos);
        }
        dst[threadIdx.x] = at;
    }
    __syncthreads();
    const int per_head = c.head_dim / 8;
    const int per_row = c.n_kv_heads * per_head;
    for (int x = threadIdx.x; x < tokens * per_row; x += kAppendThreads) {
        const int r = x / per_row, y = x - r * per_row;
        const int h = y / per_head, d = (y - h * per_head) * 8;
        const int64_t at = dst[r];
        if (at < 0) continue;
        const int64_t to = at + (int64_t)h * c.head_stride + d;
        const u32x4 k = *(const u32x4*)(P.src[0] + (first + r) * P.token_stride[0] + h * P.head_stride[0] + d);
        const u32x4 v = *(const u32x4*)(P.src[1] + (first + r) * P.token_stride[1] + h * P.head_stride[1] + d);
        *(u32x4*)(c.key + to) = k;
        *(u32x4*)(c.value + to) = v;
    }
}

constexpr int kPoolThreads = 1024;
constexpr int kPoolWaves = kPoolThreads / kWave;
constexpr int kBallots = 16;            // of 64 pages, per wavefront and step

// Words of `work`: for the slots, what the calls note (three arrays), then for
// the pages one array and a half and the counts of blocks of 4096.
__host__ __device__ inline int64_t work_list(const PagesParams& p) { return 3 * p.n_slots; }

// What one workgroup decides about few slots stays in LDS, and with many in
// the work array: 4096 slots 22 us so, 34 there.
constexpr int kLdsSlots = 4096, kLdsList = 4096;
struct PoolLds {
    int32_t starts[kLdsSlots];
    int32_t notes[kLdsSlots];
    int32_t list[kLdsList];
};

// The counts of kPoolThreads x kBallots consecutive pages, kBallots a lane:
// a wavefront's ballots cover 1024 of them.
struct PageCounts {
    int32_t r[kBallots];
    // `none` for pages past the last one
    __device__ __forceinline__ void load(const PagesParams& P, int64_t base, int32_t none = 1) {
        const int64_t w0 = base + (int64_t)(threadIdx.x / kWave) * kBallots * kWave + lane_id();
#pragma unroll
        for (int i = 0; i < kBallots; ++i) {
            const int64_t p = w0 + i * kWave;
            r[i] = p < P.n_pages ? P.ref[p] : none;
        }
    }
};

// The first `want` free pages in ascending order, to list[]; returns how many
// free pages were seen (at least min(want, all)).  One workgroup of
// kPoolThreads; `c` holds the counts of the first pages (their loads are under way
// while the caller finds out what it wants).
__device__ int64_t list_free(const PagesParams& P, PageCounts& c, int64_t want, int32_t* list) {
    __shared__ int32_t counts[2][kPoolWaves];
    constexpr int64_t kStep = (int64_t)kPoolThreads * kBallots;
    const int wave = threadIdx.x / kWave, lane = lane_id();
    int64_t found = 0;
    int parity = 0;
    for (int64_t base = 0; base < P.n_pages && found < want; base += kStep, parity ^= 1) {
        const int64_t w0 = base + (int64_t)wave * kBallots * kWave;
        uint64_t bits[kBallots];
        int32_t n = 0;
#pragma unroll
        for (int i = 0; i < kBallots; ++i) {
            bits[i] = __ballot(c.r[i] == 0);
            n += __popcll(bits[i]);
        }
        if (base + kStep < P.n_pages) c.load(P, base + kStep);
        if (lane == 0) counts[parity][wave] = n;
        __syncthreads();
        int32_t before = 0, all = 0;
        for (int w = 0; w < kPoolWaves; ++w) {
            before += w < wave ? counts[parity][w] : 0;
            all += counts[parity][w];
        }
        int64_t rank = found + before;
#pragma unroll
        for (int i = 0; i < kBallots; ++i) {
            const int64_t at = rank + __popcll(bits[i] & ((1ull << lane) - 1));
            if ((bits[i] >> lane & 1) && at < want) list[at] = (int32_t)(w0 + i * kWave + lane);
            rank += __popcll(bits[i]);
        }
        found += all;
    }
    __syncthreads();
    return found;
}

// Sum of x over the lanes before this one and over earlier calls (`carry`,
// uniform); one workgroup of kPoolThreads.
__device__ int64_t running_sum(int64_t x, int64_t* carry) {
    __shared__ uint64_t sums[kPoolWaves];
    const int wave = threadIdx.x / kWave;
    const uint64_t incl = wave_incl_scan_u64((uint64_t)x);
    __syncthreads();                    // sums of the call before are read
    if (lane_id() == kWave - 1) sums[wave] = incl;
    __syncthreads();
    uint64_t before = 0, all = 0;
    for (int w = 0; w < kPoolWaves; ++w) {
        before += w < wave ? sums[w] : 0;
        all += sums[w];
    }
    const int64_t r = *carry + (int64_t)(before + incl) - x;
    *carry += (int64_t)all;
    return r;
}

__device__ __forceinline__ int32_t saturate(int64_t x) { return (int32_t)min(x, (int64_t)INT32_MAX); }

// Full pages of `tokens` (0 .. 2^31 - 1), and pages with the last one.
__device__ __forceinline__ int32_t full_pages(const PagesParams& P, int32_t tokens) {
    return (int32_t)div_u32((uint32_t)tokens, P.div_page);
}
__device__ __forceinline__ bool partly(const PagesParams& P, int32_t tokens) {
    return (int64_t)full_pages(P, tokens) * P.page_tokens != tokens;
}
__device__ __forceinline__ int32_t pages_of(const PagesParams& P, int32_t tokens) {
    return full_pages(P, tokens) + partly(P, tokens);
}

// What a slot asks for: its pages now and the further ones, and the status
// that does not depend on the pool.
struct Wish {
    int32_t new_len, have, need, status;
};

__device__ __forceinline__ Wish wish(const PagesParams& P, int32_t length, int32_t add) {
    Wish w = {0, 0, 0, TL_PAGES_OK};
    const int64_t new_len = (int64_t)length + add, room = (int64_t)P.table_width * P.page_tokens;
    if (length < 0 || add < 0) w.status = TL_PAGES_BAD;
    else if (new_len > room || new_len > INT32_MAX) w.status = TL_PAGES_TABLE_FULL;
    else {
        w.new_len = (int32_t)new_len;
        w.have = pages_of(P, length);
        w.need = pages_of(P, w.new_len) - w.have;
    }
    return w;
}

// One workgroup: (1) where each slot's pages begin among the free ones, (2)
// the free pages, (3) page k to the slot that it falls to (found in the starts,
// which are sorted), (4) lengths and statuses.  A chain of memory round
// trips, not work: 80 slots of a pool of 131072 pages take 7.8 us.
__global__ __launch_bounds__(kPoolThreads) void extend_kernel(PagesParams P, const int32_t* add, int32_t* status,
                                                              int32_t* work) {
    __shared__ PoolLds lds;
    const bool small = P.n_slots <= kLdsSlots;
    int32_t* const starts = small ? lds.starts : work;
    int32_t* const have = small ? lds.notes : work + P.n_slots;
    PageCounts counts;
    counts.load(P, 0);
    int64_t total = 0;
    Wish mine = {};                     // of slot threadIdx.x
    // tokens granted before stand beside these until an append has placed them
    const bool keep = P.granted && P.granted[P.n_slots] == 0;
    for (int64_t b0 = 0; b0 < P.n_slots; b0 += kPoolThreads) {
        const int64_t b = b0 + threadIdx.x;
        Wish w = {};
        if (b < P.n_slots) w = wish(P, P.length[b], add[b]);
        const int64_t at = running_sum(w.need, &total);
        if (b < P.n_slots) {
            starts[b] = saturate(at);
            have[b] = w.have;
        }
        if (b0 == 0) mine = w;
    }
    const int64_t want = min(total, P.n_pages);
    int32_t* const list = want <= kLdsList ? lds.list : work + work_list(P);
    __syncthreads();
    const int64_t found = min(list_free(P, counts, want, list), P.n_pages);
    for (int64_t k = threadIdx.x; k < min(want, found); k += kPoolThreads) {
        int64_t lo = 0, hi = P.n_slots;     // starts[lo] <= k < starts[hi]
        while (hi - lo > 1) {
            const int64_t mid = (lo + hi) >> 1;
            if (starts[mid] <= k) lo = mid;
            else hi = mid;
        }
        if ((lo + 1 < P.n_slots ? (int64_t)starts[lo + 1] : total) > found) continue;
        const int32_t page = list[k];
        P.table[lo * P.table_width + have[lo] + (k - starts[lo])] = page;
        P.ref[page] = 1;
    }
    for (int64_t b = threadIdx.x; b < P.n_slots; b += kPoolThreads) {
        const Wish w = b < kPoolThreads ? mine : wish(P, P.length[b], add[b]);
        const bool fits = w.need == 0 || starts[b] + (int64_t)w.need <= found;
        status[b] = w.status != TL_PAGES_OK ? w.status : fits ? TL_PAGES_OK : TL_PAGES_NONE_FREE;
        if (P.granted) {
            const int32_t entry = keep ? P.granted[b] : 0, had = tokens_granted(entry);
            const bool served = w.status == TL_PAGES_OK && fits;
            P.granted[b] = !served ? ~had : add[b] > 0 ? saturate((int64_t)had + add[b]) : entry;
        }
        if (w.status == TL_PAGES_OK && fits) P.length[b] = w.new_len;
    }
    if (P.granted && threadIdx.x == 0) P.granted[P.n_slots] = 0;    // (read before the barriers above)
}

// One workgroup decides the forks: validity (of several with one child the
// first counts), which need a page, and which page that is.  work[n_slots + f]:
// the child's length, -1 where the fork is not served.  Latency: 64 forks
// 7.3 us, their rows in a launch of their own 2.8 (17.8 in this one).
__global__ __launch_bounds__(kPoolThreads) void fork_kernel(PagesParams P, int64_t n_forks, const int32_t* parent,
                                                            const int32_t* child, int32_t* copy_src,
                                                            int32_t* copy_dst, int32_t* status, int32_t* work) {
    __shared__ PoolLds lds;
    const bool small = P.n_slots <= kLdsSlots;
    int32_t* const claim = small ? lds.notes : work;
    int32_t* const lens = work + P.n_slots;
    int32_t* const starts = small ? lds.starts : work + 2 * P.n_slots;
    const int64_t room = (int64_t)P.table_width * P.page_tokens;
    auto in_range = [&](int32_t s) { return s >= 0 && s < P.n_slots; };
    PageCounts counts;
    counts.load(P, 0);
    // fork threadIdx.x's slots and length stay in registers
    const bool any = threadIdx.x < n_forks;
    const int32_t my_parent = any ? parent[threadIdx.x] : -1, my_child = any ? child[threadIdx.x] : -1;
    const int32_t parent_len = in_range(my_parent) ? P.length[my_parent] : -1;
    const int32_t child_len = in_range(my_child) ? P.length[my_child] : -1;
    int32_t my_len = -1;
    auto child_of = [&](int64_t f) { return f < kPoolThreads ? my_child : child[f]; };
    for (int64_t f = threadIdx.x; f < n_forks; f += kPoolThreads)
        if (in_range(child_of(f))) claim[child_of(f)] = INT32_MAX;
    if (!small) __threadfence();
    __syncthreads();
    for (int64_t f = threadIdx.x; f < n_forks; f += kPoolThreads)
        if (in_range(child_of(f))) atomicMin(&claim[child_of(f)], (int32_t)f);
    if (!small) __threadfence();
    __syncthreads();
    int64_t total = 0;
    for (int64_t f0 = 0; f0 < n_forks; f0 += kPoolThreads) {
        const int64_t f = f0 + threadIdx.x;
        int32_t len = -1;
        if (f < n_forks && in_range(child_of(f))) {
            const int32_t first = __hip_atomic_load(&claim[child_of(f)], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const int32_t from = f0 == 0 ? my_parent : parent[f];
            len = f0 == 0 ? parent_len : in_range(from) ? P.length[from] : -1;
            if (first != f || (f0 == 0 ? child_len : P.length[child[f]]) != 0 || len > room) len = -1;
        }
        len = max(len, -1);
        const int64_t at = running_sum(len > 0 && partly(P, len), &total);
        if (f < n_forks) {
            lens[f] = len;
            starts[f] = saturate(at);
        }
        if (f0 == 0) my_len = len;
    }
    const int64_t want = min(total, P.n_pages);
    int32_t* const list = want <= kLdsList ? lds.list : work + work_list(P);
    // (the page to copy is looked up while the free ones are listed)
    auto last_page = [&](int32_t from, int32_t len) {
        return len > 0 && partly(P, len) ? P.table[(int64_t)from * P.table_width + full_pages(P, len)] : -1;
    };
    const int32_t my_src = last_page(my_parent, my_len);
    const int64_t found = list_free(P, counts, want, list);
    for (int64_t f = threadIdx.x; f < n_forks; f += kPoolThreads) {
        const int32_t len = f < kPoolThreads ? my_len : lens[f];
        int32_t src = -1, dst = -1, st = len < 0 ? TL_PAGES_BAD : TL_PAGES_OK;
        if (len > 0 && partly(P, len)) {
            if (starts[f] < min(found, want)) {
                src = f < kPoolThreads ? my_src : last_page(parent[f], len);
                dst = list[starts[f]];
                P.ref[dst] = 1;
            } else {
                st = TL_PAGES_NONE_FREE;
                lens[f] = -1;
            }
        }
        copy_src[f] = src;
        copy_dst[f] = dst;
        status[f] = st;
    }
}

// A workgroup per fork: the child's row, the shared pages' counts, its length.
__global__ __launch_bounds__(256) void fork_rows_kernel(PagesParams P, const int32_t* parent, const int32_t* child,
                                                        const int32_t* copy_dst, const int32_t* work, int64_t first) {
    const int64_t f = blockIdx.x + first;
    const int32_t len = work[P.n_slots + f];
    if (len < 0) return;
    const int32_t full = full_pages(P, len);
    const int32_t* const from = P.table + (int64_t)parent[f] * P.table_width;
    int32_t* const to = P.table + (int64_t)child[f] * P.table_width;
    for (int32_t i = threadIdx.x; i < full; i += 256) {
        const int32_t page = from[i];
        to[i] = page;
        if (page >= 0 && page < P.n_pages) atomicAdd(&P.ref[page], 1);
    }
    if (threadIdx.x == 0) {
        if (partly(P, len)) to[full] = copy_dst[f];
        P.length[child[f]] = len;
        if (P.granted) P.granted[child[f]] = 0;
    }
}

// A workgroup per slot.  Whoever takes the length away frees the pages, so
// that a slot named twice leaves once.
__global__ __launch_bounds__(256) void free_kernel(PagesParams P, const int32_t* slots, int64_t first) {
    __shared__ int32_t taken;
    const int32_t slot = slots[blockIdx.x + first];
    if (slot < 0 || slot >= P.n_slots) return;
    if (threadIdx.x == 0) taken = atomicExch(&P.length[slot], 0);
    __syncthreads();
    const int64_t have = min(pages_of(P, max(taken, 0)), P.table_width);
    const int32_t* const row = P.table + (int64_t)slot * P.table_width;
    for (int64_t i = threadIdx.x; i < have; i += 256) {
        const int32_t page = row[i];
        if (page >= 0 && page < P.n_pages) atomicSub(&P.ref[page], 1);
    }
}

// ---- compaction: pages in blocks of kBlockPages, 256 threads each
constexpr int kBlockPages = 4096;
constexpr int kBlockWaves = 4;
static_assert(kBlockPages == kBlockWaves * kBallots * kWave);
__host__ __device__ inline int64_t page_blocks(const PagesParams& p) { return (p.n_pages + kBlockPages - 1) / kBlockPages; }

// Of the work array's pages: what becomes of page p (kept: kStays; a page
// that moves, or a free one that takes it: the move's number; else kUnused),
// then the moved pages' counts, then the live pages of each block.
constexpr int32_t kStays = -1, kUnused = -2;
struct CompactWork {
    int32_t* fate;
    int32_t* moved_ref;
    int32_t* counts;
    int32_t* n_live;
};
__host__ __device__ inline CompactWork compact_work(const PagesParams& p, int32_t* work) {
    CompactWork w;
    w.fate = work + work_list(p);
    w.moved_ref = w.fate + p.n_pages;
    w.counts = w.moved_ref + p.n_pages / 2;
    w.n_live = w.counts + page_blocks(p);
    return w;
}

// Sum over the workgroup's threads.
template <int WAVES>
__device__ int64_t block_sum(int64_t x) {
    __shared__ uint64_t sums[WAVES];
    const uint64_t s = wave_sum_u64((uint64_t)x);
    __syncthreads();
    if (lane_id() == 0) sums[threadIdx.x / kWave] = s;
    __syncthreads();
    uint64_t all = 0;
    for (int w = 0; w < WAVES; ++w) all += sums[w];
    return (int64_t)all;
}

__global__ __launch_bounds__(256) void count_live_kernel(PagesParams P, int32_t* counts) {
    PageCounts c;
    c.load(P, (int64_t)blockIdx.x * kBlockPages, 0);
    int64_t n = 0;
#pragma unroll
    for (int i = 0; i < kBallots; ++i) n += c.r[i] > 0;
    n = block_sum<kBlockWaves>(n);
    if (threadIdx.x == 0) counts[blockIdx.x] = (int32_t)n;
}

// With L live pages, `low` of them below L: a free page p < L has p - (live
// pages before p) free ones before it, a live page p >= L has (live pages
// before p) - low moving ones before it.  Equal numbers meet.  WAVES > kBlockWaves:
// one workgroup holds all pages and needs no counts of blocks.
template <int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void plan_moves_kernel(PagesParams P, CompactWork W, int32_t* copy_src,
                                                                   int32_t* copy_dst, int32_t* n_copies) {
    const int64_t mine = blockIdx.x;
    PageCounts c;
    c.load(P, mine * kBlockPages, 0);
    const int64_t lane_page = (int64_t)(threadIdx.x / kWave) * kBallots * kWave + lane_id();
    int64_t n_live, mine_before = 0, low = 0;
    if constexpr (WAVES > kBlockWaves) {
        int64_t n = 0;
#pragma unroll
        for (int i = 0; i < kBallots; ++i) n += c.r[i] > 0;
        n_live = block_sum<WAVES>(n);
#pragma unroll
        for (int i = 0; i < kBallots; ++i) low += c.r[i] > 0 && lane_page + i * kWave < n_live;
    } else {
        const int64_t blocks = page_blocks(P);
        int64_t n = 0;
        for (int64_t k = threadIdx.x; k < blocks; k += 256) {
            n += W.counts[k];
            mine_before += k < mine ? W.counts[k] : 0;
        }
        n_live = block_sum<WAVES>(n);
        mine_before = block_sum<WAVES>(mine_before);
        const int64_t edge = n_live / kBlockPages;
        for (int64_t k = threadIdx.x; k < edge; k += 256) low += W.counts[k];
        PageCounts e;
        e.load(P, edge * kBlockPages, 0);
#pragma unroll
        for (int i = 0; i < kBallots; ++i) low += e.r[i] > 0 && edge * kBlockPages + lane_page + i * kWave < n_live;
    }
    low = block_sum<WAVES>(low);
    if (mine == 0 && threadIdx.x == 0) {
        *n_copies = (int32_t)(n_live - low);
        *W.n_live = (int32_t)n_live;
    }
    // the ranks of this block's pages
    __shared__ int32_t counts[WAVES];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int64_t w0 = mine * kBlockPages + (int64_t)wave * kBallots * kWave;
    uint64_t bits[kBallots];
    int32_t own = 0;
#pragma unroll
    for (int i = 0; i < kBallots; ++i) {
        bits[i] = __ballot(c.r[i] > 0);
        own += __popcll(bits[i]);
    }
    if (lane == 0) counts[wave] = own;
    __syncthreads();
    int64_t before = mine_before;
    for (int w = 0; w < wave; ++w) before += counts[w];
#pragma unroll
    for (int i = 0; i < kBallots; ++i) {
        const int64_t p = w0 + i * kWave + lane;
        const bool is_live = bits[i] >> lane & 1;
        const int64_t at = before + __popcll(bits[i] & ((1ull << lane) - 1));
        before += __popcll(bits[i]);
        if (p >= P.n_pages) continue;
        int32_t fate = is_live ? kStays : kUnused;
        if (is_live && p >= n_live) {
            fate = (int32_t)(at - low);
            copy_src[fate] = (int32_t)p;
            W.moved_ref[fate] = c.r[i];
        } else if (!is_live && p < n_live) {
            fate = (int32_t)(p - at);
            copy_dst[fate] = (int32_t)p;
        }
        W.fate[p] = fate;
    }
}

// The state after the moves.  Counts and table entries are each read and
// written by one thread, so the new state may lie where the old one does.
__global__ __launch_bounds__(256) void remap_kernel(PagesParams P, CompactWork W, const int32_t* copy_dst,
                                                    int32_t* ref_out, int32_t* table_out) {
    const int64_t step = (int64_t)gridDim.x * 256;
    const int64_t me = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t n_live = *W.n_live;
    for (int64_t p = me; p < P.n_pages; p += step) {
        const int32_t fate = W.fate[p];
        ref_out[p] = p >= n_live ? 0 : fate == kStays ? P.ref[p] : W.moved_ref[fate];
    }
    for (int64_t e = me; e < P.n_slots * P.table_width; e += step) {
        const int64_t b = e / P.table_width, i = e - b * P.table_width;
        const int32_t page = P.table[e];
        int32_t to = page;
        if (i * P.page_tokens < P.length[b] && page >= 0 && page < P.n_pages) {
            const int32_t fate = W.fate[page];
            to = page < n_live ? (fate == kStays ? page : -1) : fate >= 0 ? copy_dst[fate] : -1;
        }
        table_out[e] = to;
    }
}

constexpr int kCopyThreads = 256;

// A workgroup copies whole pages, 64 bytes per lane and step: four loads are
// under way before the first store waits.  Past the caches, which would only lose
// what others read: 13286 pages of 8 KB in 8 planes (1.7 GB) 0.31 ms, 5.3 TB/s
// (0.33 ms through them).
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(CopyParams P) {
    int64_t pairs = P.n_pairs;
    if (P.n_live) pairs = min(pairs, (int64_t)max(*P.n_live, 0));
    const int64_t items = pairs * P.n_planes;
    const int64_t n = P.page_bytes / 16;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int64_t pair = it / P.n_planes, plane = it - pair * P.n_planes;
        const int32_t s = P.src[pair], d = P.dst[pair];
        if (s < 0 || s >= P.n_pages || d < 0 || d >= P.n_pages || s == d) continue;
        unsigned char* const base = P.pages + plane * P.plane_stride;
        const u32x4* const from = (const u32x4*)(base + s * P.page_stride);
        u32x4* const to = (u32x4*)(base + d * P.page_stride);
        for (int64_t i = threadIdx.x; i < n; i += 4 * kCopyThreads) {
            u32x4 x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (i + q * kCopyThreads < n) x[q] = __builtin_nontemporal_load(&from[i + q * kCopyThreads]);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (i + q * kCopyThreads < n) __builtin_nontemporal_store(x[q], &to[i + q * kCopyThreads]);
        }
    }
}

}  // namespace

hipError_t launch_append(const AppendParams& p, hipStream_t stream) {
    // few tokens: one a workgroup, so that they are spread over the chip (4095
    // 8.0 us so, 8.5 with 16); many: 16, which saves workgroups (65415 112 us, 152)
    const int tokens = p.c.n_tokens < 4096 ? 1 : kAppendTokens;
    const int64_t blocks = (p.c.n_tokens + tokens - 1) / tokens;
    return launch_all(blocks, kAppendThreads, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL(append_kernel, grid, dim3(kAppendThreads), 0, stream, p, tokens, first);
    });
}

uint64_t pages_work_words(const PagesParams& p) {
    return (uint64_t)(work_list(p) + p.n_pages + p.n_pages / 2 + page_blocks(p) + 1);
}

hipError_t launch_pages_extend(const PagesParams& p, const int32_t* add, int32_t* status, int32_t* work,
                               hipStream_t stream) {
    hipLaunchKernelGGL(extend_kernel, dim3(1), dim3(kPoolThreads), 0, stream, p, add, status, work);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesParams& p, int64_t n_forks, const int32_t* parent, const int32_t* child,
                             int32_t* copy_src, int32_t* copy_dst, int32_t* status, int32_t* work,
                             hipStream_t stream) {
    hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(kPoolThreads), 0, stream, p, n_forks, parent, child, copy_src,
                       copy_dst, status, work);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return launch_all(n_forks, 256, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL(fork_rows_kernel, grid, dim3(256), 0, stream, p, parent, child, copy_dst, work, first);
    });
}

hipError_t launch_pages_free(const PagesParams& p, int64_t n_free, const int32_t* slots, hipStream_t stream) {
    return launch_all(n_free, 256, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL(free_kernel, grid, dim3(256), 0, stream, p, slots, first);
    });
}

hipError_t launch_pages_compact(const PagesParams& p, int32_t* ref_out, int32_t* table_out, int32_t* copy_src,
                                int32_t* copy_dst, int32_t* n_copies, int32_t* work, hipStream_t stream) {
    const CompactWork w = compact_work(p, work);
    hipError_t e;
    // pools that one workgroup holds: a launch less (up to 8000 pages with their
    // copies 22.4 us so, 25.5 with counts of blocks; 16000 30.0 and 33.0)
    if (p.n_pages <= (int64_t)kPoolThreads * kBallots) {
        hipLaunchKernelGGL((plan_moves_kernel<kPoolWaves>), dim3(1), dim3(kPoolThreads), 0, stream, p, w, copy_src,
                           copy_dst, n_copies);
    } else {
        const unsigned blocks = (unsigned)page_blocks(p);
        hipLaunchKernelGGL(count_live_kernel, dim3(blocks), dim3(256), 0, stream, p, w.counts);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((plan_moves_kernel<kBlockWaves>), dim3(blocks), dim3(256), 0, stream, p, w, copy_src,
                           copy_dst, n_copies);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t work_items = std::max<int64_t>(p.n_pages, p.n_slots * p.table_width);
    const int64_t remap = std::min<int64_t>(std::max<int64_t>((work_items + 255) / 256, 1), 4096);
    hipLaunchKernelGGL(remap_kernel, dim3((unsigned)remap), dim3(256), 0, stream, p, w, copy_dst, ref_out, table_out);
    return hipGetLastError();
}

hipError_t launch_pages_copy(const CopyParams& p, hipStream_t stream) {
    // eight workgroups of a CU at most, twice over
    const int64_t blocks = std::min<int64_t>(p.n_pairs * p.n_planes, 256 * 16);
    hipLaunchKernelGGL(copy_kernel, dim3((unsigned)blocks), dim3(kCopyThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace tl
