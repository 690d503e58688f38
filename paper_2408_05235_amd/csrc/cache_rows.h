// Device side of the packed rows and the page table (tl_kv_view): which
// sequence a row belongs to, its position, and where a cached token lies.
#pragma once

#include "cache.h"

namespace tl {

// The tokens of an entry of `granted`: g, or refused (-1 - g) when it had got g.
__device__ __forceinline__ int32_t tokens_granted(int32_t granted) { return granted < 0 ? ~granted : granted; }

// The rows of sequence b: first and count (0 for malformed offsets), and the
// number of its cached tokens that exist (0 where its rows have no position).
struct SeqRows {
    int64_t first;
    int32_t n, length;
};

__device__ __forceinline__ int64_t clamp_offset(const CacheView& c, int64_t o) {
    return o < 0 ? 0 : o > c.n_tokens ? c.n_tokens : o;
}

// length[b] as it was given, but not below 0 (positions go by it).
__device__ __forceinline__ int32_t given_length(const CacheView& c, int64_t b) { return max(c.length[b], 0); }

// Tokens that the table has room for.
__device__ __forceinline__ int64_t table_tokens(const CacheView& c) { return (int64_t)c.table_width * c.page_tokens; }

__device__ __forceinline__ SeqRows seq_rows(const CacheView& c, int64_t b) {
    SeqRows s;
    if (c.q_offset) {
        s.first = clamp_offset(c, c.q_offset[b]);
        const int64_t end = clamp_offset(c, c.q_offset[b + 1]);
        s.n = end > s.first ? (int32_t)(end - s.first) : 0;
    } else {
        s.first = b;
        s.n = 1;
    }
    s.length = given_length(c, b);
    if (c.granted) {
        const int32_t got = c.granted[b];
        if ((got < 0 || !c.refused_only) && s.n > tokens_granted(got)) s.length = 0;
    }
    return s;
}

// The sequence of packed row i: the last b with q_offset[b] <= i.  False when
// the row belongs to none.
__device__ __forceinline__ bool find_seq(const CacheView& c, int64_t i, int64_t* seq) {
    if (!c.q_offset) {
        *seq = i;
        return true;
    }
    int64_t lo = 0, hi = c.n_seqs;          // q_offset[lo] <= i < q_offset[hi], as far as they are sorted
    if (c.q_offset[0] > i) return false;
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if (c.q_offset[mid] <= i) lo = mid;
        else hi = mid;
    }
    *seq = lo;
    return i < c.q_offset[lo + 1];
}

// Element offset of row 0 of head 0 of the page that holds token t, plus the
// row's; -1 when it has no page.  0 <= t < table_tokens(c).
__device__ __forceinline__ int64_t token_offset(const CacheView& c, const int32_t* table_row, int32_t t) {
    const uint32_t i = div_u32((uint32_t)t, c.div_page);
    const int32_t page = table_row[i];
    if (page < 0 || page >= c.n_pages) return -1;
    return (int64_t)page * c.page_stride + (int64_t)((uint32_t)t - i * (uint32_t)c.page_tokens) * c.token_stride;
}

}  // namespace tl
