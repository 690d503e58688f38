// Host side of the paged cache and its attention: argument validation (before
// anything is enqueued) and kernel dispatch.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>

#include "cache.h"
#include "status.h"
#include "tl.h"

namespace {

using tl::fail;
using tl::from_hip;
using tl::ok;

constexpr int64_t kMaxCount = 0x7fffffffll;

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Sizes of the structs without `granted`, which is NULL there.
constexpr size_t kAppendSize = offsetof(tl_kv_append_args, granted);
constexpr size_t kAttendSize = offsetof(tl_attend_args, granted);
constexpr size_t kPagesSize = offsetof(tl_pages, granted);

// Checks of a cache view and the packed rows that go with it, and their
// translation; `who` prefixes messages.
tl_status view_params(const tl_kv_view* v, int64_t n_tokens, const int64_t* q_offset, const char* who,
                      tl::CacheView* c) {
    if (v->struct_size < sizeof(tl_kv_view))
        return fail(TL_EINVAL, "%s: cache.struct_size %u < %zu", who, v->struct_size, sizeof(tl_kv_view));
    if (v->dtype != TL_BF16 && v->dtype != TL_F16)
        return fail(TL_EINVAL, "%s: dtype %d is neither TL_BF16 nor TL_F16", who, v->dtype);
    if (v->n_kv_heads < 1) return fail(TL_EINVAL, "%s: n_kv_heads %d < 1", who, v->n_kv_heads);
    if (v->head_dim < 8 || v->head_dim > TL_MAX_HEAD_DIM || v->head_dim % 8 != 0)
        return fail(TL_EINVAL, "%s: head_dim %d is not a multiple of 8 in [8, %d]", who, v->head_dim,
                    TL_MAX_HEAD_DIM);
    if (v->page_tokens < 1 || v->page_tokens > TL_MAX_BLOCK_TOKENS)
        return fail(TL_EINVAL, "%s: page_tokens %d outside [1, %d]", who, v->page_tokens, TL_MAX_BLOCK_TOKENS);
    if (v->table_width < 0) return fail(TL_EINVAL, "%s: table_width %d < 0", who, v->table_width);
    if (v->n_pages < 0 || v->n_pages > kMaxCount)
        return fail(TL_EINVAL, "%s: n_pages %lld outside [0, 2^31-1]", who, (long long)v->n_pages);
    if (v->n_seqs < 0 || v->n_seqs > kMaxCount)
        return fail(TL_EINVAL, "%s: n_seqs %lld outside [0, 2^31-1]", who, (long long)v->n_seqs);
    if (n_tokens < 0 || n_tokens > kMaxCount)
        return fail(TL_EINVAL, "%s: n_tokens %lld outside [0, 2^31-1]", who, (long long)n_tokens);
    if (!q_offset && n_tokens != v->n_seqs)
        return fail(TL_EINVAL, "%s: %lld tokens for %lld sequences without q_offset", who, (long long)n_tokens,
                    (long long)v->n_seqs);
    if (v->page_stride < 0 || v->head_stride < 0 || v->token_stride < 0 || v->page_stride % 8 != 0 ||
        v->head_stride % 8 != 0 || v->token_stride % 8 != 0)
        return fail(TL_EINVAL, "%s: page strides must be non-negative multiples of 8 elements", who);
    if (n_tokens > 0 && v->n_seqs > 0) {
        if (!v->length || (v->table_width > 0 && !v->page_table))
            return fail(TL_EINVAL, "%s: NULL required pointer", who);
        if (v->n_pages > 0 && (!v->key_pages || !v->value_pages)) return fail(TL_EINVAL, "%s: NULL pages", who);
    }
    if (!aligned16(v->key_pages) || !aligned16(v->value_pages))
        return fail(TL_EINVAL, "%s: pages must be 16-byte aligned", who);
    *c = tl::CacheView{};
    c->n_kv_heads = v->n_kv_heads;
    c->head_dim = v->head_dim;
    c->page_tokens = v->page_tokens;
    c->table_width = v->table_width;
    c->n_pages = v->n_pages;
    c->n_seqs = v->n_seqs;
    c->page_stride = v->page_stride;
    c->head_stride = v->head_stride;
    c->token_stride = v->token_stride;
    c->div_page = tl::make_divu32((uint32_t)v->page_tokens);
    c->key = (uint16_t*)v->key_pages;
    c->value = (uint16_t*)v->value_pages;
    c->table = v->page_table;
    c->length = v->length;
    c->n_tokens = n_tokens;
    c->q_offset = q_offset;
    return TL_OK;
}

tl_status attend_params(const tl_attend_args* a, const char* who, tl::AttendParams* p) {
    if (a->struct_size < kAttendSize)
        return fail(TL_EINVAL, "%s: struct_size %u < %zu", who, a->struct_size, kAttendSize);
    *p = tl::AttendParams{};
    const tl_status st = view_params(&a->cache, a->n_tokens, a->q_offset, who, &p->c);
    if (st != TL_OK) return st;
    if (a->n_heads < 1 || a->n_heads % a->cache.n_kv_heads != 0)
        return fail(TL_EINVAL, "%s: n_heads %d is not a positive multiple of n_kv_heads %d", who, a->n_heads,
                    a->cache.n_kv_heads);
    if (!(a->scale > 0.0f) || !std::isfinite(a->scale * 2.0f))      // (x log2 e below)
        return fail(TL_EINVAL, "%s: scale must be finite and positive", who);
    if (a->window < 0 || a->sinks < 0) return fail(TL_EINVAL, "%s: window or sinks < 0", who);
    if (a->max_length < 0) return fail(TL_EINVAL, "%s: max_length %d < 0", who, a->max_length);
    if (a->query_token_stride < 0 || a->query_head_stride < 0 || a->query_token_stride % 8 != 0 ||
        a->query_head_stride % 8 != 0)
        return fail(TL_EINVAL, "%s: query strides must be non-negative multiples of 8 elements", who);
    if (a->n_tokens > 0 && (!a->query || !a->out)) return fail(TL_EINVAL, "%s: NULL required pointer", who);
    if (!aligned16(a->query) || !aligned16(a->out) || !aligned16(a->workspace))
        return fail(TL_EINVAL, "%s: query, out and workspace must be 16-byte aligned", who);
    if ((int64_t)a->n_heads * a->n_tokens > kMaxCount)
        return fail(TL_EUNSUPPORTED, "%s: n_tokens x n_heads beyond 2^31-1", who);
    p->f16 = a->cache.dtype == TL_F16;
    p->n_heads = a->n_heads;
    p->group = a->n_heads / a->cache.n_kv_heads;
    p->query = (const uint16_t*)a->query;
    p->query_token_stride = a->query_token_stride;
    p->query_head_stride = a->query_head_stride;
    p->scale = a->scale;
    p->window = a->window;
    p->sinks = a->sinks;
    p->out = (uint16_t*)a->out;
    p->lse = a->lse;
    p->max_length = a->max_length;
    p->workspace = a->workspace;
    p->workspace_bytes = a->workspace ? a->workspace_bytes : 0;
    p->c.granted = a->struct_size >= sizeof(tl_attend_args) ? a->granted : nullptr;
    p->c.refused_only = true;
    if (p->c.n_pages == 0) p->c.table_width = 0;    // nothing is in the cache
    return TL_OK;
}

// `lengths`: whether the call uses table and lengths (compaction without
// slots does not).
tl_status pages_params(const tl_pages* g, const char* who, tl::PagesParams* p) {
    if (!g) return fail(TL_EINVAL, "%s: pages is NULL", who);
    if (g->struct_size < kPagesSize)
        return fail(TL_EINVAL, "%s: struct_size %u < %zu", who, g->struct_size, kPagesSize);
    if (g->page_tokens < 1 || g->page_tokens > TL_MAX_BLOCK_TOKENS)
        return fail(TL_EINVAL, "%s: page_tokens %d outside [1, %d]", who, g->page_tokens, TL_MAX_BLOCK_TOKENS);
    if (g->n_pages < 0 || g->n_pages > kMaxCount)
        return fail(TL_EINVAL, "%s: n_pages %lld outside [0, 2^31-1]", who, (long long)g->n_pages);
    if (g->n_slots < 0 || g->n_slots > kMaxCount)
        return fail(TL_EINVAL, "%s: n_slots %lld outside [0, 2^31-1]", who, (long long)g->n_slots);
    if (g->table_width < 0) return fail(TL_EINVAL, "%s: table_width %d < 0", who, g->table_width);
    if ((g->n_pages > 0 && !g->ref) || (g->n_slots > 0 && !g->length) ||
        (g->n_slots > 0 && g->table_width > 0 && !g->page_table))
        return fail(TL_EINVAL, "%s: NULL required pointer", who);
    *p = tl::PagesParams{};
    p->page_tokens = g->page_tokens;
    p->table_width = g->table_width;
    p->n_pages = g->n_pages;
    p->n_slots = g->n_slots;
    p->ref = g->ref;
    p->table = g->page_table;
    p->length = g->length;
    p->granted = g->struct_size >= sizeof(tl_pages) ? g->granted : nullptr;
    p->div_page = tl::make_divu32((uint32_t)g->page_tokens);
    return TL_OK;
}

}  // namespace

extern "C" {

tl_status tl_kv_append(const tl_kv_append_args* a, void* stream) {
    const char* const who = "tl_kv_append";
    if (!a) return fail(TL_EINVAL, "%s: args is NULL", who);
    if (a->struct_size < kAppendSize)
        return fail(TL_EINVAL, "%s: struct_size %u < %zu", who, a->struct_size, kAppendSize);
    tl::AppendParams p{};
    const tl_status st = view_params(&a->cache, a->n_tokens, a->q_offset, who, &p.c);
    if (st != TL_OK) return st;
    if (a->n_tokens > 0 && (!a->key || !a->value)) return fail(TL_EINVAL, "%s: NULL required pointer", who);
    if (!aligned16(a->key) || !aligned16(a->value))
        return fail(TL_EINVAL, "%s: key and value must be 16-byte aligned", who);
    const int64_t strides[4] = {a->key_token_stride, a->key_head_stride, a->value_token_stride, a->value_head_stride};
    for (int64_t s : strides)
        if (s < 0 || s % 8 != 0)
            return fail(TL_EINVAL, "%s: strides must be non-negative multiples of 8 elements", who);
    p.src[0] = (const uint16_t*)a->key;
    p.src[1] = (const uint16_t*)a->value;
    p.token_stride[0] = a->key_token_stride;
    p.token_stride[1] = a->value_token_stride;
    p.head_stride[0] = a->key_head_stride;
    p.head_stride[1] = a->value_head_stride;
    if (a->struct_size >= sizeof(tl_kv_append_args) && a->granted) {
        p.c.granted = a->granted;
        p.appended = a->granted + p.c.n_seqs;
    }
    if (a->n_tokens == 0 || p.c.n_seqs == 0 || p.c.n_pages == 0 || p.c.table_width == 0) return ok();
    return from_hip(tl::launch_append(p, (hipStream_t)stream), "tl_kv_append: launch");
}

tl_status tl_attend(const tl_attend_args* a, void* stream) {
    if (!a) return fail(TL_EINVAL, "tl_attend: args is NULL");
    tl::AttendParams p;
    const tl_status st = attend_params(a, "tl_attend", &p);
    if (st != TL_OK) return st;
    if (a->n_tokens == 0 || p.c.n_seqs == 0) return ok();
    return from_hip(tl::launch_attend(p, (hipStream_t)stream), "tl_attend: launch");
}

uint64_t tl_attend_workspace_bytes(const tl_attend_args* a) {
    tl::AttendParams p;
    if (!a || attend_params(a, "tl_attend_workspace_bytes", &p) != TL_OK) return 0;
    return tl::attend_workspace_bytes(p);
}

uint64_t tl_pages_work_words(const tl_pages* g) {
    tl::PagesParams p;
    if (pages_params(g, "tl_pages_work_words", &p) != TL_OK) return 0;
    return tl::pages_work_words(p);
}

tl_status tl_pages_extend(const tl_pages* g, const int32_t* add, int32_t* status, int32_t* work, void* stream) {
    tl::PagesParams p;
    const tl_status st = pages_params(g, "tl_pages_extend", &p);
    if (st != TL_OK) return st;
    if (p.n_slots == 0) return ok();
    if (!add || !status || !work) return fail(TL_EINVAL, "tl_pages_extend: NULL required pointer");
    return from_hip(tl::launch_pages_extend(p, add, status, work, (hipStream_t)stream), "tl_pages_extend: launch");
}

tl_status tl_pages_fork(const tl_pages* g, int64_t n_forks, const int32_t* parent, const int32_t* child,
                        int32_t* copy_src, int32_t* copy_dst, int32_t* status, int32_t* work, void* stream) {
    tl::PagesParams p;
    const tl_status st = pages_params(g, "tl_pages_fork", &p);
    if (st != TL_OK) return st;
    if (n_forks < 0 || n_forks > p.n_slots)
        return fail(TL_EINVAL, "tl_pages_fork: n_forks %lld outside [0, n_slots]", (long long)n_forks);
    if (n_forks == 0) return ok();
    if (!parent || !child || !copy_src || !copy_dst || !status || !work)
        return fail(TL_EINVAL, "tl_pages_fork: NULL required pointer");
    return from_hip(tl::launch_pages_fork(p, n_forks, parent, child, copy_src, copy_dst, status, work,
                                          (hipStream_t)stream),
                    "tl_pages_fork: launch");
}

tl_status tl_pages_free(const tl_pages* g, int64_t n_free, const int32_t* slots, void* stream) {
    tl::PagesParams p;
    const tl_status st = pages_params(g, "tl_pages_free", &p);
    if (st != TL_OK) return st;
    if (n_free < 0 || n_free > kMaxCount)
        return fail(TL_EINVAL, "tl_pages_free: n_free %lld outside [0, 2^31-1]", (long long)n_free);
    if (n_free == 0 || p.n_slots == 0) return ok();
    if (!slots) return fail(TL_EINVAL, "tl_pages_free: NULL required pointer");
    return from_hip(tl::launch_pages_free(p, n_free, slots, (hipStream_t)stream), "tl_pages_free: launch");
}

tl_status tl_pages_compact(const tl_pages* g, int32_t* ref_out, int32_t* table_out, int32_t* copy_src,
                           int32_t* copy_dst, int32_t* n_copies, int32_t* work, void* stream) {
    tl::PagesParams p;
    const tl_status st = pages_params(g, "tl_pages_compact", &p);
    if (st != TL_OK) return st;
    if (!n_copies || !work || (p.n_pages > 0 && !ref_out) || (p.n_pages > 1 && (!copy_src || !copy_dst)) ||
        (p.n_slots > 0 && p.table_width > 0 && !table_out))
        return fail(TL_EINVAL, "tl_pages_compact: NULL required pointer");
    return from_hip(tl::launch_pages_compact(p, ref_out, table_out, copy_src, copy_dst, n_copies, work,
                                             (hipStream_t)stream),
                    "tl_pages_compact: launch");
}

tl_status tl_pages_copy(void* pages, int64_t n_pages, int64_t page_bytes, int64_t page_stride, int32_t n_planes,
                        int64_t plane_stride, const int32_t* copy_src, const int32_t* copy_dst, int64_t n_pairs,
                        const int32_t* n_live, void* stream) {
    if (n_pages < 0 || n_pages > kMaxCount)
        return fail(TL_EINVAL, "tl_pages_copy: n_pages %lld outside [0, 2^31-1]", (long long)n_pages);
    if (n_pairs < 0 || n_pairs > kMaxCount)
        return fail(TL_EINVAL, "tl_pages_copy: n_pairs %lld outside [0, 2^31-1]", (long long)n_pairs);
    if (n_planes < 0) return fail(TL_EINVAL, "tl_pages_copy: n_planes %d < 0", n_planes);
    if (page_bytes < 0 || page_stride < 0 || plane_stride < 0 ||
        ((page_bytes | page_stride | plane_stride) & 15) != 0 || !aligned16(pages))
        return fail(TL_EINVAL, "tl_pages_copy: pages, their size and strides must be multiples of 16 bytes");
    if (n_pages == 0 || n_pairs == 0 || n_planes == 0 || page_bytes == 0) return ok();
    if (!pages || !copy_src || !copy_dst) return fail(TL_EINVAL, "tl_pages_copy: NULL required pointer");
    tl::CopyParams p{};
    p.pages = (unsigned char*)pages;
    p.n_pages = n_pages;
    p.page_bytes = page_bytes;
    p.page_stride = page_stride;
    p.n_planes = n_planes;
    p.plane_stride = plane_stride;
    p.src = copy_src;
    p.dst = copy_dst;
    p.n_pairs = n_pairs;
    p.n_live = n_live;
    return from_hip(tl::launch_pages_copy(p, (hipStream_t)stream), "tl_pages_copy: launch");
}

}  // extern "C"
