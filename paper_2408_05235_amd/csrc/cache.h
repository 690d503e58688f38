// Internal interface between the host side of the paged cache and its
// attention (cache_api.cpp) and their kernels (pages.hip, attend.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_util.h"

namespace tl {

// One layer's pages and the sequences that use them (tl_kv_view).
struct CacheView {
    int32_t n_kv_heads, head_dim, page_tokens, table_width;
    int64_t n_pages, n_seqs;
    int64_t page_stride, head_stride, token_stride;   // elements
    DivU32 div_page;                // by page_tokens
    uint16_t* key;
    uint16_t* value;
    const int32_t* table;           // [n_seqs][table_width]
    const int32_t* length;          // [n_seqs]
    int64_t n_tokens;
    const int64_t* q_offset;        // [n_seqs + 1]; NULL = one token each
    const int32_t* granted;         // [n_seqs + 1], nullable: tokens that the sequences got
    bool refused_only;              // ... which count only where a sequence was refused
};

struct AppendParams {
    CacheView c;
    int32_t* appended;              // c.granted's last word
    const uint16_t* src[2];         // key, value
    int64_t token_stride[2], head_stride[2];
};

struct AttendParams {
    CacheView c;
    bool f16;                       // else bf16
    int32_t n_heads, group;         // group: query heads per KV head
    const uint16_t* query;
    int64_t query_token_stride, query_head_stride;
    float scale;
    int32_t window, sinks;
    int32_t max_length;             // 0 = unknown
    uint16_t* out;
    float* lse;                     // nullable
    void* workspace;                // nullable
    uint64_t workspace_bytes;
};

struct BoundsParams {
    CacheView c;                    // (without values)
    bool f16;
    int8_t* bounds;
    float* scale;
    int64_t scale_stride;
    int64_t slots;                  // places of touched pages, gaps included
};

struct SelectPagesParams {
    CacheView c;                    // (without keys and values)
    bool f16;
    int32_t group;                  // query heads per KV head
    const uint16_t* query;
    int64_t query_token_stride, query_head_stride;
    const int8_t* bounds;
    const float* scale;
    int64_t scale_stride;
    int32_t n_select, first, last;
    int32_t* selected;
    void* workspace;
    uint64_t workspace_bytes;
};

struct AttendPagesParams {
    AttendParams a;
    const int32_t* selected;
    int32_t n_select;
};

struct PagesParams {
    int32_t page_tokens, table_width;
    int64_t n_pages, n_slots;
    int32_t* ref;
    int32_t* table;
    int32_t* length;
    int32_t* granted;               // nullable
    DivU32 div_page;
};

struct CopyParams {
    unsigned char* pages;
    int64_t n_pages, page_bytes, page_stride, plane_stride, n_pairs;
    int32_t n_planes;
    const int32_t* src;
    const int32_t* dst;
    const int32_t* n_live;          // nullable
};

hipError_t launch_append(const AppendParams& p, hipStream_t stream);
hipError_t launch_attend(const AttendParams& p, hipStream_t stream);
// Workspace bytes that launch_attend splits its work with.
uint64_t attend_workspace_bytes(const AttendParams& p);

hipError_t launch_page_bounds(const BoundsParams& p, hipStream_t stream);
hipError_t launch_select_pages(const SelectPagesParams& p, hipStream_t stream);
// Workspace bytes that a call needs at least, and can use.
uint64_t select_workspace_least(const SelectPagesParams& p);
uint64_t select_workspace_bytes(const SelectPagesParams& p);
hipError_t launch_attend_pages(const AttendPagesParams& p, hipStream_t stream);
uint64_t attend_pages_workspace_bytes(const AttendPagesParams& p);

// int32 words of `work` of the page calls.
uint64_t pages_work_words(const PagesParams& p);
hipError_t launch_pages_extend(const PagesParams& p, const int32_t* add, int32_t* status, int32_t* work,
                               hipStream_t stream);
hipError_t launch_pages_fork(const PagesParams& p, int64_t n_forks, const int32_t* parent, const int32_t* child,
                             int32_t* copy_src, int32_t* copy_dst, int32_t* status, int32_t* work,
                             hipStream_t stream);
hipError_t launch_pages_free(const PagesParams& p, int64_t n_free, const int32_t* slots, hipStream_t stream);
hipError_t launch_pages_compact(const PagesParams& p, int32_t* ref_out, int32_t* table_out, int32_t* copy_src,
                                int32_t* copy_dst, int32_t* n_copies, int32_t* work, hipStream_t stream);
hipError_t launch_pages_copy(const CopyParams& p, hipStream_t stream);

}  // namespace tl
