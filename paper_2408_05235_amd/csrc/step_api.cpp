// Host side of the norm before a product and of the next tokens: argument
// validation (before anything is enqueued) and kernel dispatch.
#include <hip/hip_runtime.h>

#include <cmath>

#include "status.h"
#include "step.h"
#include "tl.h"

namespace {

using tl::fail;
using tl::from_hip;
using tl::ok;

constexpr int64_t kMaxCount = 0x7fffffffll;

bool known_type(int32_t dtype) { return dtype == TL_BF16 || dtype == TL_F16 || dtype == TL_F32; }
bool aligned(const void* p, int32_t dtype) { return ((uintptr_t)p & (dtype == TL_F32 ? 3u : 1u)) == 0; }

// A call's output: where it lies, and its bytes (0: there is none).
struct Output {
    const void* at;
    uint64_t bytes;
};
bool overlap(const Output& a, const Output& b) {
    const uintptr_t x = (uintptr_t)a.at, y = (uintptr_t)b.at;
    return a.bytes && b.bytes && (x <= y ? y - x < a.bytes : x - y < b.bytes);
}

}  // namespace

extern "C" {

tl_status tl_norm(const tl_norm_args* a, void* stream) {
    const char* const who = "tl_norm";
    if (!a) return fail(TL_EINVAL, "%s: args is NULL", who);
    if (a->struct_size < sizeof(tl_norm_args))
        return fail(TL_EINVAL, "%s: struct_size %u < %zu", who, a->struct_size, sizeof(tl_norm_args));
    if (!known_type(a->dtype)) return fail(TL_EINVAL, "%s: dtype %d is none of TL_BF16, TL_F16 and TL_F32", who, a->dtype);
    if (a->n_rows < 0 || a->n_rows > kMaxCount)
        return fail(TL_EINVAL, "%s: n_rows %lld outside [0, 2^31-1]", who, (long long)a->n_rows);
    if (a->n_cols < 1 || a->n_cols > TL_MAX_COLUMNS)
        return fail(TL_EINVAL, "%s: n_cols %d outside [1, %d]", who, a->n_cols, TL_MAX_COLUMNS);
    if (a->group != TL_NORM_SAME && a->group != 0 &&
        (a->group < 16 || a->group > 512 || (a->group & (a->group - 1)) != 0))
        return fail(TL_EINVAL, "%s: group %d is neither TL_NORM_SAME nor 0 nor a power of two in [16, 512]", who, a->group);
    if (!(a->eps >= 0.0f) || !std::isfinite(a->eps)) return fail(TL_EINVAL, "%s: eps must be finite and not negative", who);
    if (a->x_stride < 0 || a->residual_stride < 0) return fail(TL_EINVAL, "%s: strides must not be negative", who);
    if (a->n_rows > 0) {
        if (!a->x || !a->weight || !a->out || (a->group != TL_NORM_SAME && !a->scale))
            return fail(TL_EINVAL, "%s: NULL required pointer", who);
        if (a->sum && !a->residual) return fail(TL_EINVAL, "%s: sum without residual", who);
    }
    if (!aligned(a->x, a->dtype) || !aligned(a->residual, a->dtype) || !aligned(a->weight, a->dtype) ||
        !aligned(a->sum, a->dtype) || (a->group == TL_NORM_SAME && !aligned(a->out, a->dtype)) ||
        ((uintptr_t)a->scale & 3u) != 0)
        return fail(TL_EINVAL, "%s: pointers must be aligned to their elements", who);
    if (a->n_rows == 0) return ok();
    const uint64_t rows = (uint64_t)a->n_rows, cols = (uint64_t)a->n_cols, size = a->dtype == TL_F32 ? 4 : 2;
    const uint64_t scales = a->group < 0 ? 0 : a->group == 0 ? 1 : (cols + a->group - 1) / a->group;
    const Output out{a->out, rows * cols * (a->group < 0 ? size : 1)}, scale{a->scale, rows * scales * sizeof(float)},
        sum{a->sum, a->sum ? rows * cols * size : 0};
    if (overlap(out, sum) || overlap(out, scale) || overlap(scale, sum))
        return fail(TL_EINVAL, "%s: out, scale and sum must not overlap", who);
    tl::NormParams p{};
    p.n_rows = a->n_rows;
    p.n_cols = a->n_cols;
    p.dtype = a->dtype;
    p.group = a->group;
    p.eps = a->eps;
    p.x = a->x;
    p.residual = a->residual;
    p.weight = a->weight;
    p.x_stride = a->x_stride;
    p.residual_stride = a->residual_stride;
    p.out = a->out;
    p.scale = a->scale;
    p.sum = a->sum;
    return from_hip(tl::launch_norm(p, (hipStream_t)stream), "tl_norm: launch");
}

tl_status tl_sample(const tl_sample_args* a, void* stream) {
    const char* const who = "tl_sample";
    if (!a) return fail(TL_EINVAL, "%s: args is NULL", who);
    if (a->struct_size < sizeof(tl_sample_args))
        return fail(TL_EINVAL, "%s: struct_size %u < %zu", who, a->struct_size, sizeof(tl_sample_args));
    if (!known_type(a->dtype)) return fail(TL_EINVAL, "%s: dtype %d is none of TL_BF16, TL_F16 and TL_F32", who, a->dtype);
    if (a->n_rows < 0 || a->n_rows > kMaxCount)
        return fail(TL_EINVAL, "%s: n_rows %lld outside [0, 2^31-1]", who, (long long)a->n_rows);
    if (a->n_cols < 1 || a->n_cols > TL_MAX_COLUMNS)
        return fail(TL_EINVAL, "%s: n_cols %d outside [1, %d]", who, a->n_cols, TL_MAX_COLUMNS);
    if (a->stride < 0) return fail(TL_EINVAL, "%s: stride must not be negative", who);
    if (a->n_rows > 0 && (!a->logits || !a->u || !a->token)) return fail(TL_EINVAL, "%s: NULL required pointer", who);
    if (!aligned(a->logits, a->dtype)) return fail(TL_EINVAL, "%s: logits must be aligned to their elements", who);
    if (a->n_rows == 0) return ok();
    tl::SampleParams p{};
    p.n_rows = a->n_rows;
    p.stride = a->stride;
    p.n_cols = a->n_cols;
    p.dtype = a->dtype;
    p.logits = a->logits;
    p.u = a->u;
    p.temperature = a->temperature;
    p.top_k = a->top_k;
    p.top_p = a->top_p;
    p.min_p = a->min_p;
    p.token = a->token;
    p.logprob = a->logprob;
    return from_hip(tl::launch_sample(p, (hipStream_t)stream), "tl_sample: launch");
}

}  // extern "C"
