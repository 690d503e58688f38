// The next tokens from their logits (tl_sample).
//
// Weights are whole numbers (2^40 for the largest), so that their sums, and with
// them the token, do not depend on how a row is cut.  A filter is a threshold: the
// kept tokens are those above a logit, and of those that equal it the first few in
// index order, which all weigh the same.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "device_util.h"
#include "step.h"
#include "tl.h"
#include "tl_internal.h"

namespace tl {
namespace {

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / kWave;
constexpr double kUnit = 0x1p40;

template <int DT>
using elem = std::conditional_t<DT == TL_F32, float, uint16_t>;

// A logit; NaN counts as -inf, and there is one zero.
template <int DT>
__device__ __forceinline__ float logit(elem<DT> x) {
    float f;
    if constexpr (DT == TL_F32) f = x;
    else if constexpr (DT == TL_F16) f = (float)__builtin_bit_cast(_Float16, x);
    else f = __builtin_bit_cast(float, (uint32_t)x << 16);
    return f != f ? -INFINITY : f + 0.0f;
}

// Orders as the logits do; -inf is kLeast, below every other.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr uint32_t kLeast = 0x007fffffu;

// (x - m) / T in 64 bits, 0 at the largest whatever T is.
__device__ __forceinline__ double exponent(float x, float m, double inverse) {
    return x == m ? 0.0 : x == -INFINITY || m == INFINITY ? -INFINITY : ((double)x - (double)m) * inverse;
}
__device__ __forceinline__ uint64_t weight_of(float x, float m, double inverse) {
    return (uint64_t)rint(exp(exponent(x, m, inverse)) * kUnit);
}

struct SampleLds {
    uint64_t sums[2048];
    uint32_t counts[2048];
    uint64_t wave[kSampleWaves];
    uint32_t wave_ties[kSampleWaves];
    uint64_t found[3];
};

__device__ __forceinline__ uint64_t block_sum(uint64_t v, SampleLds& lds) {
    v = wave_sum_u64(v);
    __syncthreads();
    if (lane_id() == 0) lds.wave[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < kSampleWaves; ++w) v += lds.wave[w];
    return v;
}

template <int DT>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleParams P, int64_t first) {
    __shared__ SampleLds lds;
    const int64_t row = blockIdx.x + first;
    const elem<DT>* const x = (const elem<DT>*)P.logits + row * P.stride;
    const int32_t V = P.n_cols;
    const int tid = threadIdx.x, wave = tid / kWave, lane = lane_id();

    // the largest, and its first place: its key above the place's complement
    uint64_t top = 0;
    for (int32_t i = tid; i < V; i += kSampleThreads)
        top = max(top, (uint64_t)order_of(logit<DT>(x[i])) << 32 | (uint32_t)~i);
    for (int o = 1; o < kWave; o <<= 1) top = max(top, (uint64_t)__shfl_xor((unsigned long long)top, o));
    if (lane == 0) lds.wave[wave] = top;
    __syncthreads();
    for (int w = 0; w < kSampleWaves; ++w) top = max(top, lds.wave[w]);
    const uint32_t most = (uint32_t)(top >> 32);
    const float T = P.temperature ? P.temperature[row] : 1.0f;
    if (most == kLeast || !(T > 0.0f)) {
        if (tid == 0) {
            P.token[row] = most == kLeast ? -1 : (int32_t)~(uint32_t)top;
            if (P.logprob) P.logprob[row] = most == kLeast ? -INFINITY : 0.0f;
        }
        return;
    }
    const float m = value_of(most);
    const double inverse = 1.0 / (double)T;

    // kept: keys above `least`, and the first `ties` of those that equal it
    uint32_t least = kLeast;
    uint32_t ties = 0;
    const int32_t k = P.top_k ? P.top_k[row] : 0;
    // the threshold by digits of 11, 11 and 10 bits, by count (rank `left`) or by weight
    auto narrow = [&](bool by_weight, uint64_t left, uint32_t below, uint32_t below_ties) {
        uint32_t prefix = 0, mask = 0;
        for (int step = 0; step < 3; ++step) {
            const int shift = step == 0 ? 21 : step == 1 ? 10 : 0, n = step == 2 ? 1024 : 2048;
            for (int e = tid; e < 2048; e += kSampleThreads) {
                lds.sums[e] = 0;
                lds.counts[e] = 0;
            }
            __syncthreads();
            for (int32_t i = tid; i < V; i += kSampleThreads) {
                const float f = logit<DT>(x[i]);
                const uint32_t key = order_of(f);
                if (key < below || (key & mask) != prefix) continue;
                const uint32_t digit = key >> shift & (n - 1);
                if (!by_weight) atomicAdd(&lds.counts[digit], 1u);
                else if (key != below)       // (those come below)
                    atomicAdd((unsigned long long*)&lds.sums[digit], (unsigned long long)weight_of(f, m, inverse));
            }
            __syncthreads();
            if (by_weight && tid == 0 && (below & mask) == prefix && below_ties > 0)
                lds.sums[below >> shift & (n - 1)] += below_ties * weight_of(value_of(below), m, inverse);
            __syncthreads();
            if (wave == 0) {
                // lane l has n / 64 digits from the top
                const int per = n / kWave, d0 = n - 1 - lane * per;
                uint64_t sum = 0;
                for (int e = 0; e < per; ++e) sum += by_weight ? lds.sums[d0 - e] : lds.counts[d0 - e];
                uint64_t at = wave_incl_scan_u64(sum) - sum;
                for (int e = 0; e < per; ++e) {
                    const uint64_t d = by_weight ? lds.sums[d0 - e] : lds.counts[d0 - e];
                    if (at < left && at + d >= left) {
                        lds.found[0] = (uint64_t)(d0 - e);
                        lds.found[1] = left - at;
                    }
                    at += d;
                }
            }
            __syncthreads();
            prefix |= (uint32_t)lds.found[0] << shift;
            mask |= (uint32_t)(n - 1) << shift;
            left = lds.found[1];
            __syncthreads();
        }
        least = prefix;
        const uint64_t w = by_weight ? weight_of(value_of(prefix), m, inverse) : 1;
        ties = (uint32_t)((left + w - 1) / w);
    };
    if (k > 0 && k < V) narrow(false, (uint64_t)k, 0, 0);
    const float p = P.top_p ? P.top_p[row] : 1.0f;
    if (p < 1.0f) {
        uint64_t sum = 0;
        for (int32_t i = tid; i < V; i += kSampleThreads) {
            const float f = logit<DT>(x[i]);
            if (order_of(f) > least) sum += weight_of(f, m, inverse);
        }
        const uint64_t total = block_sum(sum, lds) + ties * weight_of(value_of(least), m, inverse);
        const double need = ceil((double)p * (double)total);
        const uint64_t left = need < 1.0 ? 1 : min((uint64_t)need, total);
        __syncthreads();
        narrow(true, left, least, ties);
    }
    const float q = P.min_p ? P.min_p[row] : 0.0f;
    const uint64_t lightest = q > 0.0f ? (uint64_t)ceil((double)fminf(q, 1.0f) * kUnit) : 0;
    auto kept = [&](float f) {
        const uint64_t w = order_of(f) > least ? weight_of(f, m, inverse) : 0;
        return w >= lightest ? w : 0;
    };
    uint64_t tie = ties ? weight_of(value_of(least), m, inverse) : 0;
    if (tie < lightest) tie = 0;

    // the token: a range of the row per wavefront, then the range's own
    const int32_t range = (V + kSampleWaves - 1) / kSampleWaves;
    int32_t i0 = min(wave * range, V);
    const int32_t i1 = min(i0 + range, V);
    uint64_t sum = 0;
    uint32_t equal = 0;
    for (int32_t i = i0 + lane; i < i1; i += kWave) {
        const float f = logit<DT>(x[i]);
        sum += kept(f);
        equal += order_of(f) == least;
    }
    sum = wave_sum_u64(sum);
    equal = (uint32_t)wave_sum((int32_t)equal);
    __syncthreads();
    if (lane == 0) {
        lds.wave[wave] = sum;
        lds.wave_ties[wave] = equal;
    }
    __syncthreads();
    uint64_t total = 0, before = 0;
    uint32_t ties_before = 0, all_ties = 0;
    for (int w = 0; w < kSampleWaves; ++w) {
        if (w == wave) before = total, ties_before = all_ties;
        total += lds.wave[w];
        all_ties += lds.wave_ties[w];
    }
    total += min(all_ties, ties) * tie;
    before += min(ties_before, ties) * tie;
    const double u = (double)P.u[row];
    const double at = floor(u * (double)total);
    const uint64_t r = at > 0.0 ? at < (double)total ? (uint64_t)at : total - 1 : 0;
    const uint64_t end = before + sum + (min(ties_before + equal, ties) - min(ties_before, ties)) * tie;
    if (r < before || r >= end) return;         // (one wavefront goes on)
    for (; i0 < i1; i0 += kWave) {
        const int32_t i = i0 + lane;
        const float f = i < i1 ? logit<DT>(x[i]) : -INFINITY;
        const bool eq = i < i1 && ties > 0 && order_of(f) == least;
        const uint64_t mask = __ballot(eq);
        const uint32_t rank = ties_before + __popcll(mask & ((1ull << lane) - 1));
        const uint64_t w = i >= i1 ? 0 : eq ? rank < ties ? tie : 0 : kept(f);
        const uint64_t incl = before + wave_incl_scan_u64(w);
        const uint64_t hit = __ballot(incl > r);
        if (hit) {
            if (lane == __ffsll((unsigned long long)hit) - 1) {
                P.token[row] = i;
                if (P.logprob) P.logprob[row] = (float)(exponent(f, m, inverse) - log((double)total / kUnit));
            }
            return;
        }
        before = lane63_u64(incl);
        ties_before += __popcll(mask);
    }
}

template <int DT>
hipError_t launch_type(const SampleParams& p, hipStream_t stream) {
    return launch_all(p.n_rows, kSampleThreads, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((sample_kernel<DT>), grid, dim3(kSampleThreads), 0, stream, p, first);
    });
}

}  // namespace

hipError_t launch_sample(const SampleParams& p, hipStream_t stream) {
    if (p.dtype == TL_F32) return launch_type<TL_F32>(p, stream);
    return p.dtype == TL_F16 ? launch_type<TL_F16>(p, stream) : launch_type<TL_BF16>(p, stream);
}

}  // namespace tl
