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

// How a row's elements are read: 16 bytes a lane, rows from any element on.
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t piece16;
typedef __attribute__((ext_vector_type(4), aligned(4))) uint32_t piece32;
template <int DT>
struct Piece {
    static constexpr int kPer = DT == TL_F32 ? 4 : 8;
    typedef std::conditional_t<DT == TL_F32, piece32, piece16> vec;
    __device__ static __forceinline__ void split(vec v, float (&x)[kPer]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (a value of its own: a bit cast of a vector's element takes the first one)
            const uint32_t w = v[i];
            if constexpr (DT == TL_F32) {
                x[i] = logit<DT>(__builtin_bit_cast(float, w));
            } else {
                x[2 * i] = logit<DT>((uint16_t)w);
                x[2 * i + 1] = logit<DT>((uint16_t)(w >> 16));
            }
        }
    }
};

// f(index, logit) for the elements of [i0, i1), a wavefront's, in no order.
template <int DT, class F>
__device__ __forceinline__ void each_of(const elem<DT>* x, int32_t i0, int32_t i1, F f) {
    using P = Piece<DT>;
    constexpr int kStep = kWave * P::kPer, kBatch = DT == TL_F32 ? 4 : 2;
    int32_t i = i0 + lane_id() * P::kPer;
    for (; i0 + kBatch * kStep <= i1; i0 += kBatch * kStep, i += kBatch * kStep) {
        typename P::vec v[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) v[b] = *(const typename P::vec*)(x + i + b * kStep);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            float y[P::kPer];
            P::split(v[b], y);
#pragma unroll
            for (int e = 0; e < P::kPer; ++e) f(i + b * kStep + e, y[e]);
        }
    }
    for (; i0 < i1; i0 += kStep, i += kStep) {
        if (i + P::kPer <= i1) {
            float y[P::kPer];
            P::split(*(const typename P::vec*)(x + i), y);
#pragma unroll
            for (int e = 0; e < P::kPer; ++e) f(i + e, y[e]);
        } else {
            for (int e = 0; i + e < i1; ++e) f(i + e, logit<DT>(x[i + e]));
        }
    }
}

// Bins of logits, from the top: 1 / kPerT of a temperature wide, the last one where all
// weights are 0 (30 temperatures below the largest: exp(-30) < 2^-41).
constexpr int kBins = 2048, kAboveBins = 256;
constexpr float kPerT = 59.0f;
struct Binning {
    float half_from, per;   // (halves, whose difference is finite; per: of them)
    __device__ __forceinline__ int operator()(float x) const {
        // (monotone: each operation is; a NaN, of infinities, goes to the top)
        return (int)fminf(fmaxf((half_from - x * 0.5f) * per + (float)kAboveBins, 0.0f), (float)(kBins - 1));
    }
};

// WAVES wavefronts hold up to CAP tokens of a row in LDS, of the bins in which a
// threshold can be.
template <int WAVES, int CAP>
struct SampleLds {
    uint32_t key[CAP], index[CAP];
    uint32_t bins[kBins];
    uint64_t sums[256];
    uint32_t counts[256];
    uint64_t wave[WAVES], light[WAVES], chunk[WAVES];
    float wave_low[WAVES], wave_high[WAVES];
    uint32_t wave_count[WAVES];
    uint64_t found[2];
    int32_t low, high;
    uint32_t n;
};

template <int WAVES>
__device__ __forceinline__ uint64_t block_sum(uint64_t v, uint64_t* of_waves) {
    v = wave_sum_u64(v);
    __syncthreads();
    if (lane_id() == 0) of_waves[wave_number()] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < WAVES; ++w) v += of_waves[w];
    return v;
}

// What is kept: keys above `least`, and those that equal it up to index `until`.
struct Kept {
    uint32_t least;
    uint32_t until;
    __device__ __forceinline__ bool operator()(uint32_t key, uint32_t index) const {
        return key > least || (key == least && index <= until);
    }
};

// One workgroup a row.  The row is read twice and a sixteenth: once for its
// largest logit and the counts of its bins, which say where the thresholds of top-k and
// top-p can lie; then for the sums of what is surely kept (and, for top-p alone, of
// all), while the tokens of the bins between go to LDS, where the thresholds are
// found; and the range of a wavefront that the number falls into.  Where those bins hold
// too many tokens the thresholds are found by digits of the whole row's keys.
template <int DT, int WAVES, int CAP>
__global__ __launch_bounds__(WAVES * kWave) void sample_kernel(SampleParams P, int64_t first) {
    constexpr int kThreads = WAVES * kWave;
    __shared__ SampleLds<WAVES, CAP> lds;
    const int64_t row = blockIdx.x + first;
    const elem<DT>* const x = (const elem<DT>*)P.logits + row * P.stride;
    const int32_t V = P.n_cols;
    const int tid = threadIdx.x, wave = wave_number(), lane = lane_id();
    // a wavefront's range of the row
    constexpr int kRound = kWave * Piece<DT>::kPer;
    const int32_t range = ((V + WAVES - 1) / WAVES + kRound - 1) / kRound * kRound;
    const int32_t i0 = (int32_t)min((int64_t)wave * range, (int64_t)V), i1 = min(i0 + range, V);

    const float T = P.temperature ? P.temperature[row] : 1.0f;
    const bool draws = T > 0.0f;
    const int32_t k = draws && P.top_k ? P.top_k[row] : 0;
    const float p = draws && P.top_p ? P.top_p[row] : 1.0f;
    const bool by_k = k > 0 && k < V, by_p = p < 1.0f;
    const bool binned = V > CAP && (by_k || by_p);

    // the largest logit, and its first place: its key above the place's complement
    uint64_t top = 0;
    Binning bin = {0.0f, 0.0f};
    if (binned) {
        // bins begin a little above the largest of a few
        float m0 = -INFINITY;
        for (int32_t i = tid; i < min(V, 4 * kThreads); i += kThreads) m0 = fmaxf(m0, logit<DT>(x[i]));
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) m0 = fmaxf(m0, __shfl_xor(m0, o));
        if (lane == 0) lds.wave_low[wave] = m0;
        for (int b = tid; b < kBins; b += kThreads) lds.bins[b] = 0;
        __syncthreads();
        for (int w = 0; w < WAVES; ++w) m0 = fmaxf(m0, lds.wave_low[w]);
        bin = {m0 == -INFINITY ? 0.0f : m0 * 0.5f, 2.0f * kPerT / T};
        float m1 = -INFINITY;
        int32_t at = 0;
        each_of<DT>(x, i0, i1, [&](int32_t i, float f) {
            // (a lane's indices ascend)
            if (f > m1) m1 = f, at = i;
            const int b = bin(f);
            if (b < kBins - 1 && f > -INFINITY) atomicAdd(&lds.bins[b], 1u);
        });
        top = (uint64_t)order_of(m1) << 32 | (uint32_t)~at;
    } else {
        float m1 = -INFINITY;
        int32_t at = 0;
        each_of<DT>(x, i0, i1, [&](int32_t i, float f) {
            if (f > m1) m1 = f, at = i;
        });
        top = (uint64_t)order_of(m1) << 32 | (uint32_t)~at;
    }
    for (int o = 1; o < kWave; o <<= 1) top = max(top, (uint64_t)__shfl_xor((unsigned long long)top, o));
    if (lane == 0) lds.wave[wave] = top;
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) top = max(top, lds.wave[w]);
    const uint32_t most = (uint32_t)(top >> 32);
    if (most == kLeast || !draws) {
        if (tid == 0) {
            P.token[row] = most == kLeast ? -1 : (int32_t)~(uint32_t)top;
            if (P.logprob) P.logprob[row] = most == kLeast ? -INFINITY : 0.0f;
        }
        return;
    }
    const float m = value_of(most);
    const double inverse = 1.0 / (double)T;
    const float q = P.min_p ? P.min_p[row] : 0.0f;
    const uint64_t lightest = q > 0.0f ? (uint64_t)ceil((double)fminf(q, 1.0f) * kUnit) : 0;

    // the bins that go to LDS: [low, high] (those above are kept, those below not)
    bool listed = by_k || by_p, counts_all = by_p, limited = by_k;
    int32_t low = 0, high = kBins - 1;
    uint64_t rank = (uint64_t)max(k, 0);            // of the last one kept by top-k, among those listed
    if (!listed) low = kBins;
    if (binned) {
        // each lane has kPerLane bins: counts before them, and what the bins' weights
        // are at least and at most (an edge is off by less than 1e-3 of a bin)
        constexpr int kPerLane = kBins / kThreads;
        uint32_t count[kPerLane], own = 0;
        float least_w[kPerLane], most_w[kPerLane], own_low = 0.0f, own_high = 0.0f;
        const float shift = (bin.half_from - m * 0.5f) / T * 2.0f;
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) {
            const int b = tid * kPerLane + e;
            count[e] = lds.bins[b];
            own += count[e];
            const float edge = shift + (float)(kAboveBins - b) / kPerT;
            most_w[e] = (float)count[e] * __expf(fminf(edge + 1e-3f / kPerT, 0.0f)) * 1.0001f;
            least_w[e] = (float)count[e] * __expf(fminf(edge - 1.001f / kPerT, 0.0f)) * 0.9999f;
            // the top bin goes up to the largest logit, which is in it where any is
            if (b == 0) {
                most_w[e] = (float)count[e];
                least_w[e] = count[e] ? fmaxf(least_w[e], 1.0f) : 0.0f;
            }
            own_low += least_w[e];
            own_high += most_w[e];
        }
        uint32_t c = (uint32_t)wave_incl_scan((int32_t)own);
        float sl = own_low, sh = own_high;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const float a = __shfl_up(sl, o), z = __shfl_up(sh, o);
            if (lane >= o) sl += a, sh += z;
        }
        __syncthreads();
        if (lane == kWave - 1) {
            lds.wave_count[wave] = c;
            lds.wave_low[wave] = sl;
            lds.wave_high[wave] = sh;
        }
        if (tid == 0) lds.low = lds.high = kBins - 1, lds.found[0] = lds.found[1] = 0;
        __syncthreads();
        float all_low = 0.0f, all_high = 0.0f;
        uint32_t all = 0;
        c -= own;
        sl -= own_low;
        sh -= own_high;
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) c += all, sl += all_low, sh += all_high;
            all += lds.wave_count[w];
            all_low += lds.wave_low[w];
            all_high += lds.wave_high[w];
        }
        if (by_k && (uint32_t)k <= all) {
            // the bin of the last one that top-k keeps
#pragma unroll
            for (int e = 0; e < kPerLane; ++e) {
                if (c < (uint32_t)k && c + count[e] >= (uint32_t)k) {
                    lds.high = tid * kPerLane + e;
                    lds.found[0] = c;
                    lds.found[1] = c + count[e];
                }
                c += count[e];
            }
            __syncthreads();
            high = lds.high;
            counts_all = false;
            const uint32_t before = (uint32_t)lds.found[0], upto = (uint32_t)lds.found[1];
            if (upto <= CAP) {
                low = 0;
            } else if (!by_p && upto - before <= CAP) {
                low = high;
                rank -= before;
            } else {
                listed = false;
            }
        } else {
            limited = false;                        // (all with a weight)
            if (by_p) {
                // fp32 sums of 2048 are off by less than 2^-12; the first bin by whose end
                // the sum can, and the one by which it must have reached top_p's
                const float reach_low = p * all_low * (1.0f - 0x1p-11f), reach_high = p * all_high * (1.0f + 0x1p-11f);
                uint32_t in = 0;
                int32_t mine_low = kBins - 1, mine_high = kBins - 1;
#pragma unroll
                for (int e = kPerLane - 1; e >= 0; --e) {
                    float upto_low = sl, upto_high = sh;
#pragma unroll
                    for (int y = 0; y <= e; ++y) upto_low += least_w[y], upto_high += most_w[y];
                    if (upto_high * (1.0f + 0x1p-11f) >= reach_low) mine_low = tid * kPerLane + e;
                    if (upto_low > 0.0f && upto_low * (1.0f - 0x1p-11f) >= reach_high) mine_high = tid * kPerLane + e;
                }
                atomicMin(&lds.low, mine_low);
                atomicMin(&lds.high, mine_high);
                __syncthreads();
                low = lds.low;
                high = lds.high;
#pragma unroll
                for (int e = 0; e < kPerLane; ++e) {
                    const int b = tid * kPerLane + e;
                    if (b >= low && b <= high) in += count[e];
                }
                in = (uint32_t)block_sum<WAVES>(in, lds.wave);
                listed = in <= CAP;
            } else {
                listed = false;                     // nothing to find: all are kept
                low = kBins;
            }
        }
    }
    const bool whole = !listed && low < kBins;      // thresholds from the row itself

    // sums of what is kept above the list, by wavefront, and of all; the list
    if (tid == 0) lds.n = 0;
    __syncthreads();
    uint64_t above = 0, light = 0, below = 0;
    if (!whole) {
        const bool sums = low > 0 || counts_all;    // (else only the list counts)
        each_of<DT>(x, i0, i1, [&](int32_t i, float f) {
            const int b = binned ? bin(f) : listed ? 0 : -1;
            if (b < low) {
                const uint64_t w = weight_of(f, m, inverse);
                above += w;
                light += w >= lightest ? w : 0;
            } else if (b <= high) {
                if (f > -INFINITY) {
                    const uint32_t at = atomicAdd(&lds.n, 1u);
                    if (at < CAP) {
                        lds.key[at] = order_of(f);
                        lds.index[at] = (uint32_t)i;
                    }
                }
            } else if (sums) {
                below += weight_of(f, m, inverse);
            }
        });
    }
    light = wave_sum_u64(light);
    if (lane == 0) lds.light[wave] = light;
    const uint64_t all_above = block_sum<WAVES>(above, lds.wave);
    const uint32_t n = min(lds.n, (uint32_t)CAP);

    // f(index, key) of the list, or of the row
    auto each = [&](auto f) {
        if (whole) each_of<DT>(x, i0, i1, [&](int32_t i, float y) { f((uint32_t)i, order_of(y)); });
        else
            for (uint32_t e = tid; e < n; e += kThreads) f(lds.index[e], lds.key[e]);
    };
    // The `left`-th largest code by digits of 8 bits, by count or by weight.  what(index,
    // key, &code) says whether a token counts; returns how much is left at the code.
    auto narrow = [&](bool by_weight, uint64_t* left, auto what) {
        uint32_t prefix = 0, mask = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int e = tid; e < 256; e += kThreads) {
                lds.sums[e] = 0;
                lds.counts[e] = 0;
            }
            __syncthreads();
            each([&](uint32_t index, uint32_t key) {
                uint32_t code;
                if (!what(index, key, &code) || (code & mask) != prefix) return;
                if (by_weight)
                    atomicAdd((unsigned long long*)&lds.sums[code >> shift & 255],
                              (unsigned long long)weight_of(value_of(key), m, inverse));
                else atomicAdd(&lds.counts[code >> shift & 255], 1u);
            });
            __syncthreads();
            if (wave == 0) {
                // lane l has the digits 255 - 4 l .. 252 - 4 l
                uint64_t d[4], sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    d[e] = by_weight ? lds.sums[255 - 4 * lane - e] : lds.counts[255 - 4 * lane - e];
                    sum += d[e];
                }
                uint64_t at = wave_incl_scan_u64(sum) - sum;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (at < *left && at + d[e] >= *left) {
                        lds.found[0] = (uint64_t)(255 - 4 * lane - e);
                        lds.found[1] = *left - at;
                    }
                    at += d[e];
                }
            }
            __syncthreads();
            prefix |= (uint32_t)lds.found[0] << shift;
            mask |= 255u << shift;
            *left = lds.found[1];
            __syncthreads();
        }
        return prefix;
    };
    // the place of the `ties`-th of the tokens that equal the threshold
    auto place = [&](uint32_t least, uint64_t ties) {
        return ~narrow(false, &ties, [&](uint32_t index, uint32_t key, uint32_t* code) {
            *code = ~index;
            return key == least;
        });
    };

    Kept kept = {kLeast, 0};
    if (limited) {
        uint64_t left = whole ? (uint64_t)k : rank;
        // (a list of the whole row has no -inf, which weigh nothing: with fewer tokens
        // all are kept)
        if (whole || binned || left < n) {
            kept.least = narrow(false, &left, [](uint32_t, uint32_t key, uint32_t* code) {
                *code = key;
                return true;
            });
            kept.until = kept.least == kLeast ? 0 : place(kept.least, left);
        }
    }
    if (by_p) {
        uint64_t inside = counts_all ? below : 0;
        each([&](uint32_t index, uint32_t key) {
            if (kept(key, index)) inside += weight_of(value_of(key), m, inverse);
        });
        const uint64_t total = all_above + block_sum<WAVES>(inside, lds.wave);
        const double need = ceil((double)p * (double)total);
        uint64_t left = need < 1.0 ? 1 : min((uint64_t)need, total);
        left = left > all_above ? left - all_above : 1;
        __syncthreads();
        const Kept k0 = kept;
        const uint32_t least = narrow(true, &left, [&](uint32_t index, uint32_t key, uint32_t* code) {
            *code = key;
            return k0(key, index);
        });
        const uint64_t w = weight_of(value_of(least), m, inverse);
        // (indices of the lowest are kept first in either filter)
        const uint32_t until = place(least, w ? (left + w - 1) / w : 1);
        kept = {least, least == k0.least ? min(until, k0.until) : until};
    }

    // what is kept of each wavefront's range
    if (tid < WAVES) lds.chunk[tid] = 0;
    __syncthreads();
    if (!whole) {
        if (tid < WAVES) atomicAdd((unsigned long long*)&lds.chunk[tid], (unsigned long long)lds.light[tid]);
        for (uint32_t e = tid; e < n; e += kThreads) {
            const uint32_t key = lds.key[e], index = lds.index[e];
            if (!kept(key, index)) continue;
            const uint64_t w = weight_of(value_of(key), m, inverse);
            if (w >= lightest) atomicAdd((unsigned long long*)&lds.chunk[index / (uint32_t)range], (unsigned long long)w);
        }
    } else {
        uint64_t sum = 0;
        each_of<DT>(x, i0, i1, [&](int32_t i, float f) {
            if (!kept(order_of(f), (uint32_t)i)) return;
            const uint64_t w = weight_of(f, m, inverse);
            sum += w >= lightest ? w : 0;
        });
        sum = wave_sum_u64(sum);
        if (lane == 0) lds.chunk[wave] = sum;
    }
    __syncthreads();
    uint64_t total = 0;
    for (int w = 0; w < WAVES; ++w) total += lds.chunk[w];
    const double at = floor((double)P.u[row] * (double)total);
    uint64_t r = at > 0.0 ? at < (double)total ? (uint64_t)at : total - 1 : 0;
    int hit = 0;
    while (hit < WAVES - 1 && r >= lds.chunk[hit]) r -= lds.chunk[hit++];

    // the range that it falls into, a stretch of it a thread
    const bool all_above_list = !binned && !listed && !whole;       // no filter
    const int32_t c0 = (int32_t)min((int64_t)hit * range, (int64_t)V), c1 = min(c0 + range, V);
    const int32_t stretch = (range + kThreads - 1) / kThreads;
    const int32_t t0 = min(c0 + tid * stretch, c1), t1 = min(t0 + stretch, c1);
    auto weight_at = [&](int32_t i, float f) -> uint64_t {
        const bool is_above = !whole && (all_above_list || (binned && bin(f) < low));
        if (!is_above && !kept(order_of(f), (uint32_t)i)) return 0;
        const uint64_t w = weight_of(f, m, inverse);
        return w >= lightest ? w : 0;
    };
    uint64_t sum = 0;
    for (int32_t i = t0; i < t1; ++i) sum += weight_at(i, logit<DT>(x[i]));
    const uint64_t incl = wave_incl_scan_u64(sum);
    if (lane == kWave - 1) lds.wave[wave] = incl;
    __syncthreads();
    uint64_t before = incl - sum;
    for (int w = 0; w < wave; ++w) before += lds.wave[w];
    if (r < before || r >= before + sum) return;    // (one thread goes on)
    for (int32_t i = t0; i < t1; ++i) {
        const float f = logit<DT>(x[i]);
        before += weight_at(i, f);
        if (before > r) {
            P.token[row] = i;
            if (P.logprob) P.logprob[row] = (float)(exponent(f, m, inverse) - log((double)total / kUnit));
            return;
        }
    }
}

template <int DT, int WAVES, int CAP>
hipError_t launch_waves(const SampleParams& p, hipStream_t stream) {
    return launch_all(p.n_rows, WAVES * kWave, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((sample_kernel<DT, WAVES, CAP>), grid, dim3(WAVES * kWave), 0, stream, p, first);
    });
}

template <int DT>
hipError_t launch_type(const SampleParams& p, hipStream_t stream) {
    if (p.n_cols <= 2048) return launch_waves<DT, 4, 2048>(p, stream);
    return launch_waves<DT, 16, 8192>(p, stream);
}

}  // namespace

hipError_t launch_sample(const SampleParams& p, hipStream_t stream) {
    if (p.dtype == TL_F32) return launch_type<TL_F32>(p, stream);
    return p.dtype == TL_F16 ? launch_type<TL_F16>(p, stream) : launch_type<TL_BF16>(p, stream);
}

}  // namespace tl
