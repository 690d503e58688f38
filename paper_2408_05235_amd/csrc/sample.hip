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
// Rows that one list of four wavefronts holds: 4096 rows of 2000 with top-p take 216 us so
// and 324 as longer ones do, 64 of them, which do not fill the card, 26 and 22.
constexpr int kShortRow = 2048;

template <int DT>
using elem = std::conditional_t<DT == TL_F32, float, uint16_t>;

template <int DT>
__device__ __forceinline__ float raw(elem<DT> x) {
    if constexpr (DT == TL_F32) return x;
    else if constexpr (DT == TL_F16) return (float)__builtin_bit_cast(_Float16, x);
    else return __builtin_bit_cast(float, (uint32_t)x << 16);
}

// A logit; NaN counts as -inf, and there is one zero.
__device__ __forceinline__ float clean(float f) { return f != f ? -INFINITY : f + 0.0f; }
template <int DT>
__device__ __forceinline__ float logit(elem<DT> x) { return clean(raw<DT>(x)); }

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

// rint(2^40 exp(e)) for e <= 0 by a table of 2^(j / 64) (P. T. P. Tang, "Table-driven
// implementation of the exponential function in IEEE floating-point arithmetic", 1989):
// e = n ln 2 / 64 + r, |r| < 0.0055, and five terms of exp(r), off by less than 2^-47
// of itself.  The sum with 2^52 rounds to a whole number, which the mantissa then is.
// (Half the instructions of the library's exponential, which sampling without filters
// is bound by: 256 rows of 128000 take 82 us with that and 69 so.)
struct Weights {
    const double* table;        // 2^(j / 64), in LDS
    double m, inverse;          // (of an infinite largest logit: 1e300 and 1)
    // (x may be a NaN or -inf: 0, as exp(-29) 2^40 < 1/2)
    __device__ __forceinline__ uint64_t operator()(float x) const {
        const double e = fmin(fmax(((double)x - m) * inverse, -29.0), 0.0);
        constexpr double kMagic = 0x1.8p52;
        const double t = fma(e, 92.332482616893656877, kMagic);    // 64 / ln 2
        const int32_t n = (int32_t)__builtin_bit_cast(uint64_t, t);
        const double r = fma(t - kMagic, -0.010830424696249145, e); // ln 2 / 64
        double y = fma(r, 1.0 / 120.0, 1.0 / 24.0);
        y = fma(y, r, 1.0 / 6.0);
        y = fma(y, r, 0.5);
        y = fma(y, r, 1.0);
        y = fma(y, r, 1.0);
        const uint64_t scaled = __builtin_bit_cast(uint64_t, y * table[n & 63]) + ((uint64_t)(uint32_t)((n >> 6) + 40) << 52);
        return __builtin_bit_cast(uint64_t, __builtin_bit_cast(double, scaled) + 0x1p52) & 0xfffffffffffffull;
    }
};

// How a row's elements are read: 16 bytes a lane, rows from any element on.
template <int DT>
struct Piece {
    static constexpr int kPer = DT == TL_F32 ? 4 : 8;
    typedef __attribute__((ext_vector_type(4))) uint32_t vec;
    // (a struct of its own: a template's argument loses what a typedef says of alignment)
    struct __attribute__((packed, aligned(sizeof(elem<DT>)))) Memory {
        vec v;
    };
    static_assert(alignof(Memory) == alignof(elem<DT>) && sizeof(Memory) == sizeof(vec));
    __device__ static __forceinline__ vec load(const elem<DT>* p) { return ((const Memory*)p)->v; }
    __device__ static __forceinline__ void split(vec v, float (&x)[kPer]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (a value of its own: a bit cast of a vector's element takes the first one)
            const uint32_t w = v[i];
            if constexpr (DT == TL_F32) {
                x[i] = __builtin_bit_cast(float, w);
            } else {
                x[2 * i] = raw<DT>((uint16_t)w);
                x[2 * i + 1] = raw<DT>((uint16_t)(w >> 16));
            }
        }
    }
};

// Elements that a workgroup reads in one go; f(index of the first, raw values) for the
// pieces of a row, in no order but a lane's indices ascend (-inf behind the row's end),
// done(chunk) behind each chunk.
template <int DT, int WAVES>
struct Chunks {
    using P = Piece<DT>;
    static constexpr int kPer = P::kPer, kBatch = DT == TL_F32 ? 4 : 2;
    static constexpr int kStep = WAVES * kWave * kPer, kSize = kBatch * kStep;
    template <class F, class Done>
    __device__ static __forceinline__ void each(const elem<DT>* x, int32_t V, F f, Done done) {
        int32_t i = (int32_t)threadIdx.x * kPer, chunk = 0;
        typename P::vec v[kBatch], next[kBatch];
        if (V >= kSize)
#pragma unroll
            for (int b = 0; b < kBatch; ++b) next[b] = P::load(x + i + b * kStep);
        for (; V - chunk * kSize >= kSize; ++chunk, i += kSize) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) v[b] = next[b];
            // (the next chunk is on its way under this one's work)
            if (V - chunk * kSize >= 2 * kSize)
#pragma unroll
                for (int b = 0; b < kBatch; ++b) next[b] = P::load(x + i + kSize + b * kStep);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                float y[kPer];
                P::split(v[b], y);
                f(i + b * kStep, y);
                __builtin_amdgcn_sched_barrier(0);      // (pieces one by one: they fill the registers)
            }
            done(chunk);
        }
        if (chunk * kSize >= V) return;
        pieces(x, i, V, f);
        done(chunk);
    }
    // A piece at a time, for what is rare: less code.
    template <class F>
    __device__ static __forceinline__ void pieces(const elem<DT>* x, int32_t i, int32_t end, F f) {
#pragma unroll 1
        for (; i < end; i += kStep) {
            float y[kPer];
            piece(x, i, end, y);
            f(i, y);
        }
    }
    __device__ static __forceinline__ void piece(const elem<DT>* x, int32_t i, int32_t end, float (&y)[kPer]) {
        if (end - i >= kPer) {
            P::split(P::load(x + i), y);
        } else {
#pragma unroll
            for (int e = 0; e < kPer; ++e) y[e] = i + e < end ? raw<DT>(x[i + e]) : -INFINITY;
        }
    }
};

// Bins of logits, from the top: 1 / kPerT of a temperature wide, the last one where all
// weights are 0 (30 temperatures below the largest: exp(-30) < 2^-41).
constexpr int kBins = 4096, kAboveBins = 2304;
constexpr float kPerT = 59.0f;
struct Binning {
    // (halves: a difference of two logits can be beyond fp32)
    float half_from, per_half, shift;       // finite, per_half > 0
    // The difference first, which is exact near `from`: by x times the scale, bins of logits
    // that are large for the temperature would be off by more than there are.
    __device__ __forceinline__ float place(float x) const {
        return fmaf(fmaf(x, -0.5f, half_from), per_half, shift);
    }
    // (monotone: each operation is; NaN goes to the last one, as -inf does)
    __device__ __forceinline__ float clamped(float x) const {
        return fmaxf(fminf(place(x), (float)(kBins - 1)), 0.0f);
    }
    __device__ __forceinline__ int operator()(float x) const { return (int)clamped(x); }
};

// WAVES wavefronts hold up to CAP tokens of a row in LDS, of the bins in which a
// threshold can be.
constexpr int kMostChunks = 512;        // of TL_MAX_COLUMNS
template <int WAVES, int CAP>
struct SampleLds {
    union {
        struct {
            uint32_t key[CAP], index[CAP];
        };
        uint64_t fine[kBins < CAP ? kBins : CAP];
    };
    uint32_t bins[kBins];
    uint64_t sums[256];
    uint32_t counts[256];
    uint64_t wave[WAVES], chunk[kMostChunks];
    double table[64];
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

// Bound by the round trips of few wavefronts (two a SIMD; with all filters they wait for 65%
// of their cycles, and vector instructions, the weights' in 64 bits most of all, take 20%).  256 rows of 128000 normal fp32 logits: the best token 27 us, without
// filters 70, top-k of 50 52, top-p of 0.9 95 us; 131 MB read once take 18.
//
// One workgroup a row.  The row is read twice and once in part: for its largest
// logit and the counts of its bins, which say where the thresholds of top-k and top-p
// can lie; then for the sums of what is surely kept (and, for top-p of all that weighs, of all), while
// the tokens of the bins between go to LDS, where the thresholds are found; and the
// chunk that the number falls into.  Where those bins hold too many tokens the
// thresholds are found by digits of the whole row's keys.
template <int DT, int WAVES, int CAP>
__global__ __launch_bounds__(WAVES * kWave) void sample_kernel(SampleParams P, int64_t first) {
    using Row = Chunks<DT, WAVES>;
    constexpr int kThreads = WAVES * kWave, kPer = Row::kPer;
    static_assert(CAP <= kShortRow || (int64_t)Row::kSize * kMostChunks >= TL_MAX_COLUMNS);
    __shared__ SampleLds<WAVES, CAP> lds;
    const int64_t row = blockIdx.x + first;
    const elem<DT>* const x = (const elem<DT>*)P.logits + row * P.stride;
    const int32_t V = P.n_cols;
    const int tid = threadIdx.x, wave = wave_number(), lane = lane_id();
    auto nothing = [](int32_t) {};
    if (tid < 64) lds.table[tid] = exp2((double)tid / 64.0);

    const float T = P.temperature ? P.temperature[row] : 1.0f;
    const bool draws = T > 0.0f;
    const int32_t k = draws && P.top_k ? P.top_k[row] : 0;
    const float p = draws && P.top_p ? P.top_p[row] : 1.0f;
    const bool by_k = k > 0 && k < V, by_p = p < 1.0f;
    const bool binned = V > CAP && (by_k || by_p);

    // the largest logit, and its first place: its key above the place's complement;
    // the counts of the bins (without them all finite logits go to the list)
    uint64_t top = 0;
    Binning bin = {0.0f, 2e-38f, (float)kAboveBins};     // (a few bins, and the last one)
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
        const float per = fminf(fmaxf(kPerT / T, 1e-37f), 1e30f), from = fminf(fmaxf(m0, -3e38f), 3e38f);
        bin = {0.5f * from, 2.0f * per, (float)kAboveBins};
    }
    {
        float m1 = -INFINITY, m2 = -INFINITY;       // a lane's largest, and of the chunk
        int32_t chunk_of = 0;
        auto largest = [&](int32_t chunk) {
            if (m2 > m1) m1 = m2, chunk_of = chunk;
            m2 = -INFINITY;
        };
        if (!binned)
            Row::each(x, V, [&](int32_t, const float (&y)[kPer]) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) m2 = fmaxf(m2, y[e]);
            }, largest);
        else
            Row::each(x, V, [&](int32_t, const float (&y)[kPer]) {
                int b[kPer];
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    m2 = fmaxf(m2, y[e]);
                    b[e] = bin(y[e]);
                }
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (b[e] < kBins - 1) atomicAdd(&lds.bins[b[e]], 1u);
            }, largest);
        // its first place, which only the best token needs, is looked for again in its chunk
        const float f = clean(m1);
        int32_t at = 0;
        if (!draws && f > -INFINITY) {
            at = V;
            const int32_t from = chunk_of * Row::kSize + tid * kPer;
#pragma unroll
            for (int b = Row::kBatch - 1; b >= 0; --b) {
                float y[kPer];
                Row::piece(x, from + b * Row::kStep, V, y);
#pragma unroll
                for (int e = kPer - 1; e >= 0; --e)
                    if (y[e] == f) at = from + b * Row::kStep + e;
            }
        }
        top = (uint64_t)order_of(f) << 32 | (uint32_t)~at;
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
    const Weights weight_of = {lds.table, m < INFINITY ? (double)m : 1e300, m < INFINITY ? inverse : 1.0};
    const float q = P.min_p ? P.min_p[row] : 0.0f;
    // the least key that min-p keeps: weights grow with the keys; 64 of them at a time
    uint32_t least_key = 0;
    if (q > 0.0f) {
        const uint64_t lightest = (uint64_t)ceil((double)fminf(q, 1.0f) * kUnit);
        uint32_t lo = kLeast, hi = most;            // lo is too light, hi is not
        __syncthreads();                            // (the table)
        while (hi - lo > 1) {
            const uint32_t step = (hi - lo + kWave - 1) / kWave, key = lo + min((lane + 1) * step, hi - lo);
            const uint64_t heavy = __ballot(weight_of(value_of(key)) >= lightest);
            const int first = __builtin_ctzll(heavy);
            hi = lo + min((first + 1) * step, hi - lo);
            lo += first * step;
        }
        least_key = hi;
    }
    const float least_logit = least_key ? value_of(least_key) : -INFINITY;

    // the bins that go to LDS: [low, high] (those above are kept, those below not)
    bool listed = by_k || by_p, counts_all = by_p && !by_k, limited = by_k;
    int32_t low = 0, high = kBins - 2;              // (the last bin has -inf, and what weighs nothing)
    uint64_t rank = (uint64_t)max(k, 0);            // of the last one kept by top-k, among those listed
    bool fine = false;                              // more tokens than the list takes
    if (!listed) low = kBins;
    if (CAP > kShortRow && binned) {
        // each lane has kPerLane bins: counts in them and before them, and what they weigh
        // about: count times the weight of the middle, which is off by half a percent (a
        // bin's width / sqrt(12)) for one token and by the root of the count less for many.
        // The bins in which top-p's threshold lies are taken from this with five times the
        // error and 1e-4 to spare; the exact sums then say whether it does.
        constexpr int kPerLane = kBins / kThreads;
        uint32_t count[kPerLane], own = 0;
        float about[kPerLane], own_sum = 0.0f, square = 0.0f;
        const float place_of_most = bin.place(m);
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) {
            const int b = tid * kPerLane + e;
            count[e] = lds.bins[b];
            own += count[e];
            const float w = __expf(fminf((place_of_most - (float)b - 0.5f) / kPerT, 0.0f));
            about[e] = (float)count[e] * w;
            own_sum += about[e];
            square = fmaf(about[e], w, square);
        }
        uint32_t c = (uint32_t)wave_incl_scan((int32_t)own);
        float sum = own_sum;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const float a = __shfl_up(sum, o);
            if (lane >= o) sum += a;
            square += __shfl_xor(square, o);
        }
        __syncthreads();
        if (lane == kWave - 1) {
            lds.wave_count[wave] = c;
            lds.wave_low[wave] = sum;
            lds.wave_high[wave] = square;
        }
        if (tid == 0) lds.low = lds.high = kBins - 2, lds.found[0] = lds.found[1] = 0;
        __syncthreads();
        float all_sum = 0.0f, all_square = 0.0f;
        uint32_t all = 0;
        c -= own;
        sum -= own_sum;
        for (int w = 0; w < WAVES; ++w) {
            if (w == wave) c += all, sum += all_sum;
            all += lds.wave_count[w];
            all_sum += lds.wave_low[w];
            all_square += lds.wave_high[w];
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
            limited = false;                        // (all with a weight: top-p counts the row's)
            counts_all = by_p;
            if (by_p) {
                const float reach = p * all_sum, error = 5.0f * 0.29f / kPerT * sqrtf(all_square) + 1e-4f * all_sum;
                int32_t mine_low = kBins - 2, mine_high = kBins - 2;
#pragma unroll
                for (int e = kPerLane - 1; e >= 0; --e) {
                    float upto = sum;
#pragma unroll
                    for (int y = 0; y <= e; ++y) upto += about[y];
                    if (upto >= reach - error) mine_low = tid * kPerLane + e;
                    if (upto >= reach + error) mine_high = tid * kPerLane + e;
                }
                atomicMin(&lds.low, mine_low);
                atomicMin(&lds.high, mine_high);
                __syncthreads();
                low = min(lds.low, lds.high);
                high = lds.high;
                uint32_t in = 0;
#pragma unroll
                for (int e = 0; e < kPerLane; ++e) {
                    const int b = tid * kPerLane + e;
                    if (b >= low && b <= high) in += count[e];
                }
                fine = block_sum<WAVES>(in, lds.wave) > CAP;
            } else {
                listed = false;                     // nothing to find: all are kept
                low = kBins;
            }
        }
    }
    bool whole = !listed && low < kBins;            // thresholds from the row itself

    // Many tokens where top-p's threshold lies: their exact sums in finer bins there (0:
    // what is above, the last one: what is below) say which one it is.
    uint64_t of_p = 0;                              // what top-p has to reach, if known
    if (CAP > kShortRow && fine) {
        const float finer = (float)(kBins - 2) / (float)(high - low + 1);
        bin = {bin.half_from, bin.per_half * finer, fmaf(bin.shift - (float)low, finer, 1.0f)};
        for (int e = tid; e < kBins; e += kThreads) lds.fine[e] = 0;
        __syncthreads();
        uint64_t over = 0, under = 0;
        Row::each(x, V, [&](int32_t, const float (&y)[kPer]) {
#pragma unroll
            for (int e0 = 0; e0 < kPer; e0 += 4) {
                uint64_t w[4];
                int b[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] = weight_of(y[e0 + e]);
                    b[e] = bin(y[e0 + e]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    over += b[e] == 0 ? w[e] : 0;
                    under += b[e] == kBins - 1 ? w[e] : 0;
                    if (b[e] > 0 && b[e] < kBins - 1)
                        atomicAdd((unsigned long long*)&lds.fine[b[e]], (unsigned long long)w[e]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }, nothing);
        over = block_sum<WAVES>(over, lds.wave);
        under = block_sum<WAVES>(under, lds.wave);
        __syncthreads();
        constexpr int kPerLane = kBins / kThreads;
        uint64_t sums[kPerLane], own = 0;
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) own += sums[e] = lds.fine[tid * kPerLane + e];
        const uint64_t inside = block_sum<WAVES>(own, lds.wave), total = over + inside + under;
        uint64_t before = wave_incl_scan_u64(own);
        __syncthreads();
        if (lane == kWave - 1) lds.wave[wave] = before;
        if (tid == 0) lds.low = 0;
        __syncthreads();
        before += over - own;
        for (int w = 0; w < wave; ++w) before += lds.wave[w];
        const double need = ceil((double)p * (double)total);
        of_p = need < 1.0 ? 1 : min((uint64_t)need, total);
#pragma unroll
        for (int e = 0; e < kPerLane; ++e) {
            if (before < of_p && before + sums[e] >= of_p) lds.low = tid * kPerLane + e;
            before += sums[e];
        }
        __syncthreads();
        low = high = lds.low;
        counts_all = false;
        if (low == 0) whole = true;                 // (the estimate was wrong)
        __syncthreads();
    }

    // sums of what is kept above the list, by chunk, and of all; the list
    if (tid == 0) lds.n = 0;
    for (int e = tid; e < kMostChunks; e += kThreads) lds.chunk[e] = 0;
    __syncthreads();
    uint64_t above = 0, light = 0, every = 0;
    if (!whole) {
        const float low_place = (float)low, end_place = (float)(high + 1);
        auto list = [&](int32_t i, float f, float place) {
            if (place < low_place || place >= end_place) return;
            const uint32_t at = atomicAdd(&lds.n, 1u);
            if (at < CAP) {
                lds.key[at] = order_of(f + 0.0f);
                lds.index[at] = (uint32_t)i;
            }
        };
        if (low == 0 && !counts_all)                // only the list counts
            Row::each(x, V, [&](int32_t i, const float (&y)[kPer]) {
                float place[kPer];
#pragma unroll
                for (int e = 0; e < kPer; ++e) place[e] = bin.clamped(y[e]);
#pragma unroll
                for (int e = 0; e < kPer; ++e) list(i + e, y[e], place[e]);
            }, nothing);
        else
            Row::each(x, V, [&](int32_t i, const float (&y)[kPer]) {
                float place[kPer];
#pragma unroll
                for (int e0 = 0; e0 < kPer; e0 += 4) {
                    uint64_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[e] = weight_of(y[e0 + e]);
                        place[e0 + e] = bin.clamped(y[e0 + e]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t over = place[e0 + e] < low_place ? w[e] : 0;
                        every += w[e];
                        above += over;
                        light += y[e0 + e] >= least_logit ? over : 0;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (low < kBins)
#pragma unroll
                    for (int e = 0; e < kPer; ++e) list(i + e, y[e], place[e]);
            }, [&](int32_t chunk) {
                light = wave_sum_u64(light);
                if (lane == 0) atomicAdd((unsigned long long*)&lds.chunk[chunk], (unsigned long long)light);
                light = 0;
            });
    }
    const uint64_t all_above = block_sum<WAVES>(above, lds.wave);
    const uint32_t n = min(lds.n, (uint32_t)CAP);
    if (lds.n > CAP) whole = true;

    // f(index, key) of the list, or of the row
    auto each = [&](auto f) __attribute__((always_inline)) {
        if (whole)
            Row::pieces(x, tid * kPer, V, [&](int32_t i, const float (&y)[kPer]) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) f((uint32_t)(i + e), order_of(clean(y[e])));
            });
        else
            for (uint32_t e = tid; e < n; e += kThreads) f(lds.index[e], lds.key[e]);
    };
    // The thresholds, each as the `left`-th largest code of some tokens, by count or by
    // weight, by digits of 8 bits from the highest bit in which the codes differ: top-k's
    // key, up to which index tokens that equal it are kept, and the same for top-p.  (A
    // loop, so that its code is there once.)
    Kept kept = {kLeast, 0};
    uint32_t equal = 0;                     // the key whose places are looked for
    uint64_t left = 0;
#pragma unroll 1
    for (int stage = 0; stage < 4; ++stage) {
        const bool places = stage & 1, by_weight = stage == 2;
        if (stage == 0) {
            // (a list of the whole row has no -inf, which weigh nothing: with fewer tokens
            // all are kept)
            left = whole ? (uint64_t)k : rank;
            if (!limited || !(whole || binned || left < n)) {
                ++stage;
                continue;
            }
        }
        if (stage == 2) {
            if (!by_p) break;
            uint64_t inside = 0;
            each([&](uint32_t index, uint32_t key) {
                if (kept(key, index)) inside += weight_of(value_of(key));
            });
            inside = block_sum<WAVES>(inside, lds.wave);
            const uint64_t total = !whole && counts_all ? block_sum<WAVES>(every, lds.wave) : inside;
            const double need = ceil((double)p * (double)total);
            left = need < 1.0 ? 1 : min((uint64_t)need, total);
            if (fine) left = of_p;
            if (!whole) {
                if (left <= all_above || left > all_above + inside) {
                    // (the estimate was wrong: again, with the whole row's sum)
                    whole = true;
                    --stage;
                    continue;
                }
                left -= all_above;
            }
        }
        auto code_of = [&](uint32_t index, uint32_t key, uint32_t* code) {
            *code = places ? ~index : key;
            return places ? key == equal : stage == 0 || kept(key, index);
        };
        uint32_t lo = ~0u, hi = 0;
        each([&](uint32_t index, uint32_t key) {
            uint32_t code;
            if (!code_of(index, key, &code)) return;
            lo = min(lo, code);
            hi = max(hi, code);
        });
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            lo = min(lo, (uint32_t)__shfl_xor((int)lo, o));
            hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
        }
        __syncthreads();
        if (lane == 0) lds.wave[wave] = (uint64_t)hi << 32 | lo;
        __syncthreads();
        for (int w = 0; w < WAVES; ++w) {
            lo = min(lo, (uint32_t)lds.wave[w]);
            hi = max(hi, (uint32_t)(lds.wave[w] >> 32));
        }
        int bits = lo >= hi ? 0 : 32 - __builtin_clz(lo ^ hi);
        uint32_t mask = bits >= 32 ? 0 : ~0u << bits, found = hi & mask, tokens = 0;
#pragma unroll 1
        do {
            const int take = min(bits, 8), shift = bits - take;
            const uint32_t digits = (1u << take) - 1;
            for (int e = tid; e < 256; e += kThreads) {
                lds.sums[e] = 0;
                lds.counts[e] = 0;
            }
            __syncthreads();
            each([&](uint32_t index, uint32_t key) {
                uint32_t code;
                if (!code_of(index, key, &code) || (code & mask) != found) return;
                const uint64_t one = by_weight ? weight_of(value_of(key)) : 1;
                atomicAdd((unsigned long long*)&lds.sums[code >> shift & digits], (unsigned long long)one);
                atomicAdd(&lds.counts[code >> shift & digits], 1u);
            });
            __syncthreads();
            if (wave == 0) {
                // lane l has the digits 255 - 4 l .. 252 - 4 l
                uint64_t d[4], sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    d[e] = lds.sums[255 - 4 * lane - e];
                    sum += d[e];
                }
                uint64_t at = wave_incl_scan_u64(sum) - sum;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (at < left && at + d[e] >= left) {
                        lds.found[0] = (uint64_t)(255 - 4 * lane - e);
                        lds.found[1] = left - at;
                    }
                    at += d[e];
                }
            }
            __syncthreads();
            const uint32_t digit = (uint32_t)lds.found[0] & digits;
            found |= digit << shift;
            mask |= digits << shift;
            left = lds.found[1];
            tokens = lds.counts[digit];
            bits = shift;
            __syncthreads();
        } while (bits > 0);
        if (places) {
            // (of equal ones those that top-k keeps are the first, and so are top-p's)
            kept.until = min(kept.until, ~found);
            continue;
        }
        const uint64_t w = by_weight ? weight_of(value_of(found)) : 1;
        const uint64_t ties = w ? (left + w - 1) / w : 1;
        if (found != kept.least) kept.until = ~0u;
        kept.least = equal = found;
        left = ties;
        if (found == kLeast) kept.until = 0;
        // (top-p's count what top-k keeps: as many or fewer than there are)
        if (ties >= tokens || found == kLeast) ++stage;
    }

    // what is kept of each chunk
    if (least_key > kept.least) kept = {least_key, ~0u};
    __syncthreads();
    if (!whole) {
        for (uint32_t e = tid; e < n; e += kThreads) {
            const uint32_t key = lds.key[e], index = lds.index[e];
            if (!kept(key, index)) continue;
            atomicAdd((unsigned long long*)&lds.chunk[index / (uint32_t)Row::kSize],
                      (unsigned long long)weight_of(value_of(key)));
        }
    } else {
        for (int e = tid; e < kMostChunks; e += kThreads) lds.chunk[e] = 0;
        __syncthreads();
        uint64_t sum = 0;
#pragma unroll 1
        for (int32_t chunk = 0; chunk * Row::kSize < V; ++chunk) {
            const int32_t from = chunk * Row::kSize;
            Row::pieces(x, from + tid * kPer, V - from < Row::kSize ? V : from + Row::kSize,
                        [&](int32_t i, const float (&y)[kPer]) {
#pragma unroll
                            for (int e = 0; e < kPer; ++e)
                                if (kept(order_of(clean(y[e])), (uint32_t)(i + e))) sum += weight_of(y[e]);
                        });
            sum = wave_sum_u64(sum);
            if (lane == 0) atomicAdd((unsigned long long*)&lds.chunk[chunk], (unsigned long long)sum);
            sum = 0;
        }
    }
    __syncthreads();
    const int chunks = (V + Row::kSize - 1) / Row::kSize;
    uint64_t total = 0;
    for (int w = 0; w < chunks; ++w) total += lds.chunk[w];
    const double at = floor((double)P.u[row] * (double)total);
    uint64_t r = at > 0.0 ? at < (double)total ? (uint64_t)at : total - 1 : 0;
    int hit = 0;
    while (hit < chunks - 1 && r >= lds.chunk[hit]) r -= lds.chunk[hit++];

    // the chunk that it falls into, a stretch of it a thread
    constexpr int kStretch = Row::kSize / kThreads;
    const int32_t t0 = hit * Row::kSize + tid * kStretch;
    float y[Row::kBatch][kPer];
#pragma unroll
    for (int b = 0; b < Row::kBatch; ++b) Row::piece(x, t0 + b * kPer, V, y[b]);
    uint64_t w[kStretch], sum = 0;
#pragma unroll
    for (int e = 0; e < kStretch; ++e) {
        const float f = clean(y[e / kPer][e % kPer]);
        const uint32_t key = order_of(f);
        const bool is_above = !whole && bin(f) < low;
        w[e] = (is_above ? key >= least_key : kept(key, (uint32_t)(t0 + e))) ? weight_of(f) : 0;
        sum += w[e];
        if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    const uint64_t incl = wave_incl_scan_u64(sum);
    if (lane == kWave - 1) lds.wave[wave] = incl;
    __syncthreads();
    uint64_t before = incl - sum;
    for (int w = 0; w < wave; ++w) before += lds.wave[w];
    if (r < before || r >= before + sum) return;    // (one thread goes on)
    int32_t token = -1;
    float f = 0.0f;
#pragma unroll
    for (int e = 0; e < kStretch; ++e) {
        before += w[e];
        if (token < 0 && before > r) {
            token = t0 + e;
            f = clean(y[e / kPer][e % kPer]);
        }
    }
    P.token[row] = token;
    if (P.logprob) P.logprob[row] = (float)(exponent(f, m, inverse) - log((double)total / kUnit));
}

template <int DT, int WAVES, int CAP>
hipError_t launch_waves(const SampleParams& p, hipStream_t stream) {
    return launch_all(p.n_rows, WAVES * kWave, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((sample_kernel<DT, WAVES, CAP>), grid, dim3(WAVES * kWave), 0, stream, p, first);
    });
}

template <int DT>
hipError_t launch_type(const SampleParams& p, hipStream_t stream) {
    if (p.n_cols <= kShortRow) return launch_waves<DT, 4, kShortRow>(p, stream);
    return launch_waves<DT, 8, 7168>(p, stream);
}

}  // namespace

hipError_t launch_sample(const SampleParams& p, hipStream_t stream) {
    if (p.dtype == TL_F32) return launch_type<TL_F32>(p, stream);
    return p.dtype == TL_F16 ? launch_type<TL_F16>(p, stream) : launch_type<TL_BF16>(p, stream);
}

}  // namespace tl
