// The norm before a product (tl_norm): y = h * (1 / sqrt(mean h^2 + eps)) * w for
// h = x (+ residual), in the inputs' type or in e4m3 with scales.
//
// 64 rows of 4096 take 4.0 us, a launch and its round trips; 16384 of 8192 with a
// residual to e4m3 (944 MB) 163 us, 5.8 TB/s.
// Bound by memory: each input is read once and each output written once, so a
// row stays in registers between its sum of squares and its output (norm_kernel),
// as long as 1024 threads hold it; longer ones are read twice (norm_long_kernel).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "device_util.h"
#include "step.h"
#include "tl.h"
#include "tl_internal.h"

namespace tl {
namespace {

constexpr int kPer = 8;                 // columns of a lane's piece
constexpr float kMostE4m3 = 448.0f;
constexpr float kLeastScale = 0x1p-100f;

// Rows begin at any element: pieces are read and written at that alignment
// (which the memory units take; a piece of 16 bytes is one instruction all the same).
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t piece16;
typedef __attribute__((ext_vector_type(4), aligned(4))) uint32_t piece32;
typedef __attribute__((ext_vector_type(2), aligned(1))) uint32_t piece8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

template <int DT>
using elem = std::conditional_t<DT == TL_F32, float, uint16_t>;

template <int DT>
__device__ __forceinline__ float to_f32(elem<DT> x) {
    if constexpr (DT == TL_F32) return x;
    else if constexpr (DT == TL_F16) return (float)__builtin_bit_cast(_Float16, x);
    else return __builtin_bit_cast(float, (uint32_t)x << 16);
}

template <int DT>
__device__ __forceinline__ elem<DT> round_to(float x) {
    if constexpr (DT == TL_F32) return x;
    else if constexpr (DT == TL_F16) return __builtin_bit_cast(uint16_t, (_Float16)x);
    else return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// A piece as it lies in memory, n (1 .. 8) columns; the others are 0.
template <int DT>
struct Raw {
    uint32_t v[DT == TL_F32 ? 8 : 4];
};
// ONCE: nobody reads it again, and it does not have to take others' place in the caches.
template <int DT, bool ONCE>
__device__ __forceinline__ Raw<DT> load_raw(const elem<DT>* p, int n) {
    Raw<DT> r;
    if (n == kPer) {
        if constexpr (DT == TL_F32) {
            const piece32 a = ONCE ? __builtin_nontemporal_load((const piece32*)p) : *(const piece32*)p;
            const piece32 b = ONCE ? __builtin_nontemporal_load((const piece32*)(p + 4)) : *(const piece32*)(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r.v[i] = a[i];
                r.v[4 + i] = b[i];
            }
        } else {
            const piece16 a = ONCE ? __builtin_nontemporal_load((const piece16*)p) : *(const piece16*)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) r.v[i] = a[i];
        }
        return r;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if constexpr (DT == TL_F32) {
            r.v[i] = i < n ? __builtin_bit_cast(uint32_t, p[i]) : 0;
        } else {
            const uint32_t x = i < n ? p[i] : 0;
            r.v[i / 2] = i % 2 ? r.v[i / 2] | x << 16 : x;
        }
    }
    return r;
}
template <int DT>
__device__ __forceinline__ void expand(const Raw<DT>& r, float (&x)[kPer]) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if constexpr (DT == TL_F32) x[i] = __builtin_bit_cast(float, r.v[i]);
        else x[i] = to_f32<DT>((uint16_t)(r.v[i / 2] >> (16 * (i % 2))));
    }
}
template <int DT, bool ONCE = false>
__device__ __forceinline__ void load_piece(const elem<DT>* p, int n, float (&x)[kPer]) {
    expand<DT>(load_raw<DT, ONCE>(p, n), x);
}

// (ALIGN bytes: of a template's argument a typedef's alignment would be lost.  Through the
// caches: past them 16384 rows of 8192 take as long, 163 us in e4m3 and 181 in bf16.)
template <int ALIGN, class V>
__device__ __forceinline__ void store(V v, void* to) {
    typedef V there __attribute__((aligned(ALIGN)));
    *(there*)to = v;
}

template <int DT>
__device__ __forceinline__ void store_piece(elem<DT>* p, int n, const float (&x)[kPer]) {
    if (n == kPer) {
        if constexpr (DT == TL_F32) {
            piece32 a, b;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = __builtin_bit_cast(uint32_t, x[i]);
                b[i] = __builtin_bit_cast(uint32_t, x[4 + i]);
            }
            store<4>(a, p);
            store<4>(b, p + 4);
        } else {
            piece16 a;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (DT == TL_F16)
                    a[i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x[2 * i], (_Float16)x[2 * i + 1]});
                else a[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
            }
            store<2>(a, p);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < n) p[i] = round_to<DT>(x[i]);
}

// Division by a scale s: the product with 1 / s, corrected by what it leaves of y, which
// is the quotient rounded once (P. Markstein, "Computation of elementary functions on the
// IBM RISC System/6000 processor", 1990; 1 / s is rounded correctly).  By an infinite s
// the product alone: 0, or NaN.
struct Scale {
    float value, inverse;
    __device__ __forceinline__ explicit Scale(float s) : value(s == INFINITY ? 0.0f : s), inverse(1.0f / s) {}
    __device__ __forceinline__ float quotient(float y) const {
        const float q = y * inverse;
        return fmaf(fmaf(-q, value, y), inverse, q);
    }
};

// y / s to e4m3: nearest even, NaN stays NaN.  (The largest value of a scale is
// 448 times it up to a rounding, hence the clamp.)
__device__ __forceinline__ void store_e4m3(uint8_t* p, int n, const float (&y)[kPer], Scale s) {
    float z[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const float t = s.quotient(y[i]);
        z[i] = t != t ? t : fminf(fmaxf(t, -kMostE4m3), kMostE4m3);
    }
    piece8 q;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * i], z[4 * i + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * i + 2], z[4 * i + 3], w, true);
        q[i] = (uint32_t)w;
    }
    if (n == kPer) {
        store<1>(q, p);
        return;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (i < n) p[i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
}

// The largest absolute value by its bits: a NaN is larger than all others and
// is what comes out.
__device__ __forceinline__ uint32_t max_abs(const float (&y)[kPer], uint32_t m) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) m = max(m, __builtin_bit_cast(uint32_t, y[i]) & 0x7fffffffu);
    return m;
}

__device__ __forceinline__ float scale_of(uint32_t most) {
    const float s = __builtin_bit_cast(float, most) / kMostE4m3;
    return s < kLeastScale ? kLeastScale : s;       // (NaN stays)
}

// A row's threads: THREADS consecutive ones, whole wavefronts.
template <int THREADS>
struct Reduce {
    static constexpr int kWaves = THREADS / kWave;
    float* sums;            // of the row's wavefronts, in LDS
    uint32_t* mosts;
    __device__ __forceinline__ float sum(float v) const {
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
        if constexpr (kWaves == 1) return v;
        if (lane_id() == 0) sums[threadIdx.x % THREADS / kWave] = v;
        __syncthreads();
        v = sums[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += sums[w];
        return v;
    }
    __device__ __forceinline__ uint32_t most(uint32_t v) const {
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
        if constexpr (kWaves == 1) return v;
        if (lane_id() == 0) mosts[threadIdx.x % THREADS / kWave] = v;
        __syncthreads();
        v = mosts[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v = max(v, mosts[w]);
        return v;
    }
};

// The largest of `group` / 8 consecutive lanes (2 .. 64, a power of two).
__device__ __forceinline__ uint32_t group_most(uint32_t v, int lanes) {
    for (int o = 1; o < lanes; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
    return v;
}

enum { kSame, kRowScale, kGroupScale };

// What is behind a row's end has no say in a scale: where the root is infinite it would be
// NaN (0 x inf).  (Without a branch around it: 16384 rows of 8192 take 155 us, 157 with one.)
__device__ __forceinline__ void none_behind(float (&y)[kPer], int n) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) y[i] = i < n ? y[i] : 0.0f;
}

__device__ __forceinline__ float inverse_root(float squares, const NormParams& P) {
    return 1.0f / sqrtf(squares / (float)P.n_cols + P.eps);
}

// THREADS threads hold a row, CH pieces of 8 columns each.
template <int DT, int OUT, int CH, int THREADS, bool RES>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_kernel(NormParams P, int64_t first) {
    constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kRows = kBlock / THREADS;
    __shared__ float sums[kRows][THREADS / kWave];
    __shared__ uint32_t mosts[kRows][THREADS / kWave];
    const int r = threadIdx.x / THREADS, t = threadIdx.x % THREADS;
    const int64_t at = (blockIdx.x + first) * kRows + r;
    const int64_t row = min(at, P.n_rows - 1);      // (rows behind the last one compute it again and write nothing)
    const bool real = at < P.n_rows;
    const Reduce<THREADS> reduce = {sums[r], mosts[r]};
    const int W = P.n_cols;
    const elem<DT>* const x = (const elem<DT>*)P.x + row * P.x_stride;
    const elem<DT>* const res = (const elem<DT>*)P.residual + row * P.residual_stride;
    const elem<DT>* const weight = (const elem<DT>*)P.weight;
    float h[CH][kPer];
    Raw<DT> w[CH];                                  // (as it lies: half the registers in 16 bits)
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * THREADS + t) * kPer, n = min(W - col, kPer);
#pragma unroll
        for (int i = 0; i < kPer; ++i) h[c][i] = 0.0f;
        w[c] = Raw<DT>{};
        if (n > 0) {
            load_piece<DT, true>(x + col, n, h[c]);
            if constexpr (RES) {
                float y[kPer];
                load_piece<DT, true>(res + col, n, y);
#pragma unroll
                for (int i = 0; i < kPer; ++i) h[c][i] += y[i];
            }
            w[c] = load_raw<DT, false>(weight + col, n);
        }
    }
    float squares = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < kPer; ++i) squares = fmaf(h[c][i], h[c][i], squares);
    const float f = inverse_root(reduce.sum(squares), P);
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * THREADS + t) * kPer, n = min(W - col, kPer);
        if constexpr (RES)
            if (real && n > 0 && P.sum) store_piece<DT>((elem<DT>*)P.sum + row * W + col, n, h[c]);
        float y[kPer];
        expand<DT>(w[c], y);
#pragma unroll
        for (int i = 0; i < kPer; ++i) h[c][i] = h[c][i] * f * y[i];
        if constexpr (OUT != kSame) none_behind(h[c], n);
        if constexpr (OUT == kSame) {
            if (real && n > 0) store_piece<DT>((elem<DT>*)P.out + row * W + col, n, h[c]);
        } else if constexpr (OUT == kRowScale) {
            most = max_abs(h[c], most);
        } else {
            const float s = scale_of(group_most(max_abs(h[c], 0), P.group / kPer));
            if (real && n > 0) {
                store_e4m3((uint8_t*)P.out + row * W + col, n, h[c], Scale(s));
                if (col % P.group == 0) P.scale[row * ((W + P.group - 1) / P.group) + col / P.group] = s;
            }
        }
    }
    if constexpr (OUT == kRowScale) {
        const float s = scale_of(reduce.most(most));
        const Scale by(s);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * THREADS + t) * kPer, n = min(W - col, kPer);
            if (real && n > 0) store_e4m3((uint8_t*)P.out + row * W + col, n, h[c], by);
        }
        if (real && t == 0) P.scale[row] = s;
    }
}

// A row of any length, read twice (thrice where its largest value is needed
// first).  Each thread writes only what it alone reads, after its last read, so
// that outputs may be inputs.
template <int DT, int OUT>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormParams P, int64_t first) {
    __shared__ float sums[1024 / kWave];
    __shared__ uint32_t mosts[1024 / kWave];
    const Reduce<1024> reduce = {sums, mosts};
    const int64_t row = blockIdx.x + first;
    const int64_t W = P.n_cols;
    const elem<DT>* const x = (const elem<DT>*)P.x + row * P.x_stride;
    const elem<DT>* const res = P.residual ? (const elem<DT>*)P.residual + row * P.residual_stride : nullptr;
    const elem<DT>* const weight = (const elem<DT>*)P.weight;
    auto load = [&](int64_t col, int n, float (&h)[kPer]) {
        load_piece<DT>(x + col, n, h);
        if (res) {
            float y[kPer];
            load_piece<DT>(res + col, n, y);
#pragma unroll
            for (int i = 0; i < kPer; ++i) h[i] += y[i];
        }
    };
    float squares = 0.0f;
    for (int64_t col = threadIdx.x * kPer; col < W; col += 1024 * kPer) {
        float h[kPer], part = 0.0f;
        load(col, (int)min(W - col, (int64_t)kPer), h);
#pragma unroll
        for (int i = 0; i < kPer; ++i) part = fmaf(h[i], h[i], part);
        squares += part;
    }
    const float f = inverse_root(reduce.sum(squares), P);
    auto normed = [&](int64_t col, int n, float (&h)[kPer]) {
        float w[kPer];
        load_piece<DT>(weight + col, n, w);
#pragma unroll
        for (int i = 0; i < kPer; ++i) h[i] = h[i] * f * w[i];
        if constexpr (OUT != kSame) none_behind(h, n);
    };
    float s = 0.0f;
    if constexpr (OUT == kRowScale) {
        uint32_t most = 0;
        for (int64_t col = threadIdx.x * kPer; col < W; col += 1024 * kPer) {
            const int n = (int)min(W - col, (int64_t)kPer);
            float h[kPer];
            load(col, n, h);
            normed(col, n, h);
            most = max_abs(h, most);
        }
        s = scale_of(reduce.most(most));
        if (threadIdx.x == 0) P.scale[row] = s;
    }
    // (whole wavefronts go on together: the groups' lanes look at each other)
    for (int64_t c0 = 0; c0 < W; c0 += 1024 * kPer) {
        const int64_t col = c0 + threadIdx.x * kPer;
        const int n = (int)max(min(W - col, (int64_t)kPer), (int64_t)0);
        float h[kPer] = {};
        if (n > 0) {
            load(col, n, h);
            if (P.sum) store_piece<DT>((elem<DT>*)P.sum + row * W + col, n, h);
            normed(col, n, h);
        }
        if constexpr (OUT == kSame) {
            if (n > 0) store_piece<DT>((elem<DT>*)P.out + row * W + col, n, h);
        } else {
            if constexpr (OUT == kGroupScale) s = scale_of(group_most(max_abs(h, 0), P.group / kPer));
            if (n > 0) {
                store_e4m3((uint8_t*)P.out + row * W + col, n, h, Scale(s));
                if constexpr (OUT == kGroupScale)
                    if (col % P.group == 0) P.scale[row * ((W + P.group - 1) / P.group) + col / P.group] = s;
            }
        }
    }
}

template <int DT, int OUT, int CH, int THREADS>
hipError_t launch_row(const NormParams& p, hipStream_t stream) {
    constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kRows = kBlock / THREADS;
    return launch_all((p.n_rows + kRows - 1) / kRows, kBlock, [&](dim3 grid, int64_t first) {
        if (p.residual) hipLaunchKernelGGL((norm_kernel<DT, OUT, CH, THREADS, true>), grid, dim3(kBlock), 0, stream, p, first);
        else hipLaunchKernelGGL((norm_kernel<DT, OUT, CH, THREADS, false>), grid, dim3(kBlock), 0, stream, p, first);
    });
}

template <int DT, int OUT>
hipError_t launch_out(const NormParams& p, hipStream_t stream) {
    // (64 rows of 8192 take 3.3 us with 512 threads, 4.1 with 256, and 16384 of them with
    // a residual to e4m3 173 and 177; 1999 of 5000 take 8.7 with 256 threads, 10.6 with 512)
    const int pieces = (int)(((int64_t)p.n_cols + kPer - 1) / kPer);
    if (pieces <= 64) return launch_row<DT, OUT, 1, 64>(p, stream);
    if (pieces <= 128) return launch_row<DT, OUT, 1, 128>(p, stream);
    if (pieces <= 256) return launch_row<DT, OUT, 1, 256>(p, stream);
    if (pieces <= 512) return launch_row<DT, OUT, 2, 256>(p, stream);
    if (pieces <= 768) return launch_row<DT, OUT, 3, 256>(p, stream);
    if (pieces <= 1024) return launch_row<DT, OUT, 2, 512>(p, stream);
    if (pieces <= 2048) return launch_row<DT, OUT, 4, 512>(p, stream);
    if (pieces <= 4096) return launch_row<DT, OUT, 4, 1024>(p, stream);
    return launch_all(p.n_rows, 1024, [&](dim3 grid, int64_t first) {
        hipLaunchKernelGGL((norm_long_kernel<DT, OUT>), grid, dim3(1024), 0, stream, p, first);
    });
}

template <int DT>
hipError_t launch_type(const NormParams& p, hipStream_t stream) {
    if (p.group < 0) return launch_out<DT, kSame>(p, stream);
    if (p.group == 0) return launch_out<DT, kRowScale>(p, stream);
    return launch_out<DT, kGroupScale>(p, stream);
}

}  // namespace

hipError_t launch_norm(const NormParams& p, hipStream_t stream) {
    if (p.dtype == TL_F32) return launch_type<TL_F32>(p, stream);
    return p.dtype == TL_F16 ? launch_type<TL_F16>(p, stream) : launch_type<TL_BF16>(p, stream);
}

}  // namespace tl
