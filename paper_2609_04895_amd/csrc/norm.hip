// norm.hip - what stands between two layer steps: the residual's addition with
// its root-mean-square norm, r = fl(residual + delta), h = r w / sqrt(mean r^2 +
// eps), and rows into 8 bits (mx8.h), as an output of the norm or on their own.
//
// One pass over the data: each thread keeps its values of a row in registers
// between the sum of squares and the outputs, so every input is read and every
// output written once.  Both kernels are bound by HBM for many rows (8192 rows of
// 2880 bf16 values with an fp32 delta: 47.7 us, 5.5 TB/s; 604 million values into 8
// bits: 294 us, 6.2 TB/s) and by the launch and one trip to memory for few (one row
// of 2048: 2.7 us).
//
// r is rounded to the residual's type before it is squared, so that the norm is
// that of the residual as stored.  Squares, their sum and the factor are fp64, and r w
// times the factor is rounded to fp32 once (Factor); h in bf16 and in 8 bits is
// rounded from that fp32 value.  In fp32 the squares of values beyond 2^64 or below
// 2^-75 leave the range, so do r w where h does not (r = 2^126, w = 4) and the factor
// of values below 2^-128; and with fp32 sums and r s w values next to a border of two
// 8-bit numbers fell to the other side one and a half to two times as often as in a
// plain fp32 form.
#include <algorithm>

#include "cmoe_internal.h"
#include "mx8.h"

namespace cmoe {

namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Eight consecutive values, widened to fp32.  NT: nontemporal, where there are so
// many that the caches would not keep them: the norm's outputs from kNormNT bytes on,
// all of quantize from 2^26 values on (604 million bf16 values 301 us against 311;
// 1.4 million fp32 values 4.5 us against 3.0).
template <bool NT, typename V>
__device__ inline V get(const void* p) {
    if constexpr (NT)
        return __builtin_nontemporal_load(static_cast<const V*>(p));
    else
        return *static_cast<const V*>(p);
}
template <bool NT, typename V>
__device__ inline void put(void* p, V v) {
    if constexpr (NT)
        __builtin_nontemporal_store(v, static_cast<V*>(p));
    else
        *static_cast<V*>(p) = v;
}

template <bool BF16, bool NT = false>
__device__ inline void load8(const void* p, int64_t i, float* v) {
    if constexpr (BF16) {
        const bf16x8 r = get<NT, bf16x8>(static_cast<const __bf16*>(p) + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)r[j];
    } else {
        const float* q = static_cast<const float*>(p) + i;
        const f32x4 a = get<NT, f32x4>(q), b = get<NT, f32x4>(q + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = a[j];
            v[4 + j] = b[j];
        }
    }
}

template <bool BF16, bool NT = false>
__device__ inline void store8(void* p, int64_t i, const float* v) {
    if constexpr (BF16) {
        bf16x8 r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = (__bf16)v[j];
        put<NT>(static_cast<__bf16*>(p) + i, r);
    } else {
        float* q = static_cast<float*>(p) + i;
        put<NT>(q, f32x4{v[0], v[1], v[2], v[3]});
        put<NT>(q + 4, f32x4{v[4], v[5], v[6], v[7]});
    }
}

template <bool BF16>
__device__ inline float load1(const void* p, int64_t i) {
    if constexpr (BF16)
        return (float)static_cast<const __bf16*>(p)[i];
    else
        return static_cast<const float*>(p)[i];
}

template <bool BF16>
__device__ inline float rounded(float v) {
    if constexpr (BF16)
        return (float)(__bf16)v;
    else
        return v;
}

template <bool BF16>
__device__ inline void store1(void* p, int64_t i, float v) {
    if constexpr (BF16)
        static_cast<__bf16*>(p)[i] = (__bf16)v;
    else
        static_cast<float*>(p)[i] = v;
}

__device__ inline double wave_sum(double v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// Sum over the TPR threads of a row, in a fixed order; every thread gets it.
// TPR > 64: red holds one partial per wavefront and the row is the workgroup's.
template <int TPR>
__device__ inline double row_sum(double v, double* red) {
    v = wave_sum(v);
    if constexpr (TPR > 64) {
        const int wv = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[wv] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) v += red[w];
    }
    return v;
}

// s = 1 / sqrt(mean + eps), applied to r w and rounded to fp32 once.  s = 2^e m, 1 <= m
// < 2: r 2^e is at most sqrt(d), so that 2^e r w is in range where h is.  m is the sum
// of two fp32 numbers, and so is the product of fp32 values (that of bf16 values is
// exact), but for what falls below fp32's range.  fp64 products instead: bf16, 8192
// rows of 2880, 72 against 52 us; fp32, 8192 rows of 8192, 251 against 200.
template <bool BF16>
struct Factor {
    int e;
    float hi, lo;
    __device__ Factor(double sum, const NormArgs& a) {
        const double s = 1.0 / sqrt(sum / a.d + (double)a.eps);
        // not of a row of zeros without an eps, of infinities or a NaN, whose finite
        // values a power below all of them takes out of the product
        const bool normal = s > 0.0 && s < INFINITY;
        e = normal ? ilogb(s) : -512;
        const double m = ldexp(s, -e);
        hi = (float)m;
        lo = normal ? (float)(m - (double)hi) : 0.0f;
    }
    __device__ float times(float r, float w) const {
        const float v = ldexpf(r, e), p = v * w;
        const float rest = BF16 ? p * lo : __builtin_fmaf(p, lo, __builtin_fmaf(v, w, -p) * hi);
        return __builtin_fmaf(p, hi, fabsf(p) < INFINITY ? rest : 0.0f);  // h beyond fp32 is p's infinity
    }
};

__device__ inline int live_rows(const NormArgs& a) {
    return a.n_rows ? min(max(*a.n_rows, 0), a.rows) : a.rows;
}

constexpr int kThreads = 256;  // threads of a workgroup with one wavefront per row: four rows

// d % 8 == 0 and every row 16-byte aligned.  TPR threads per row, thread t taking
// the groups of 8 values t, t + TPR, ... (NV at most); the four groups of a block
// of 32 lie in neighbouring lanes.
template <bool BF16, int DELTA, int TPR, int NV, bool NT>
__global__ __launch_bounds__(TPR > kThreads ? TPR : kThreads) void norm_kernel(NormArgs a) {
    __shared__ double red[TPR > 64 ? TPR / 64 : 1];
    constexpr int RPG = TPR >= kThreads ? 1 : kThreads / TPR;  // rows per workgroup
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPG + threadIdx.x / TPR;
    if (row >= live_rows(a)) return;  // whole wavefronts, and whole workgroups where they share a row
    const int ng = a.d / 8;
    float r[NV][8] = {};
    double ss = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int g = t + i * TPR;
        if (g < ng) load8<BF16>(a.residual, row * a.residual_stride + 8 * g, r[i]);
    }
    if constexpr (DELTA != 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int g = t + i * TPR;
            if (g < ng) {
                float v[8];
                load8<DELTA == 2>(a.delta, row * a.delta_stride + 8 * g, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) r[i][j] = rounded<BF16>(r[i][j] + v[j]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int g = t + i * TPR;
        if (g < ng) {
#pragma unroll
            for (int j = 0; j < 8; ++j) ss = __builtin_fma((double)r[i][j], (double)r[i][j], ss);
            if (a.residual_out) store8<BF16, NT>(a.residual_out, row * a.residual_out_stride + 8 * g, r[i]);
        }
    }
    const Factor<BF16> s(row_sum<TPR>(ss, red), a);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int g = t + i * TPR;
        const bool in = g < ng;
        if (in) {
            float w[8];
            if (a.weight) load8<BF16>(a.weight, 8 * g, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) r[i][j] = s.times(r[i][j], a.weight ? w[j] : 1.0f);
            if (a.h) store8<BF16, NT>(a.h, row * a.h_stride + 8 * g, r[i]);
        }
        if (a.h8) {  // d % 32 == 0: the lanes of a block are all in or all out
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = mx_max(m, r[i][j]);
            m = mx_max(m, __shfl_xor(m, 1));
            m = mx_max(m, __shfl_xor(m, 2));
            if (in) {
                const uint32_t byte = mx_scale_byte(m);
                const uint2 q = mx_pack8(r[i], byte);
                put<NT>(a.h8 + row * a.h8_stride + 8 * g, u32x2{q.x, q.y});
                if ((g & 3) == 0) a.h8_scale[row * a.h8_scale_stride + g / 4] = (uint8_t)byte;
            }
        }
    }
}

// Any d, any alignment: one workgroup per row, one value per thread and step.
// The second pass reads the inputs again (from the caches) and does the
// additions again.
template <bool BF16, int DELTA>
__global__ __launch_bounds__(kThreads) void norm_any_kernel(NormArgs a) {
    __shared__ double red[kThreads / 64];
    const int64_t row = blockIdx.x;
    if (row >= live_rows(a)) return;
    auto value = [&](int i) {
        float v = load1<BF16>(a.residual, row * a.residual_stride + i);
        if constexpr (DELTA != 0) v = rounded<BF16>(v + load1<DELTA == 2>(a.delta, row * a.delta_stride + i));
        return v;
    };
    double ss = 0.0;
    for (int i = threadIdx.x; i < a.d; i += kThreads) {
        const double v = (double)value(i);
        ss = __builtin_fma(v, v, ss);
    }
    const Factor<BF16> s(row_sum<kThreads>(ss, red), a);
    for (int i0 = 0; i0 < a.d; i0 += kThreads) {
        const int i = i0 + threadIdx.x;
        float v = 0.0f;
        if (i < a.d) {
            v = value(i);
            // every element is read for the last time by the thread that overwrites it
            if (a.residual_out) store1<BF16>(a.residual_out, row * a.residual_out_stride + i, v);
            v = s.times(v, a.weight ? load1<BF16>(a.weight, i) : 1.0f);
            if (a.h) store1<BF16>(a.h, row * a.h_stride + i, v);
        }
        if (a.h8) {
            float m = mx_max(v, 0.0f);
#pragma unroll
            for (int k = 1; k < kMxBlock; k <<= 1) m = mx_max(m, __shfl_xor(m, k));
            if (i < a.d) {
                const uint32_t byte = mx_scale_byte(m);
                a.h8[row * a.h8_stride + i] =
                    (uint8_t)(byte == kMxBad ? kMxNaN2 : mx_pair<false>(v, v, mx_inverse(byte), 0));
                if (i % kMxBlock == 0) a.h8_scale[row * a.h8_scale_stride + i / kMxBlock] = (uint8_t)byte;
            }
        }
    }
}

// Bytes of outputs from which they are written nontemporally: an XCD's L2.  Cached /
// nontemporal, us, behind a kernel that writes delta and before one that reads h (bf16,
// fp32 delta, all three outputs): 1024 x 256 (1.3 MB) 3.4 / 3.5, 2048 x 512 (5.2 MB)
// 4.3 / 4.2, 2048 x 1024 (10 MB) 6.7 / 6.6, 2048 x 2880 (29 MB) 16.1 / 14.3, 8192 x 4096
// (168 MB) 73.8 / 60.8; on its own 8192 x 2880 52.7 / 48.1.
constexpr int64_t kNormNT = 1 << 22;

template <bool BF16, int DELTA, bool NT>
void launch_rows(const NormArgs& a, hipStream_t st) {
    const int ng = a.d / 8;
    auto go = [&](auto kernel, int tpr) {
        const int rpg = tpr >= kThreads ? 1 : kThreads / tpr;
        launch_kernel(kernel, dim3((unsigned)((a.rows + rpg - 1) / rpg)), dim3(tpr > kThreads ? tpr : kThreads), st, Timing{}, a);
    };
    // A wavefront per row for many narrow ones, a workgroup otherwise.  Wavefront /
    // workgroup, us, bf16 rows, in the order of kernels above:
    //   rows of  512: 1024 rows 3.7 / 3.7, 4096 6.4 / 7.8, 16384 18.0 / 26.3
    //           1024: 1024 5.1 / 4.4, 2048 6.6 / 6.6, 4096 9.5 / 11.4, 12000 24.6 / 27.2
    //           2048: 1024 8.7 / 6.5, 3000 15.1 / 15.0, 4096 15.6 / 18.1, 6000 22.2 / 23.7, 8192 33.0 / 30.5
    //           2880: 3000 18.4 / 19.7, 4096 22.5 / 25.5, 5000 27.0 / 29.8, 6000 37.3 / 34.4, 16384 95.8 / 92.6
    //           4096: 1024 15.0 / 9.6, 4096 30.4 / 32.7, 8192 61.9 / 60.8, 16384 147 / 131
    // (on their own, 4096 rows of 4096 31.3 / 31.2.)
    if (ng <= 64 && a.rows >= 1024)
        go(norm_kernel<BF16, DELTA, 64, 1, NT>, 64);
    else if (ng <= 128 && a.rows >= 2048)
        go(norm_kernel<BF16, DELTA, 64, 2, NT>, 64);
    else if (ng <= 256 && a.rows >= 4096 && a.rows < 6144)
        go(norm_kernel<BF16, DELTA, 64, 4, NT>, 64);
    else if (ng <= 384 && a.rows >= 4096 && a.rows < 6144)
        go(norm_kernel<BF16, DELTA, 64, 6, NT>, 64);
    else if (ng <= 256)
        go(norm_kernel<BF16, DELTA, 256, 1, NT>, 256);
    else if (ng <= 512)
        go(norm_kernel<BF16, DELTA, 256, 2, NT>, 256);
    else if (ng <= 1024)
        go(norm_kernel<BF16, DELTA, 1024, 1, NT>, 1024);
    else
        go(norm_kernel<BF16, DELTA, 1024, 4, NT>, 1024);
}

template <bool BF16, int DELTA>
hipError_t launch_norm_t(const NormArgs& a, bool aligned, hipStream_t st) {
    const int e = BF16 ? 2 : 4;
    const int64_t bytes = (int64_t)a.rows * a.d * ((a.residual_out ? e : 0) + (a.h ? e : 0) + (a.h8 ? 1 : 0));
    if (!aligned || a.d / 8 > 4096)
        launch_kernel(norm_any_kernel<BF16, DELTA>, dim3((unsigned)a.rows), dim3(kThreads), st, Timing{}, a);
    else if (bytes >= kNormNT)
        launch_rows<BF16, DELTA, true>(a, st);
    else
        launch_rows<BF16, DELTA, false>(a, st);
    return hipGetLastError();
}

// Sixteen values per thread, half a block, 16-byte loads and stores.  unit: the
// half block's number in its row.
template <bool BF16, bool NT>
__device__ inline void quantize16(const void* src, int64_t at, uint8_t* q, uint8_t* scale, int64_t unit, bool in) {
    float v[16] = {};
    float m = 0.0f;
    if (in) {
        load8<BF16, NT>(src, at, v);
        load8<BF16, NT>(src, at + 8, v + 8);
#pragma unroll
        for (int j = 0; j < 16; ++j) m = mx_max(m, v[j]);
    }
    m = mx_max(m, __shfl_xor(m, 1));
    if (!in) return;
    const uint32_t byte = mx_scale_byte(m);
    const uint2 a = mx_pack8(v, byte), b = mx_pack8(v + 8, byte);
    put<NT>(q + 16 * unit, u32x4{a.x, a.y, b.x, b.y});
    if ((unit & 1) == 0) scale[unit / 2] = (uint8_t)byte;
}

// Rows that follow each other without gaps: one long row.
template <bool BF16, bool NT>
__global__ __launch_bounds__(kThreads) void quantize_flat_kernel(QuantizeArgs a) {
    const int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const bool in = u < a.rows * (a.cols / 16);
    quantize16<BF16, NT>(a.src, 16 * u, a.q, a.scale, u, in);
}

// Rows apart: tpr threads (a power of two, at least 2) per row and step.
// grid: x = rows / (kThreads / tpr) rounded up, y = workgroups that share a row
template <bool BF16>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(QuantizeArgs a, int tpr) {
    const int64_t row = (int64_t)blockIdx.x * (kThreads / tpr) + threadIdx.x / tpr;
    const int64_t t = threadIdx.x % tpr, n = a.cols / 16;
    for (int64_t u0 = (int64_t)blockIdx.y * tpr; u0 < n; u0 += (int64_t)gridDim.y * tpr) {
        const int64_t u = u0 + t;
        quantize16<BF16, false>(a.src, row * a.src_stride + 16 * u, a.q + row * a.q_stride, a.scale + row * a.scale_stride, u,
                         row < a.rows && u < n);
    }
}

template <bool BF16>
hipError_t launch_quantize_t(const QuantizeArgs& a, hipStream_t st) {
    const int64_t units = a.rows * (a.cols / 16);
    if (a.rows == 1 || (a.src_stride == a.cols && a.q_stride == a.cols && a.scale_stride == a.cols / kMxBlock)) {
        launch_kernel(units >= 1 << 22 ? quantize_flat_kernel<BF16, true> : quantize_flat_kernel<BF16, false>,
                      dim3((unsigned)((units + kThreads - 1) / kThreads)), dim3(kThreads), st, Timing{}, a);
    } else {
        int tpr = 2;
        while (tpr < kThreads && tpr < a.cols / 16) tpr *= 2;
        const int64_t rpg = kThreads / tpr, groups = (a.rows + rpg - 1) / rpg, steps = (a.cols / 16 + tpr - 1) / tpr;
        // few long rows: as many workgroups each as give the device 4096 in all
        const int64_t share = std::max<int64_t>(1, std::min(steps, 4096 / groups));
        launch_kernel(quantize_rows_kernel<BF16>, dim3((unsigned)groups, (unsigned)share), dim3(kThreads), st, Timing{}, a, tpr);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, bool aligned, hipStream_t st) {
    const int delta = a.delta == nullptr ? 0 : a.delta_bf16 ? 2 : 1;
    if (a.bf16)
        return delta == 0   ? launch_norm_t<true, 0>(a, aligned, st)
               : delta == 1 ? launch_norm_t<true, 1>(a, aligned, st)
                            : launch_norm_t<true, 2>(a, aligned, st);
    return delta == 0   ? launch_norm_t<false, 0>(a, aligned, st)
           : delta == 1 ? launch_norm_t<false, 1>(a, aligned, st)
                        : launch_norm_t<false, 2>(a, aligned, st);
}

hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t st) {
    return a.bf16 ? launch_quantize_t<true>(a, st) : launch_quantize_t<false>(a, st);
}

}  // namespace cmoe
