// moe.hip - a whole MoE layer for a few tokens, straight from the weight pool:
// router, Top-K, gates, SwiGLU experts and their gated sum, without an expert
// cache.
//
//   z = W_r h + b,  S = the K largest z (lower index on equal ones),
//   g = softmax of z over S,  y = sum_k g_k W_down,k (silu(W_gate,k x) * (W_up,k x)).
//
// Tokens of an expert are the 16 columns of a matrix-core tile (a unit), weight
// rows its 16 rows; the wavefronts of a workgroup share the sum's length.
#include <algorithm>

#include "cmoe_internal.h"

namespace cmoe {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kMaxUnits = kMaxN + kMoeTokens * kMaxK / kMoeUnitTokens;

__device__ inline int live_tokens(const MoeArgs& a) {
    return a.n_tokens ? min(max(*a.n_tokens, 0), a.T) : a.T;
}

// ---------------------------------------------------------------- router
// Logits in fp64, rounded to fp32 once after the bias, as the cache step's
// router does: they decide the selection.  A bias of -inf takes its expert out
// whatever the sum is.
constexpr int kRouterTokens = 8, kRouterThreads = 256;

template <bool BF16>
__device__ inline void load8(const void* p, int64_t i, float* v) {
    if constexpr (BF16) {
        const bf16x8 r = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(p) + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)r[j];
    } else {
        const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
        const f32x4 a = q[0], b = q[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = a[j];
            v[4 + j] = b[j];
        }
    }
}

// grid: x = experts, y = groups of kRouterTokens tokens
template <bool BF16>
__global__ __launch_bounds__(kRouterThreads) void moe_router_kernel(MoeArgs a) {
    __shared__ double red[kRouterThreads / 64][kRouterTokens];
    const int e = blockIdx.x, t0 = blockIdx.y * kRouterTokens, tid = threadIdx.x;
    const int n = min(live_tokens(a) - t0, kRouterTokens);
    if (n <= 0) return;
    double acc[kRouterTokens] = {};
    for (int i = tid * 8; i < a.d; i += kRouterThreads * 8) {
        float w[8];
        load8<BF16>(a.w_router, (int64_t)e * a.d + i, w);
#pragma unroll
        for (int t = 0; t < kRouterTokens; ++t) {
            float x[8];
            load8<BF16>(a.h, (int64_t)(t0 + min(t, n - 1)) * a.h_stride + i, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[t] = __builtin_fma((double)w[j], (double)x[j], acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < kRouterTokens; ++t) {
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) acc[t] += __shfl_xor(acc[t], m);
        if ((tid & 63) == 0) red[tid >> 6][t] = acc[t];
    }
    __syncthreads();
    if (tid < n) {
        double s = 0.0;
#pragma unroll
        for (int w = 0; w < kRouterThreads / 64; ++w) s += red[w][tid];
        const float b = a.bias ? a.bias[e] : 0.0f;
        a.z[(int64_t)(t0 + tid) * a.N + e] = b == -INFINITY ? -INFINITY : (float)(s + (double)b);
    }
    // the experts' 8-bit input as bf16, in which each value is exact
    for (int64_t t = t0 + e; a.h8 && t < t0 + n; t += a.N) {
        for (int i = tid; i < a.d; i += kRouterThreads) {
            const uint32_t byte = a.h8_scale[t * a.h8_scale_stride + i / 32];
            const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a.h8[t * a.h8_stride + i], __uint_as_float(byte << 23), false);
            reinterpret_cast<__bf16*>(a.x)[t * a.d + i] = byte == 255 ? (__bf16)NAN : v[0];
        }
    }
}

// ---------------------------------------------------------------- Top-K
// Order of the logits as unsigned numbers: NaN above everything, -0 equal to 0.
__device__ inline uint32_t rank_key(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return z != z ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// One wavefront per token: K times the largest remaining (logit, lower index).
__global__ __launch_bounds__(64) void moe_topk_kernel(MoeArgs a) {
    const int t = blockIdx.x, lane = threadIdx.x;
    if (t >= live_tokens(a)) return;
    unsigned long long key[kMaxN / 64];
#pragma unroll
    for (int j = 0; j < kMaxN / 64; ++j) {
        const int e = lane + 64 * j;
        key[j] = e < a.N ? ((unsigned long long)rank_key(a.z[(int64_t)t * a.N + e]) << 8 | (255 - e)) + 1 : 0;
    }
    int mine = -1;
    for (int k = 0; k < a.K; ++k) {
        unsigned long long m = 0;
#pragma unroll
        for (int j = 0; j < kMaxN / 64; ++j) m = max(m, key[j]);
#pragma unroll
        for (int s = 32; s >= 1; s >>= 1) m = max(m, __shfl_xor(m, s));
        if (lane == k) mine = 255 - (int)((m - 1) & 255);
#pragma unroll
        for (int j = 0; j < kMaxN / 64; ++j) key[j] = key[j] == m ? 0 : key[j];
    }
    const float z = mine >= 0 ? a.z[(int64_t)t * a.N + mine] : -INFINITY;
    const float top = __shfl(z, 0);
    const bool none = z == -INFINITY;
    const float p = none ? 0.0f : expf(z - top);
    float s = p;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if (lane < a.K) {
        const int64_t i = (int64_t)t * a.K + lane;
        const int e = none ? -1 : mine;
        const float g = none ? 0.0f : p / s;
        a.sel[i] = e;
        a.gate[i] = g;
        if (a.selected) a.selected[i] = e;
        if (a.gates) a.gates[i] = g;
    }
}

// ---------------------------------------------------------------- plan
// The experts' tokens, from the selection: each workgroup builds it in LDS.
struct Plan {
    unsigned long long mask[kMaxN];  // tokens of each expert, one bit each
    uint16_t first[kMaxN];           // row of an expert's first token: rows are (expert, token) in order
    uint16_t unit[kMaxUnits];        // expert | (pass << 8): tokens 16 pass .. of it
    int units;
};

__device__ inline void build_plan(const MoeArgs& a, Plan& p) {
    const int tid = threadIdx.x;
    for (int i = tid; i < kMaxN; i += blockDim.x) p.mask[i] = 0;
    __syncthreads();
    const int n = live_tokens(a) * a.K;
    for (int i = tid; i < n; i += blockDim.x) {
        const int e = a.sel[i];
        if (e >= 0) atomicOr(&p.mask[e], 1ull << (i / a.K));
    }
    __syncthreads();
    if (tid < 64) {  // four experts per lane: prefix sums of rows and units
        int rows[4], units[4], sr = 0, su = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            rows[j] = __popcll(p.mask[4 * tid + j]);
            units[j] = (rows[j] + kMoeUnitTokens - 1) / kMoeUnitTokens;
            sr += rows[j];
            su += units[j];
        }
        int ir = sr, iu = su;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int r = __shfl_up(ir, m), u = __shfl_up(iu, m);
            if (tid >= m) {
                ir += r;
                iu += u;
            }
        }
        int r = ir - sr, u = iu - su;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            p.first[4 * tid + j] = (uint16_t)r;
            for (int q = 0; q < units[j]; ++q) p.unit[u++] = (uint16_t)((4 * tid + j) | q << 8);
            r += rows[j];
        }
        if (tid == 63) p.units = iu;
    }
    __syncthreads();
}

// Token of the n-th set bit (n < popcount).
__device__ inline int nth_token(unsigned long long m, int n) {
    for (int i = 0; i < n; ++i) m &= m - 1;
    return __ffsll(m) - 1;
}

// ---------------------------------------------------------------- products
// A wavefront's part of a 16-row tile: lane (r, q) holds W[row r][64 c + 16 q ..
// + 16] of chunk c (64 values of the sum) and x[token r][the same]; the matrix
// core pairs them, whatever the order of the 64.
template <int FORMAT>
struct Weights;

template <>
struct Weights<kMoeBf16> {
    static constexpr int kPlanes = 3;
    struct A { u32x4 v[2]; };
    struct B { u32x4 v[2]; };
    __device__ static A load_a(const void* w, const uint8_t*, int64_t at, int) {
        const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(w) + at);
        return A{__builtin_nontemporal_load(p), __builtin_nontemporal_load(p + 1)};
    }
    __device__ static B load_b(const void* x, int64_t at) {
        const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(x) + at);
        return B{p[0], p[1]};
    }
    __device__ static f32x4 mul(const A& a, const B& b, f32x4 c) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.v[j]), __builtin_bit_cast(bf16x8, b.v[j]), c, 0, 0, 0);
        return c;
    }
};

template <>
struct Weights<kMoeMx8> {
    static constexpr int kPlanes = 3;
    struct A { u32x4 v; uint32_t byte; };
    using B = Weights<kMoeBf16>::B;
    __device__ static A load_a(const void* w, const uint8_t* scales, int64_t at, int) {
        return A{__builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(w) + at)), scales[at >> 5]};
    }
    __device__ static B load_b(const void* x, int64_t at) { return Weights<kMoeBf16>::load_b(x, at); }
    // the 8-bit weights are exact in bf16
    __device__ static f32x4 mul(const A& a, const B& b, f32x4 c) {
        const float s = __uint_as_float(a.byte << 23);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            bf16x8 w;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a.v[2 * j + i], s, false);
                const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a.v[2 * j + i], s, true);
                w[4 * i] = lo[0];
                w[4 * i + 1] = lo[1];
                w[4 * i + 2] = hi[0];
                w[4 * i + 3] = hi[1];
            }
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, b.v[j]), c, 0, 0, 0);
        }
        return c;
    }
};

template <>
struct Weights<kMoeF32> {
    static constexpr int kPlanes = 1;
    struct A { f32x4 v[4]; };
    using B = A;
    __device__ static A load_a(const void* w, const uint8_t*, int64_t at, int) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(w) + at);
        A a;
#pragma unroll
        for (int j = 0; j < 4; ++j) a.v[j] = __builtin_nontemporal_load(p + j);
        return a;
    }
    __device__ static B load_b(const void* x, int64_t at) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(x) + at);
        return B{{p[0], p[1], p[2], p[3]}};
    }
    __device__ static f32x4 mul(const A& a, const B& b, f32x4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j][i], b.v[j][i], c, 0, 0, 0);
        return c;
    }
};

__device__ inline float silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// fp32 as the sum of three bf16 numbers, exactly but for its last bit or two:
// the intermediate loses nothing on the bf16 matrix core.
__device__ inline void split3(float v, __bf16* p) {
    p[0] = (__bf16)v;
    const float r = fabsf((float)p[0]) < INFINITY ? v - (float)p[0] : 0.0f;
    p[1] = (__bf16)r;
    p[2] = (__bf16)(r - (float)p[1]);
}

// Adds the wavefronts' tiles in order; lane (c, g) of wavefront 0 gets rows
// 4 g .. 4 g + 3 of column c.
template <int NA>
__device__ inline void join(f32x4 (&acc)[NA], f32x4 (*red)[NA][64]) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < NA; ++i) red[wv][i][lane] = acc[i];
    __syncthreads();
    if (wv == 0)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            for (int w = 1; w < kWaves; ++w) acc[i] += red[w][i][lane];
}

// grid: x = F / 16, y = units
template <int FORMAT>
__global__ __launch_bounds__(kThreads) void moe_up_kernel(MoeArgs a) {
    using W = Weights<FORMAT>;
    __shared__ Plan plan;
    __shared__ f32x4 red[kWaves][2][64];
    build_plan(a, plan);
    if ((int)blockIdx.y >= plan.units) return;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int unit = plan.unit[blockIdx.y], e = unit & 255, pass = unit >> 8;
    const unsigned long long m = plan.mask[e];
    const int n = min(__popcll(m) - pass * kMoeUnitTokens, kMoeUnitTokens);
    const int token = nth_token(m, pass * kMoeUnitTokens + min(r, n - 1));
    const int f0 = blockIdx.x * 16;
    const int64_t gate = ((int64_t)e * 3 * a.F + f0 + r) * a.d + 16 * q, up = gate + (int64_t)a.F * a.d;
    const void* x = a.h8 ? a.x : a.h;
    const int64_t xb = (int64_t)token * (a.h8 ? a.d : a.h_stride) + 16 * q;
    f32x4 acc[2] = {};
    for (int c = wv; c < a.d / 64; c += kWaves) {
        const auto g = W::load_a(a.experts, a.scales, gate + 64 * c, q);
        const auto u = W::load_a(a.experts, a.scales, up + 64 * c, q);
        const auto b = W::load_b(x, xb + 64 * c);
        acc[0] = W::mul(g, b, acc[0]);
        acc[1] = W::mul(u, b, acc[1]);
    }
    join(acc, red);
    if (wv == 0 && r < n) {
        const int64_t row = plan.first[e] + pass * kMoeUnitTokens + r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float v = silu_mul(acc[0][j], acc[1][j]);
            const int f = f0 + 4 * q + j;
            if constexpr (FORMAT == kMoeF32) {
                static_cast<float*>(a.act)[row * a.F + f] = v;
            } else {
                __bf16 p[3];
                split3(v, p);
#pragma unroll
                for (int i = 0; i < 3; ++i) static_cast<__bf16*>(a.act)[(row * 3 + i) * a.F + f] = p[i];
            }
        }
    }
}

// grid: x = d / 16, y = units
template <int FORMAT>
__global__ __launch_bounds__(kThreads) void moe_down_kernel(MoeArgs a) {
    using W = Weights<FORMAT>;
    __shared__ Plan plan;
    __shared__ f32x4 red[kWaves][1][64];
    build_plan(a, plan);
    if ((int)blockIdx.y >= plan.units) return;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int unit = plan.unit[blockIdx.y], e = unit & 255, pass = unit >> 8;
    const int n = min(__popcll(plan.mask[e]) - pass * kMoeUnitTokens, kMoeUnitTokens);
    const int64_t row0 = plan.first[e] + pass * kMoeUnitTokens, row = row0 + min(r, n - 1);
    const int j0 = blockIdx.x * 16;
    const int64_t at = (int64_t)e * 3 * a.F * a.d + (int64_t)2 * a.F * a.d + (int64_t)(j0 + r) * a.F + 16 * q;
    f32x4 acc[1] = {};
    for (int c = wv; c < a.F / 64; c += kWaves) {
        const auto w = W::load_a(a.experts, a.scales, at + 64 * c, q);
#pragma unroll
        for (int i = W::kPlanes - 1; i >= 0; --i)
            acc[0] = W::mul(w, W::load_b(a.act, (row * W::kPlanes + i) * a.F + 16 * q + 64 * c), acc[0]);
    }
    join(acc, red);
    if (wv == 0 && r < n) *reinterpret_cast<f32x4*>(a.out + (row0 + r) * a.d + j0 + 4 * q) = acc[0];
}

// grid: x = tokens
__global__ __launch_bounds__(kThreads) void moe_sum_kernel(MoeArgs a) {
    __shared__ Plan plan;
    __shared__ int row[kMaxK];
    const int t = blockIdx.x;
    build_plan(a, plan);
    if (t >= live_tokens(a)) return;
    if (threadIdx.x < a.K) {
        const int e = a.sel[(int64_t)t * a.K + threadIdx.x];
        row[threadIdx.x] = e < 0 ? -1 : plan.first[e] + __popcll(plan.mask[e] & ((1ull << t) - 1));
    }
    __syncthreads();
    for (int j = threadIdx.x; j < a.d; j += kThreads) {
        float s = 0.0f;
        for (int k = 0; k < a.K; ++k)
            if (row[k] >= 0) s += a.gate[(int64_t)t * a.K + k] * a.out[(int64_t)row[k] * a.d + j];
        a.y[(int64_t)t * a.y_stride + j] = s;
    }
}

template <int FORMAT>
void launch_experts(const MoeArgs& a, hipStream_t st) {
    const int rows = a.T * a.K, units = std::min(rows, a.N + rows / kMoeUnitTokens);
    launch_kernel(moe_up_kernel<FORMAT>, dim3(a.F / 16, units), dim3(kThreads), st, Timing{}, a);
    launch_kernel(moe_down_kernel<FORMAT>, dim3(a.d / 16, units), dim3(kThreads), st, Timing{}, a);
}

}  // namespace

hipError_t launch_moe(const MoeArgs& a, hipStream_t st) {
    const dim3 grid(a.N, (a.T + kRouterTokens - 1) / kRouterTokens);
    launch_kernel(a.bf16 ? moe_router_kernel<true> : moe_router_kernel<false>, grid, dim3(kRouterThreads), st, Timing{}, a);
    launch_kernel(moe_topk_kernel, dim3(a.T), dim3(64), st, Timing{}, a);
    if (a.format == kMoeF32)
        launch_experts<kMoeF32>(a, st);
    else if (a.format == kMoeBf16)
        launch_experts<kMoeBf16>(a, st);
    else
        launch_experts<kMoeMx8>(a, st);
    launch_kernel(moe_sum_kernel, dim3(a.T), dim3(kThreads), st, Timing{}, a);
    return hipGetLastError();
}

}  // namespace cmoe
