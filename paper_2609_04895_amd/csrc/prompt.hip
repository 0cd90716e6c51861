// prompt.hip - what an MoE layer needs around its grouped products when it runs a
// prompt's tokens: logits, selection and gates, the rows' order by expert, and the
// gated sum.
//
// Four launches before the products (logits; selection, with a mask of each chunk's
// tokens for every expert; each expert's tokens counted over the chunks; rows placed)
// and one behind them.  A row's place is its expert's first row, the expert's tokens in
// the chunks before, and the mask's bits below its own: no atomic decides an order, so
// results do not depend on the order of workgroups.  4096 tokens of 128 experts, top-8,
// d = 2048: logits 51 to 58 us, selection 10 to 11, counting and placing 5 each, hardly
// more than launches, the sum 27.
#include <algorithm>

#include "cmoe_internal.h"
#include "select.h"

namespace cmoe {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef double f64x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;

__device__ inline int live_tokens(const PromptArgs& a) { return a.n_tokens ? min(max(*a.n_tokens, 0), a.T) : a.T; }

__device__ inline void load8(const float* p, float* v) {
    const f32x4* s = reinterpret_cast<const f32x4*>(p);
    const f32x4 a = s[0], b = s[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = a[j];
        v[4 + j] = b[j];
    }
}

// Logits, summed in fp64 and rounded to fp32 once after the bias: they decide the
// selection.  The fp64 matrix core takes a tile of 16 experts by 16 tokens and four
// values of the sum, lane (r, q) = 16 q + r one value of row r each, so a lane's eight
// consecutive values go into eight of its instructions; the order of the sum is the
// same for both operands.  A workgroup takes TE x TT tiles, its wavefronts an eighth of
// the sum each, and the loads of the next 32 values are under way while these are
// multiplied.  Bound by the fp64 matrix core and the loads' way to it: 4096 x 128 x 2048
// in 51 us, 42 of the core's 78 TFLOP/s; 2048 x 128 x 4096 in 48.
// grid: x = experts / (16 TE), y = tokens / (16 TT), rounded up
template <bool BF16>
struct Eight {  // eight consecutive values as they lie in memory
    u32x4 v[BF16 ? 1 : 2];
    __device__ void load(const void* p, int64_t i) {
        const u32x4* s = reinterpret_cast<const u32x4*>(static_cast<const char*>(p) + i * (BF16 ? 2 : 4));
#pragma unroll
        for (int k = 0; k < (BF16 ? 1 : 2); ++k) v[k] = s[k];
    }
    __device__ double operator[](int j) const {
        if constexpr (BF16) return (double)__uint_as_float(j % 2 ? v[0][j / 2] & 0xFFFF0000u : v[0][j / 2] << 16);
        return (double)__uint_as_float(v[BF16 ? 0 : j / 4][j % 4]);
    }
};

constexpr int kLogitWaves = 8;
template <bool BF16, int TE, int TT>
__global__ __launch_bounds__(64 * kLogitWaves) void prompt_logits_kernel(PromptArgs a) {
    __shared__ double red[kLogitWaves - 1][TE * TT * 4][64];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, wv = threadIdx.x >> 6;
    const int e0 = blockIdx.x * TE * 16, t0 = blockIdx.y * TT * 16, rows = live_tokens(a);
    if (t0 >= rows) return;
    int64_t we[TE], xt[TT];
#pragma unroll
    for (int e = 0; e < TE; ++e) we[e] = (int64_t)min(e0 + 16 * e + r, a.N - 1) * a.d + 8 * q;
#pragma unroll
    for (int t = 0; t < TT; ++t) xt[t] = (int64_t)min(t0 + 16 * t + r, rows - 1) * a.h_stride + 8 * q;
    f64x4 acc[TE][TT] = {};
    const int steps = a.d / 32;
    Eight<BF16> w[TE], x[TT];
    auto load = [&](int s) {
#pragma unroll
        for (int e = 0; e < TE; ++e) w[e].load(a.w_router, we[e] + 32 * s);
#pragma unroll
        for (int t = 0; t < TT; ++t) x[t].load(a.h, xt[t] + 32 * s);
    };
    if (wv < steps) load(wv);
    for (int s = wv; s < steps; s += kLogitWaves) {
        Eight<BF16> wn[TE], xn[TT];
#pragma unroll
        for (int e = 0; e < TE; ++e) wn[e] = w[e];
#pragma unroll
        for (int t = 0; t < TT; ++t) xn[t] = x[t];
        if (s + kLogitWaves < steps) load(s + kLogitWaves);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int e = 0; e < TE; ++e) acc[e][t] = __builtin_amdgcn_mfma_f64_16x16x4f64(wn[e][j], xn[t][j], acc[e][t], 0, 0, 0);
    }
    if (wv)
#pragma unroll
        for (int e = 0; e < TE; ++e)
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) red[wv - 1][(e * TT + t) * 4 + i][lane] = acc[e][t][i];
    __syncthreads();
    if (wv) return;
    // lane (r, q) holds experts 4 i + q of a tile for token r
#pragma unroll
    for (int e = 0; e < TE; ++e)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                double s = acc[e][t][i];
#pragma unroll
                for (int k = 0; k < kLogitWaves - 1; ++k) s += red[k][(e * TT + t) * 4 + i][lane];
                const int expert = e0 + 16 * e + 4 * i + q, token = t0 + 16 * t + r;
                if (expert < a.N && token < rows) {
                    const float b = a.bias ? a.bias[expert] : 0.0f;
                    a.z[(int64_t)token * a.N + expert] = b == -INFINITY ? -INFINITY : (float)(s + (double)b);
                }
            }
}

template <bool BF16>
void launch_logits(const PromptArgs& a, hipStream_t st) {
    auto go = [&](auto kernel, int te, int tt) {
        launch_kernel(kernel, dim3((a.N + 16 * te - 1) / (16 * te), (a.T + 16 * tt - 1) / (16 * tt)), dim3(64 * kLogitWaves), st, Timing{}, a);
    };
    if ((int64_t)((a.N + 63) / 64) * ((a.T + 31) / 32) >= 256)
        go(prompt_logits_kernel<BF16, 2, 2>, 2, 2);
    else
        go(prompt_logits_kernel<BF16, 2, 1>, 2, 1);
}

// The selection of a chunk's tokens, a wavefront per token at a time, and the masks.
// grid: x = chunks
constexpr int kSelectThreads = 1024;
__global__ __launch_bounds__(kSelectThreads) void prompt_select_kernel(PromptArgs a) {
    __shared__ uint32_t mask[kMaxN];
    const int lane = threadIdx.x & 63, n = live_tokens(a), t0 = blockIdx.x * kPromptChunk;
    if (threadIdx.x < kMaxN) mask[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x >> 6; i < kPromptChunk; i += kSelectThreads / 64) {
        const int t = t0 + i;
        if (t >= n) break;
        uint32_t key[kMaxN / 64];
#pragma unroll
        for (int j = 0; j < kMaxN / 64; ++j) {
            const int e = lane + 64 * j;
            key[j] = e < a.N ? rank_key(a.z[(int64_t)t * a.N + e]) : 0;
        }
        uint32_t mine = 0;
        int expert = -1;
        for (int k = 0; k < a.K; ++k) {
            const uint32_t m = wave_max(max(max(key[0], key[1]), max(key[2], key[3])));
            int e = -1;
#pragma unroll
            for (int j = kMaxN / 64 - 1; j >= 0; --j) {
                const unsigned long long b = __ballot(key[j] == m);
                if (b) e = 64 * j + __ffsll(b) - 1;
            }
#pragma unroll
            for (int j = 0; j < kMaxN / 64; ++j) key[j] = e == lane + 64 * j ? 0 : key[j];
            if (lane == k) {
                mine = m;
                expert = e;
            }
        }
        const float z = mine ? key_logit(mine) : -INFINITY;
        const bool none = z == -INFINITY;
        const float top = __shfl(z, 0), p = none ? 0.0f : expf(z - top);
        float s = p;
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
        if (lane < a.K) {
            const int64_t at = (int64_t)t * a.K + lane;
            const float g = none ? 0.0f : p / s;
            const int e = none ? -1 : expert;
            a.gate[at] = g;
            a.expert[at] = e;
            if (a.selected) a.selected[at] = e;
            if (a.gates) a.gates[at] = g;
            if (e >= 0) atomicOr(&mask[e], 1u << i);
        }
    }
    __syncthreads();
    if (threadIdx.x < a.N) a.mask[(int64_t)blockIdx.x * a.N + threadIdx.x] = mask[threadIdx.x];
}

// Sum over the workgroup's threads up to and with each.
__device__ inline int scan(int v, int* part) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int p = __shfl_up(v, m);
        if (lane >= m) v += p;
    }
    __syncthreads();
    if (lane == 63) part[wv] = v;
    __syncthreads();
    for (int k = 0; k < wv; ++k) v += part[k];
    return v;
}

// An expert's tokens in the chunks before each.
// grid: x = experts
__global__ __launch_bounds__(kThreads) void prompt_count_kernel(PromptArgs a) {
    __shared__ int part[kWaves], sum;
    const int e = blockIdx.x, chunks = (a.T + kPromptChunk - 1) / kPromptChunk;
    if (threadIdx.x == 0) sum = 0;
    __syncthreads();
    for (int c0 = 0; c0 < chunks; c0 += kThreads) {
        const int c = c0 + threadIdx.x, v = c < chunks ? __popc(a.mask[(int64_t)c * a.N + e]) : 0;
        const int before = sum, end = before + scan(v, part);
        if (c < chunks) a.before[(int64_t)c * a.N + e] = end - v;
        __syncthreads();
        if (threadIdx.x == kThreads - 1) sum = end;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.total[e] = sum;
}

// Each selected expert's row, and each row's token.
// grid: x = chunks
__global__ __launch_bounds__(kThreads) void prompt_place_kernel(PromptArgs a) {
    __shared__ int part[kWaves], first[kMaxN];
    const int e = threadIdx.x, v = e < a.N ? a.total[e] : 0, end = scan(v, part);
    first[e] = end - v;
    if (blockIdx.x == 0 && e < a.N) {
        a.first[e] = end - v;
        if (e == a.N - 1) a.first[a.N] = end;
    }
    __syncthreads();
    const int t0 = blockIdx.x * kPromptChunk, n = min(live_tokens(a) - t0, kPromptChunk);
    for (int i = threadIdx.x; i < n * a.K; i += kThreads) {
        const int64_t at = (int64_t)t0 * a.K + i;
        const int k = a.expert[at], bit = i / a.K;
        if (k < 0) continue;
        const int64_t c = (int64_t)blockIdx.x * a.N + k;
        const int row = first[k] + a.before[c] + __popc(a.mask[c] & ((1u << bit) - 1));
        a.row[at] = row;
        a.token[row] = t0 + bit;
    }
}

// y: the gated sum over a token's experts in descending logit, of fp32 outputs or of
// halves whose 32 share a scale (product.h).  Bound by memory: 4096 tokens, top-8,
// d = 2048, bf16 y, 156 MB in 27 us, 5.8 TB/s.
// grid: x = tokens, y = d / (8 kThreads) rounded up
template <bool BF16>
__global__ __launch_bounds__(kThreads) void prompt_sum_kernel(PromptArgs a) {
    const int t = blockIdx.x, j = (blockIdx.y * kThreads + threadIdx.x) * 8;
    if (t >= live_tokens(a) || j >= a.d) return;
    float y[8] = {};
    for (int k = 0; k < a.K; ++k) {
        const int64_t at = (int64_t)t * a.K + k;
        if (a.expert[at] < 0) break;  // the rest has none either
        const float g = a.gate[at];
        const int64_t row = a.row[at];
        float v[8];
        if constexpr (BF16) {
            const half8 h = *reinterpret_cast<const half8*>(static_cast<const _Float16*>(a.out) + row * a.d + j);
            const float s = __uint_as_float(((uint32_t)a.out_scale[row * (a.d / 32) + j / 32] - 14u) << 23);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)h[i] * s;
        } else {
            load8(static_cast<const float*>(a.out) + row * a.d + j, v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += g * v[i];
    }
    if constexpr (BF16) {
        bf16x8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (__bf16)y[i];
        *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(a.y) + (int64_t)t * a.y_stride + j) = o;
    } else {
        f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(a.y) + (int64_t)t * a.y_stride + j);
        o[0] = f32x4{y[0], y[1], y[2], y[3]};
        o[1] = f32x4{y[4], y[5], y[6], y[7]};
    }
}

}  // namespace

hipError_t launch_prompt_route(const PromptArgs& a, hipStream_t st) {
    const unsigned chunks = (a.T + kPromptChunk - 1) / kPromptChunk;
    if (a.bf16)
        launch_logits<true>(a, st);
    else
        launch_logits<false>(a, st);
    launch_kernel(prompt_select_kernel, dim3(chunks), dim3(kSelectThreads), st, Timing{}, a);
    launch_kernel(prompt_count_kernel, dim3(a.N), dim3(kThreads), st, Timing{}, a);
    launch_kernel(prompt_place_kernel, dim3(chunks), dim3(kThreads), st, Timing{}, a);
    return hipGetLastError();
}

hipError_t launch_prompt_sum(const PromptArgs& a, hipStream_t st) {
    launch_kernel(a.bf16 ? prompt_sum_kernel<true> : prompt_sum_kernel<false>, dim3(a.T, (a.d / 8 + kThreads - 1) / kThreads), dim3(kThreads),
                  st, Timing{}, a);
    return hipGetLastError();
}

}  // namespace cmoe
