// moe.hip - a whole MoE layer for a few tokens, straight from the weight pool:
// router, Top-K, gates, SwiGLU experts and their gated sum, without an expert
// cache.
//
//   z = W_r h + b,  S = the K largest z (lower index on equal ones),
//   g = softmax of z over S,  y = sum_k g_k W_down,k (silu(W_gate,k x) * (W_up,k x)).
//
// Three launches: the router with the selection and the plan of the experts'
// work, W_gate and W_up, W_down with the gated sum.  What one part of a launch
// hands to another (the last workgroup of a group goes on with what all of them
// left) is stored and loaded past the caches that the chip's dies do not share,
// and counted after the stores have arrived; nothing waits in a kernel.
//
// The experts' weights are nearly all there is to read: 2 to 64 tokens use each
// of them for a handful of products.  So everything is made for their stream.
// Weight rows go from HBM into LDS without passing registers, eight whole
// 128-byte lines per instruction, and from there to the matrix core; straight
// into its operand registers an instruction would touch sixteen lines, 16 bytes
// at a time, and the same stream runs at 5.0 instead of 6.8 TB/s (800 MB).
#include <algorithm>

#include "cmoe_internal.h"

namespace cmoe {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;

__device__ inline int live_tokens(const MoeArgs& a) {
    return a.n_tokens ? min(max(*a.n_tokens, 0), a.T) : a.T;
}

// Stores and loads at the device's scope: past the L2 of one die.
template <typename T>
__device__ inline void store_device(T* p, T v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ inline T load_device(const T* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// The wavefront's stores before this have arrived when it goes on.
__device__ inline void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Whether the workgroup is the last of `total` to arrive at the counter; what the
// others stored with store_device before arriving is then there to load.
__device__ inline bool last_to_arrive(int32_t* counter, int total) {
    __shared__ int old;
    stores_done();
    __syncthreads();
    if (threadIdx.x == 0) old = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const bool last = old == total - 1;
    __syncthreads();
    return last;
}

// ---------------------------------------------------------------- router
// Eight consecutive values, widened to fp32.
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

// Sums of v[0 .. TG) over the wavefront: lane l gets that of v[l % TG].  While
// there are several values, half of them go to the partner lane, so that TG
// values take TG - 1 + log2(64 / TG) exchanges.
template <int TG>
__device__ inline double wave_sums(double* v, int lane) {
#pragma unroll
    for (int n = TG / 2; n >= 1; n /= 2) {
        const bool up = lane & n;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const double give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
            v[i] = keep + __shfl_xor(give, n);
        }
    }
#pragma unroll
    for (int m = TG; m < 64; m *= 2) v[0] += __shfl_xor(v[0], m);
    return v[0];
}

// Largest of 64 unsigned numbers, uniform.
__device__ inline uint32_t wave_max(uint32_t v) {
#define CMOE_STEP(ctrl, rows) \
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, ctrl, rows, 0xf, false))
    CMOE_STEP(0x111, 0xf);  // row_shr:1, 2, 4, 8: lane 15 of each row of 16 has the row's
    CMOE_STEP(0x112, 0xf);
    CMOE_STEP(0x114, 0xf);
    CMOE_STEP(0x118, 0xf);
    CMOE_STEP(0x142, 0xa);  // row_bcast:15 into rows 1 and 3
    CMOE_STEP(0x143, 0xc);  // row_bcast:31 into rows 2 and 3
#undef CMOE_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Order of the logits as unsigned numbers: NaN above everything, -0 equal to 0;
// 0 is below every logit.
__device__ inline uint32_t rank_key(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return z != z ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ inline float key_logit(uint32_t k) {
    return k == 0xFFFFFFFFu ? NAN : __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// The selection and gates of token t, by one wavefront: lane k ends with the
// k-th largest logit and its expert.
__device__ inline void select_experts(const MoeArgs& a, int t, bool live, int lane) {
    const int64_t at = (int64_t)t * a.K + lane;
    if (!live) {
        if (lane < a.K) store_device(a.sel + at, -1);
        return;
    }
    uint32_t key[kMaxN / 64];
#pragma unroll
    for (int j = 0; j < kMaxN / 64; ++j) {
        const int e = lane + 64 * j;
        key[j] = e < a.N ? rank_key(load_device(a.z + (int64_t)t * a.N + e)) : 0;
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
    const float z = mine ? key_logit(mine) : -INFINITY, top = __shfl(z, 0);
    const bool none = z == -INFINITY;
    const float p = none ? 0.0f : expf(z - top);
    float s = p;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if (lane < a.K) {
        const int e = none ? -1 : expert;
        const float g = none ? 0.0f : p / s;
        store_device(a.sel + at, e);
        a.gate[at] = g;
        if (a.selected) a.selected[at] = e;
        if (a.gates) a.gates[at] = g;
    }
}

// The experts' work from the selection of all tokens, by one workgroup: units of
// up to 16 tokens of an expert, and the row of every (token, expert).
__device__ inline void make_plan(const MoeArgs& a, int n) {
    __shared__ unsigned long long mask[kMaxN];  // tokens of each expert, one bit each
    __shared__ uint16_t first[kMaxN], unit0[kMaxN];
    __shared__ int units;
    const int tid = threadIdx.x, all = a.T * a.K;
    for (int i = tid; i < kMaxN; i += kThreads) mask[i] = 0;
    __syncthreads();
    for (int i = tid; i < all; i += kThreads) {
        const int e = load_device(a.sel + i);
        if (e >= 0) atomicOr(&mask[e], 1ull << (i / a.K));
    }
    __syncthreads();
    if (tid < 64) {  // four experts per lane: prefix sums of rows and units
        int rows[4], nu[4], sr = 0, su = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            rows[j] = __popcll(mask[4 * tid + j]);
            nu[j] = (rows[j] + kMoeUnitTokens - 1) / kMoeUnitTokens;
            sr += rows[j];
            su += nu[j];
        }
        int r = sr, u = su;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int pr = __shfl_up(r, m), pu = __shfl_up(u, m);
            if (tid >= m) {
                r += pr;
                u += pu;
            }
        }
        if (tid == 63) units = u;
        r -= sr;
        u -= su;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            first[4 * tid + j] = (uint16_t)r;
            unit0[4 * tid + j] = (uint16_t)u;
            r += rows[j];
            u += nu[j];
        }
    }
    __syncthreads();
    for (int e = tid; e < a.N; e += kThreads) {
        unsigned long long m = mask[e];
        int row = first[e];
        for (int u = unit0[e]; m; ++u) {
            MoeUnit r;
            r.expert = e;
            r.row = row;
            r.n = 0;
            int t = 0;
            for (int c = 0; c < kMoeUnitTokens; ++c) {
                if (m) {
                    t = __ffsll(m) - 1;
                    m &= m - 1;
                    ++r.n;
                }
                r.token[c] = (uint8_t)t;
            }
            row += r.n;
            a.plan->unit[u] = r;
        }
    }
    for (int i = tid; i < all; i += kThreads) {
        const int e = load_device(a.sel + i);
        a.row_of[i] = e < 0 ? -1 : first[e] + __popcll(mask[e] & ((1ull << (i / a.K)) - 1));
    }
    for (int i = units + tid; i < moe_max_units(all, a.N); i += kThreads) a.plan->unit[i].n = 0;
    for (int i = tid; i < a.d / 16; i += kThreads) a.rows_done[i] = 0;
    if (tid == 0) {
        a.plan->units = units;
        a.plan->groups_done = 0;
    }
    if (units == 0)  // no expert launch writes y
        for (int t = 0; t < n; ++t)
            for (int j = tid; j < a.d; j += kThreads) a.y[(int64_t)t * a.y_stride + j] = 0.0f;
}

// Logits, selection and plan.  grid: x = groups of four experts, one wavefront
// each, y = groups of TG tokens.  The logits are summed in fp64 and rounded to
// fp32 once after the bias, as the cache step's router does: they decide the
// selection.  A bias of -inf takes its expert out whatever the sum is.
template <bool BF16, int TG>
__global__ __launch_bounds__(kThreads) void moe_route_kernel(MoeArgs a) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, t0 = blockIdx.y * TG;
    const int e = blockIdx.x * kWaves + wv, rows = min(a.T - t0, TG);
    if (e < a.N) {
        double acc[TG] = {};
        for (int i = lane * 8; i < a.d; i += 512) {
            float w[8];
            load8<BF16>(a.w_router, (int64_t)e * a.d + i, w);
#pragma unroll
            for (int t = 0; t < TG; ++t) {
                float x[8];
                load8<BF16>(a.h, (int64_t)(t0 + min(t, rows - 1)) * a.h_stride + i, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[t] = __builtin_fma((double)w[j], (double)x[j], acc[t]);
            }
        }
        const double s = wave_sums<TG>(acc, lane);
        const float b = a.bias ? a.bias[e] : 0.0f;
        if (lane < rows) store_device(a.z + (int64_t)(t0 + lane) * a.N + e, b == -INFINITY ? -INFINITY : (float)(s + (double)b));
    }
    if (a.h8)  // the experts' 8-bit input as bf16, in which every value is exact
        for (int64_t t = t0 + blockIdx.x; t < t0 + rows; t += gridDim.x)
            for (int i = threadIdx.x; i < a.d; i += kThreads) {
                const uint32_t byte = a.h8_scale[t * a.h8_scale_stride + i / 32];
                const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a.h8[t * a.h8_stride + i],
                                                                           __uint_as_float(byte << 23), false);
                reinterpret_cast<__bf16*>(a.x)[t * a.d + i] = byte == 255 ? (__bf16)NAN : v[0];
            }
    if (!last_to_arrive(a.plan->logits_done + blockIdx.y, gridDim.x)) return;
    const int n = live_tokens(a);
    for (int t = wv; t < rows; t += kWaves) select_experts(a, t0 + t, t0 + t < n, lane);
    if (threadIdx.x == 0) a.plan->logits_done[blockIdx.y] = 0;
    if (last_to_arrive(&a.plan->groups_done, gridDim.y)) make_plan(a, n);
}

// ---------------------------------------------------------------- products
// Sixteen weight rows against up to 16 G columns, the sum cut into lines of 128
// bytes of a row.  A wavefront takes a range of the lines, kStage at a time: two
// instructions per line bring it in for eight rows each, lane 8 i + p the 16-byte
// unit p ^ i of row i, so that the reads of the operands, lane (r, q) = 16 q + r
// the units q and q + 4 of row r, meet every LDS bank once.  The columns' values
// come straight from the caches; both operands take the same order of the sum.
constexpr int kStage = 4;  // lines of 16 rows in flight per wavefront: 8 KB

template <int FORMAT>
struct Format;

template <>
struct Format<kMoeBf16> {
    static constexpr int kLine = 64;    // values of a line
    static constexpr int kLoads = 2;    // 16-byte loads of a column's values per line
    static constexpr int kPlanes = 3;   // bf16 numbers of an fp32 intermediate value
    static constexpr int kBytes = 2;    // of a column's value
    // first value of load i
    __device__ static int column(int i, int q) { return (q + 4 * i) * 8; }
    __device__ static f32x4 mul(const u32x4 (&w)[2], uint32_t, const u32x4* b, bool, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[i]), __builtin_bit_cast(bf16x8, b[i]), c, 0, 0, 0);
        return c;
    }
};

template <>
struct Format<kMoeMx8> {
    static constexpr int kLine = 128, kLoads = 4, kPlanes = 3, kBytes = 2;
    __device__ static int column(int i, int q) { return (q + 4 * (i >> 1)) * 16 + (i & 1) * 8; }
    // The weights become bf16, in which every value is exact; scales: the line's
    // four.  half: the line holds 64 values.
    __device__ static f32x4 mul(const u32x4 (&w)[2], uint32_t scales, const u32x4* b, bool half, f32x4 c) {
        const int q = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (i == 1 && half) break;
            const float s = __uint_as_float((scales >> (16 * i + 8 * (q >> 1)) & 255u) << 23);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                bf16x8 v;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i][2 * j + k], s, false);
                    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i][2 * j + k], s, true);
                    v[4 * k] = lo[0];
                    v[4 * k + 1] = lo[1];
                    v[4 * k + 2] = hi[0];
                    v[4 * k + 3] = hi[1];
                }
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, b[2 * i + j]), c, 0, 0, 0);
            }
        }
        return c;
    }
};

template <>
struct Format<kMoeF32> {
    static constexpr int kLine = 32, kLoads = 2, kPlanes = 1, kBytes = 4;
    __device__ static int column(int i, int q) { return (q + 4 * i) * 4; }
    __device__ static f32x4 mul(const u32x4 (&w)[2], uint32_t, const u32x4* b, bool, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i][j]), __uint_as_float(b[i][j]), c, 0, 0, 0);
        return c;
    }
};

using LdsBytes = __attribute__((address_space(3))) void*;

// 64 times 16 bytes from each lane's address to LDS, in lane order, nontemporal:
// weights are read once.
__device__ inline void stream_to_lds(const char* p, char* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p, (LdsBytes)lds, 16, 0, 2);
}

// Rows 0 .. 7 and 8 .. 15 of a tile begin at w0 and w1, `pitch` bytes apart (scales
// s0, s1, pitch / 32); columns at x[g] (this lane's, without its place in a line).
// acc[g] gets lines l0 .. l1 of `lines`.
template <int FORMAT, int G>
__device__ inline void tile_product(const char* w0, const char* w1, int64_t pitch, const uint8_t* s0, const uint8_t* s1,
                                    const char* const (&x)[G], int l0, int l1, int lines, char* stage, f32x4 (&acc)[G]) {
    using P = Format<FORMAT>;
    // as many lines at once as leave the columns' values 64 registers
    constexpr int CH = std::max(1, std::min(kStage, 16 / (P::kLoads * G)));
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, i8 = lane >> 3, p8 = (lane & 7) ^ i8;
    // 8-bit rows may end in half a line: units 4 .. 7 of it would be the next row's
    const bool ragged = FORMAT == kMoeMx8 && pitch % 128 != 0;
    w0 += i8 * pitch;
    w1 += i8 * pitch;
    const uint8_t* s = nullptr;
    if constexpr (FORMAT == kMoeMx8) s = (r < 8 ? s0 : s1) + (int64_t)(r & 7) * (pitch / 32);
    const char* place = stage + (r >> 3) * 1024 + (r & 7) * 128;
    for (int l = l0; l < l1; l += CH) {
        u32x4 b[G][CH][P::kLoads];
        uint32_t scales[CH] = {};
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (l + i < l1) {
                const int64_t at = (int64_t)(l + i) * 128 + (ragged && l + i == lines - 1 ? p8 & 3 : p8) * 16;
                stream_to_lds(w0 + at, stage + i * 2048);
                stream_to_lds(w1 + at, stage + i * 2048 + 1024);
            }
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (l + i < l1) {
                const bool half = ragged && l + i == lines - 1;
                if constexpr (FORMAT == kMoeMx8) {
                    if (half) {
                        uint16_t v;
                        __builtin_memcpy(&v, s + 4 * (l + i), 2);
                        scales[i] = v;
                    } else {
                        __builtin_memcpy(&scales[i], s + 4 * (l + i), 4);
                    }
                }
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int j = 0; j < P::kLoads; ++j)
                        if (!(half && j >= P::kLoads / 2))
                            b[g][i][j] = *reinterpret_cast<const u32x4*>(x[g] + ((int64_t)(l + i) * P::kLine + P::column(j, q)) * P::kBytes);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the lines are in LDS
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (l + i < l1) {
                const bool half = ragged && l + i == lines - 1;
                const u32x4 w[2] = {*reinterpret_cast<const u32x4*>(place + i * 2048 + (q ^ (r & 7)) * 16),
                                    *reinterpret_cast<const u32x4*>(place + i * 2048 + ((q + 4) ^ (r & 7)) * 16)};
#pragma unroll
                for (int g = 0; g < G; ++g) acc[g] = P::mul(w, scales[i], b[g][i], half, acc[g]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // and read before the next ones come
    }
}

__device__ inline float silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// fp32 as the sum of three bf16 numbers, exactly but for its last bit or two:
// the intermediate loses nothing on the bf16 matrix core.
__device__ inline void split3(float v, __bf16* p) {
    p[0] = (__bf16)v;
    const float r = fabsf((float)p[0]) < INFINITY ? v - (float)p[0] : 0.0f;
    p[1] = (__bf16)r;
    p[2] = (__bf16)(r - (float)p[1]);
}

// Gate and up projections and the SwiGLU product: a tile is eight rows of W_gate
// and the same eight of W_up; the wavefronts take a quarter of the sum each.
// grid: x = F / 8, y = units
template <int FORMAT>
__global__ __launch_bounds__(kThreads, 4) void moe_up_kernel(MoeArgs a) {
    using P = Format<FORMAT>;
    __shared__ __align__(16) char stage[kWaves][kStage * 2048];
    __shared__ f32x4 red[kWaves][64];
    const MoeUnit& unit = a.plan->unit[blockIdx.y];
    const int n = unit.n;
    if (n == 0) return;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    const int64_t pitch = (int64_t)a.d * 128 / P::kLine;  // bytes of a weight row
    const int64_t row = (int64_t)unit.expert * 3 * a.F + blockIdx.x * 8;
    const char* w = static_cast<const char*>(a.experts) + row * pitch;
    const uint8_t* s = FORMAT == kMoeMx8 ? a.scales + row * (pitch / 32) : nullptr;
    const int lines = (a.d + P::kLine - 1) / P::kLine;
    const char* x[1] = {(a.h8 ? reinterpret_cast<const char*>(a.x) : static_cast<const char*>(a.h)) +
                        unit.token[r] * (a.h8 ? (int64_t)a.d : a.h_stride) * P::kBytes};
    f32x4 acc[1] = {};
    tile_product<FORMAT, 1>(w, w + a.F * pitch, pitch, s, s + a.F * (pitch / 32), x, wv * lines / kWaves,
                            (wv + 1) * lines / kWaves, lines, stage[wv], acc);
    red[wv][lane] = acc[0];
    __syncthreads();
    // lane (c, q) of a product holds rows 4 q .. of column c: q = 0, 1 W_gate's, 2, 3 W_up's
    if (threadIdx.x < 32 && r < n) {
        f32x4 g = red[0][lane], u = red[0][lane + 32];
#pragma unroll
        for (int k = 1; k < kWaves; ++k) {
            g += red[k][lane];
            u += red[k][lane + 32];
        }
        const int64_t at = unit.row + r;
        const int f = blockIdx.x * 8 + (lane >> 4) * 4;
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = silu_mul(g[j], u[j]);
        if constexpr (FORMAT == kMoeF32) {
            *reinterpret_cast<f32x4*>(static_cast<float*>(a.act) + at * a.F + f) = v;
        } else {
            __bf16 p[4][3];
#pragma unroll
            for (int j = 0; j < 4; ++j) split3(v[j], p[j]);
#pragma unroll
            for (int i = 0; i < 3; ++i)
                *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.act) + (at * 3 + i) * a.F + f) =
                    bf16x4{p[0][i], p[1][i], p[2][i], p[3][i]};
        }
    }
}

// y of 16 outputs for all tokens, by one wavefront: the gated sum over a token's
// experts in descending logit.
__device__ inline void sum_rows(const MoeArgs& a, int j0, int lane) {
    const int n = live_tokens(a), q = lane >> 4;
    for (int t = lane & 15; t < n; t += 16) {
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < a.K; ++k) {
            const int row = a.row_of[t * a.K + k];
            if (row < 0) continue;
            const float g = a.gate[t * a.K + k];
            const unsigned long long* p =
                reinterpret_cast<const unsigned long long*>(a.out + (int64_t)row * a.d + j0 + 4 * q);
            const unsigned long long v[2] = {load_device(p), load_device(p + 1)};
            f32x4 o;
            __builtin_memcpy(&o, v, 16);
            y += g * o;
        }
        *reinterpret_cast<f32x4*>(a.y + (int64_t)t * a.y_stride + j0 + 4 * q) = y;
    }
}

// Columns of the down product for G groups of 16: column i is bf16 number i / n
// of token i % n's intermediate, so that up to five tokens take one group.
template <int FORMAT, int G>
__device__ inline void down_product(const MoeArgs& a, const MoeUnit& unit, const char* w, int64_t pitch, const uint8_t* s,
                                    int l0, int l1, int lines, char* stage, f32x4 (*red)[64]) {
    using P = Format<FORMAT>;
    const int lane = threadIdx.x & 63, r = lane & 15, n = unit.n;
    const char* x[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int i = min(16 * g + r, P::kPlanes * n - 1);
        x[g] = static_cast<const char*>(a.act) + ((unit.row + i % n) * (int64_t)P::kPlanes + i / n) * a.F * P::kBytes;
    }
    f32x4 acc[G] = {};
    tile_product<FORMAT, G>(w, w + 8 * pitch, pitch, s, s + 8 * (pitch / 32), x, l0, l1, lines, stage, acc);
#pragma unroll
    for (int g = 0; g < G; ++g) red[g][lane] = acc[g];
}

// Down projection and the gated sum: the workgroup's wavefronts are kWaves / split
// tiles of 16 rows, `split` parts of the sum each.  The wavefront that brings a
// tile's last unit adds the tile up for all tokens.
// grid: x = d / 16 / (kWaves / split) rounded up, y = units
template <int FORMAT>
__global__ __launch_bounds__(kThreads, 4) void moe_down_kernel(MoeArgs a, int split) {
    using P = Format<FORMAT>;
    constexpr int kGroups = P::kPlanes;
    __shared__ __align__(16) char stage[kWaves][kStage * 2048];
    __shared__ f32x4 red[kWaves][kGroups][64];
    const MoeUnit& unit = a.plan->unit[blockIdx.y];
    const int n = unit.n;
    if (n == 0) return;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int tile = blockIdx.x * (kWaves / split) + wv / split, part = wv % split;
    const int groups = (P::kPlanes * n + 15) / 16;
    if (tile < a.d / 16) {
        const int64_t pitch = (int64_t)a.F * 128 / P::kLine;
        const int64_t up = (int64_t)unit.expert * 3 * a.F * (a.d * 128 / P::kLine);  // bytes before the expert
        const char* w = static_cast<const char*>(a.experts) + up + 2 * a.F * ((int64_t)a.d * 128 / P::kLine) + tile * 16 * pitch;
        const uint8_t* s = FORMAT == kMoeMx8 ? a.scales + (w - static_cast<const char*>(a.experts)) / 32 : nullptr;
        const int lines = (a.F + P::kLine - 1) / P::kLine, l0 = part * lines / split, l1 = (part + 1) * lines / split;
        if (groups == 1)
            down_product<FORMAT, 1>(a, unit, w, pitch, s, l0, l1, lines, stage[wv], red[wv]);
        else if constexpr (kGroups > 1) {
            if (groups == 2)
                down_product<FORMAT, 2>(a, unit, w, pitch, s, l0, l1, lines, stage[wv], red[wv]);
            else
                down_product<FORMAT, 3>(a, unit, w, pitch, s, l0, l1, lines, stage[wv], red[wv]);
        }
    }
    __syncthreads();
    if (part != 0 || tile >= a.d / 16) return;
    if (r < n) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = P::kPlanes - 1; p >= 0; --p) {  // the smallest first
            const int i = p * n + r;
            for (int k = 0; k < split; ++k) v += red[wv + k][i >> 4][16 * q + (i & 15)];
        }
        unsigned long long o[2];
        __builtin_memcpy(o, &v, 16);
        unsigned long long* to = reinterpret_cast<unsigned long long*>(a.out + (int64_t)(unit.row + r) * a.d + tile * 16 + 4 * q);
        store_device(to, o[0]);
        store_device(to + 1, o[1]);
    }
    stores_done();
    int old = 0;
    if (lane == 0) old = __hip_atomic_fetch_add(a.rows_done + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__builtin_amdgcn_readfirstlane(old) == a.plan->units - 1) {
        asm volatile("" ::: "memory");
        sum_rows(a, tile * 16, lane);
    }
}

template <bool BF16>
void launch_route(const MoeArgs& a, hipStream_t st) {
    const unsigned gx = (a.N + kWaves - 1) / kWaves;
    if (a.T == 1)
        launch_kernel(moe_route_kernel<BF16, 1>, dim3(gx, 1), dim3(kThreads), st, Timing{}, a);
    else
        launch_kernel(moe_route_kernel<BF16, 8>, dim3(gx, (a.T + 7) / 8), dim3(kThreads), st, Timing{}, a);
}

template <int FORMAT>
void launch_experts(const MoeArgs& a, hipStream_t st) {
    const int rows = a.T * a.K, units = moe_max_units(rows, a.N);
    const int lines = (a.F + Format<FORMAT>::kLine - 1) / Format<FORMAT>::kLine;
    // parts of the down sum: four lines at least, more parts where the tiles alone
    // do not fill the device
    int split = lines >= 32 ? 4 : lines >= 16 ? 2 : 1;
    while (split < kWaves && (int64_t)(a.d / 16) * units * split < 4096) split *= 2;
    const int tiles = kWaves / split;
    launch_kernel(moe_up_kernel<FORMAT>, dim3(a.F / 8, units), dim3(kThreads), st, Timing{}, a);
    launch_kernel(moe_down_kernel<FORMAT>, dim3((a.d / 16 + tiles - 1) / tiles, units), dim3(kThreads), st, Timing{}, a, split);
}

__global__ void moe_init_kernel(MoePlan* plan) {
    plan->logits_done[threadIdx.x] = 0;
    if (threadIdx.x == 0) plan->groups_done = plan->units = 0;
}

}  // namespace

hipError_t launch_moe_init(MoePlan* plan, hipStream_t st) {
    launch_kernel(moe_init_kernel, dim3(1), dim3(kMoeTokens), st, Timing{}, plan);
    return hipGetLastError();
}

hipError_t launch_moe(const MoeArgs& a, hipStream_t st) {
    if (a.bf16)
        launch_route<true>(a, st);
    else
        launch_route<false>(a, st);
    if (a.format == kMoeF32)
        launch_experts<kMoeF32>(a, st);
    else if (a.format == kMoeBf16)
        launch_experts<kMoeBf16>(a, st);
    else
        launch_experts<kMoeMx8>(a, st);
    return hipGetLastError();
}

}  // namespace cmoe
