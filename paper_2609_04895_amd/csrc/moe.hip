// moe.hip - a whole MoE layer for a few tokens, straight from the weight pool:
// router, Top-K, gates, SwiGLU experts and their gated sum, without an expert
// cache.
//
//   z = W_r h + b,  S = the K largest z (lower index on equal ones),
//   g = softmax of z over S,  y = sum_k g_k W_down,k (silu(W_gate,k x) * (W_up,k x)).
//
// Five launches: logits, the selection with the plan of the experts' work (above 32
// tokens a launch each), W_gate and W_up, W_down, the gated sum.  Or three, for one
// token and for a few that hardly share an expert (each_alone): logits, W_gate and
// W_up with the selection in front, W_down with the gated sum behind.  A small launch
// that reads what the one before it wrote takes 4.5 us, whatever it does (2.7 where
// nothing was written just before); joins within a launch (the last workgroup to
// arrive goes on) took more, 8 to 36 us: an atomic on one address takes 7 to 11 ns, a
// fence for other workgroups 4 to 8 us.
//
// The experts' weights are nearly all there is to read: 1 to 64 tokens use each
// of them for a handful of products.  So everything is made for their stream.
// Weight rows come from HBM eight whole 128-byte lines per instruction and pass
// through LDS into the order in which the matrix core takes them; loaded straight
// into its operand registers, sixteen lines per instruction and 16 bytes of each,
// the same stream runs at 5.0 instead of 6.8 TB/s (800 MB; a plain read of it runs
// at 7.1).  The registers hold the lines in flight, not LDS (loads that go there
// directly): 302 against 268 us for the gate and up products of 64 tokens in 8 bits,
// 13.1 against 11.3 for those of one token's eight experts out of the last-level cache.
//
// Medians, us, of one call on weights that come from HBM (N x d x F, top-K, tokens;
// TB/s of the weights; plan: with the selection's launch):
//                                  logits plan    up          down      sum
//   128 x 2048 x 768, 8, bf16,  1    3.0         12.5 (4.0)   8.6 (2.9)
//   128 x 2048 x 768, 8, bf16, 61    5.6   9.7  112   (6.6)  64.3 (5.7)  4.9
//   128 x 2048 x 768, 8, 8 bit, 5    4.6   5.2   21.2 (5.4)  15.2 (3.8)  4.6
//    32 x 2880 x 2880, 4, bf16, 16   4.7   4.8  140   (6.6)  70.3 (6.6)  4.7
//   128 x 4096 x 1536, 8, 8 bit, 64  8.6   9.8  268   (6.1) 163   (5.0)  5.0
// (rates: of the weights of the experts that the tokens reach.)
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

// Sums of v[0 .. N) over the wavefront: lane l gets that of v[l % N].  While there
// are several values, half of them go to the partner lane, so that N values take
// N - 1 + log2(64 / N) exchanges.  ALL: the N of the first call.
template <int N, int ALL = N>
__device__ __forceinline__ double wave_sums(const double (&v)[N], int lane) {
    if constexpr (N == 1) {
        double s = v[0];
#pragma unroll
        for (int m = ALL; m < 64; m *= 2) s += __shfl_xor(s, m);
        return s;
    } else {
        constexpr int n = N / 2;
        const bool up = lane & n;
        double h[n];
#pragma unroll
        for (int i = 0; i < n; ++i) h[i] = (up ? v[i + n] : v[i]) + __shfl_xor(up ? v[i] : v[i + n], n);
        return wave_sums<n, ALL>(h, lane);
    }
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

// The first `count` experts of token t's selection, by one wavefront: lane k gets
// that of the k-th largest logit, or -1 (none) for a logit of -inf.  With all K of
// them it can write the gates and the outputs.
__device__ inline int select_experts(const MoeArgs& a, int t, int lane, int count, bool write) {
    uint32_t key[kMaxN / 64];
#pragma unroll
    for (int j = 0; j < kMaxN / 64; ++j) {
        const int e = lane + 64 * j;
        key[j] = e < a.N ? rank_key(a.z[(int64_t)t * a.N + e]) : 0;
    }
    uint32_t mine = 0;
    int expert = -1;
    for (int k = 0; k < count; ++k) {
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
    if (!write) return none ? -1 : expert;
    const float top = __shfl(z, 0), p = none ? 0.0f : expf(z - top);
    float s = p;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    const int e = none ? -1 : expert;
    if (lane < a.K) {
        const int64_t at = (int64_t)t * a.K + lane;
        const float g = p / s;
        a.gate[at] = none ? -1.0f : g;
        if (a.selected) a.selected[at] = e;
        if (a.gates) a.gates[at] = none ? 0.0f : g;
    }
    return e;
}

// The selection on its own, a token per workgroup.  For more than two tokens per
// wavefront of the plan's one workgroup this is the faster way in spite of its
// launch: top-8 of 128, 64 tokens 4.7 and 4.8 us against 15, 32 tokens 9.5 both ways.
__global__ __launch_bounds__(64) void moe_select_kernel(MoeArgs a) {
    const int t = blockIdx.x, lane = threadIdx.x;
    if (t >= live_tokens(a)) return;
    const int e = select_experts(a, t, lane, a.K, true);
    if (lane < a.K) a.expert[t * a.K + lane] = e;
}

// Selection of all tokens and the plan of the experts' work, units of up to 16
// tokens of an expert.  One workgroup: what its wavefronts hand each other stays in
// LDS.  Logits of rows behind the last token are there too; they are not waited
// for a count that says so, only dropped.
// Bound by latency: 5.4 us, most of it a launch's, and by the instructions of the
// selections on one CU above 16 tokens.
//
// SELECTED: moe_select_kernel has selected.
constexpr int kPlanThreads = 1024;
template <bool SELECTED>
__global__ __launch_bounds__(kPlanThreads) void moe_plan_kernel(MoeArgs a) {
    __shared__ unsigned long long mask[kMaxN];    // tokens of each expert, one bit each
    __shared__ uint8_t place[kMaxN][kMoeTokens];  // of the expert in the token's selection
    __shared__ uint16_t first[kMaxN], unit0[kMaxN];
    __shared__ int units;
    const int tid = threadIdx.x, lane = tid & 63;
    const int n = live_tokens(a);
    if (tid < kMaxN) mask[tid] = 0;
    __syncthreads();
    auto add = [&](int t, int k, int e) {
        if (e < 0) return;
        place[e][t] = (uint8_t)k;
        atomicOr(&mask[e], 1ull << t);
    };
    if constexpr (SELECTED) {
        for (int i = tid; i < n * a.K; i += kPlanThreads) add(i / a.K, i % a.K, a.expert[i]);
    } else {
        for (int t = tid >> 6; t < a.T; t += kPlanThreads / 64) {
            const int e = select_experts(a, t, lane, a.K, t < n);
            if (lane < a.K && t < n) add(t, lane, e);
        }
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
    if (tid < a.N) {
        unsigned long long m = mask[tid];
        int row = first[tid];
        for (int u = unit0[tid]; m; ++u) {
            MoeUnit r;
            r.expert = tid;
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
                r.slot[c] = (uint16_t)(t * a.K + place[tid][t]);
            }
            row += r.n;
            a.plan->unit[u] = r;
        }
    }
    for (int i = units + tid; i < moe_max_units(a.T * a.K, a.N); i += kPlanThreads) a.plan->unit[i].n = 0;
}

// Logits, summed in fp64 and rounded to fp32 once after the bias, as the cache
// step's router does: they decide the selection.  A bias of -inf takes its expert
// out whatever the sum is.  Widening a value to fp64 takes as long as four
// products: EG experts share each of a token's.  Bound by latency up to 16 tokens
// (2.8 us for one, 4.5 for 16), by fp64 above (64 tokens, 128 x 4096: 7.2 us with
// four experts by eight tokens, 13.9 with one by eight).
// grid: x = groups of EG experts, y = groups of TG tokens; the wavefronts share the sum.
template <bool BF16, int EG, int TG>
__global__ __launch_bounds__(kThreads) void moe_logits_kernel(MoeArgs a) {
    __shared__ double red[kWaves][EG * TG];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, t0 = blockIdx.y * TG, e0 = blockIdx.x * EG;
    const int rows = min(a.T - t0, TG);
    double acc[EG * TG] = {};
    for (int i = threadIdx.x * 8; i < a.d; i += kThreads * 8) {
        float w[EG][8], x[TG][8];
#pragma unroll
        for (int e = 0; e < EG; ++e) load8<BF16>(a.w_router, (int64_t)min(e0 + e, a.N - 1) * a.d + i, w[e]);
#pragma unroll
        for (int t = 0; t < TG; ++t) load8<BF16>(a.h, (int64_t)(t0 + min(t, rows - 1)) * a.h_stride + i, x[t]);
        __builtin_amdgcn_sched_barrier(0);  // every load before the first use
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            double v[EG];
#pragma unroll
            for (int e = 0; e < EG; ++e) v[e] = (double)w[e][j];
#pragma unroll
            for (int t = 0; t < TG; ++t) {
                const double u = (double)x[t][j];
#pragma unroll
                for (int e = 0; e < EG; ++e) acc[e * TG + t] = __builtin_fma(v[e], u, acc[e * TG + t]);
            }
        }
    }
    const double part = wave_sums(acc, lane);
    if (lane < EG * TG) red[wv][lane] = part;
    __syncthreads();
    if (threadIdx.x < EG * TG) {
        const int e = e0 + lane / TG, t = lane % TG;
        double s = red[0][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += red[w][lane];
        if (e < a.N && t < rows) {
            const float b = a.bias ? a.bias[e] : 0.0f;
            a.z[(int64_t)(t0 + t) * a.N + e] = b == -INFINITY ? -INFINITY : (float)(s + (double)b);
        }
    }
    if (a.h8)  // the experts' 8-bit input as bf16, exact from 2^-126 on; 16 values per thread
        for (int64_t t = t0 + blockIdx.x; t < t0 + rows; t += gridDim.x)
            for (int i = threadIdx.x; i < a.d / 16; i += kThreads) {
                const uint32_t byte = a.h8_scale[t * a.h8_scale_stride + i / 2];
                const u32x4 q = *reinterpret_cast<const u32x4*>(a.h8 + t * a.h8_stride + 16 * i);
                const float s = __uint_as_float(byte << 23);
                bf16x8 v[2];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[j], s, false);
                    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[j], s, true);
                    v[j / 2][4 * (j % 2)] = lo[0];
                    v[j / 2][4 * (j % 2) + 1] = lo[1];
                    v[j / 2][4 * (j % 2) + 2] = hi[0];
                    v[j / 2][4 * (j % 2) + 3] = hi[1];
                }
                bf16x8* to = reinterpret_cast<bf16x8*>(a.x + t * a.d + 16 * i);
                if (byte == 255)
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j / 8][j % 8] = (__bf16)NAN;
                to[0] = v[0];
                to[1] = v[1];
            }
}

// ---------------------------------------------------------------- products
// Sixteen weight rows against up to 8 NB columns, the sum cut into lines of 128
// bytes of a row.  A wavefront takes RT tiles of 16 rows and a range of the lines.
// An instruction loads one line of eight rows, lane 8 i + p the 16-byte unit p of
// row i, and goes through the wavefront's part of LDS, unit p at place p ^ i of its
// row, so that the writes, and the reads of the operands, lane (r, q) = 16 q + r
// the units q and q + 4 of row r, meet every LDS bank once.  The columns' values
// come the same way (straight into operand registers, 16 columns cost an
// instruction 64 cache lookups, and the columns of the down product as much time
// as its weights); both operands take the same order of the sum.
//
// The registers hold the lines in flight, CH per wavefront: line l + CH is asked
// for when line l has gone to LDS, which holds one line at a time.  8 KB of weights
// per wavefront and 8 to 16 wavefronts per CU: with twice as much in flight the
// rate falls (6.8 to 6.2 TB/s), with four tiles of rows it stays.
//
// 8-bit rows of an odd number of half lines (kMoeMx8Odd) begin in the middle of a
// line of memory every other time: what is loaded as one line is half of two, and
// the sum ends in half a line.  There the weights go through the caches, which keep
// a line for its second half; elsewhere they are read once, nontemporally.  Cached
// against nontemporal, gate and up and down: 64 tokens of 32 experts of 2880 x 2880
// 123 and 88 against 136 and 101 us; whole lines, 64 tokens of 128 experts of 4096 x
// 1536, 293 and 173 against 273 and 162.
constexpr int kMoeMx8Odd = 3;

template <int FORMAT>
struct Format;

template <>
struct Format<kMoeBf16> {
    static constexpr bool kScaled = false, kOdd = false;
    static constexpr int kLine = 64;   // values of a line of weights
    static constexpr int kParts = 1;   // 128-byte lines that these values take in a column
    static constexpr int kPlanes = 3;  // bf16 numbers of an fp32 intermediate value
    static constexpr int kBytes = 2;   // of a column's value
    static constexpr int kReads = 1;   // operand reads of a column per half line
    __device__ static int unit(int i, int, int q) { return q + 4 * i; }  // of half i, read j
    // half a line: unit w of the lane's row
    __device__ static f32x4 mul(const u32x4& w, uint32_t, int, const u32x4* b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, b[0]), c, 0, 0, 0);
    }
};

template <>
struct Format<kMoeMx8> {
    static constexpr bool kScaled = true, kOdd = false;
    static constexpr int kLine = 128, kParts = 2, kPlanes = 3, kBytes = 2;
    static constexpr int kReads = 2;
    __device__ static int unit(int, int j, int q) { return 2 * q + j; }  // half i is part i
    // The weights become bf16, in which every value of 2^-126 and more in magnitude
    // is exact; scales: the line's four.
    __device__ static f32x4 mul(const u32x4& w, uint32_t scales, int i, const u32x4* b, f32x4 c) {
        const int q = (threadIdx.x & 63) >> 4;
        const float s = __uint_as_float((scales >> (16 * i + 8 * (q >> 1)) & 255u) << 23);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            bf16x8 v;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * j + k], s, false);
                const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * j + k], s, true);
                v[4 * k] = lo[0];
                v[4 * k + 1] = lo[1];
                v[4 * k + 2] = hi[0];
                v[4 * k + 3] = hi[1];
            }
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, b[j]), c, 0, 0, 0);
        }
        return c;
    }
};

template <>
struct Format<kMoeMx8Odd> : Format<kMoeMx8> {
    static constexpr bool kOdd = true;
};

template <>
struct Format<kMoeF32> {
    static constexpr bool kScaled = false, kOdd = false;
    static constexpr int kLine = 32, kParts = 1, kPlanes = 1, kBytes = 4, kReads = 1;
    __device__ static int unit(int i, int, int q) { return q + 4 * i; }
    __device__ static f32x4 mul(const u32x4& w, uint32_t, int, const u32x4* b, f32x4 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[j]), __uint_as_float(b[0][j]), c, 0, 0, 0);
        return c;
    }
};

// A wavefront's weight tiles: rows 0 .. 7 and 8 .. 15 of a tile begin at w0 and w1,
// `pitch` bytes apart, the next tile `next` bytes on (scales s0, s1, all distances
// / 32).
struct Tiles {
    const char *w0, *w1;
    const uint8_t *s0, *s1;
    int64_t pitch, next;
};

// Parts of a line's columns that are held at once: both, unless there are so many
// columns that they leave no registers for the weights.
template <int FORMAT, int NB>
constexpr int kHeld = NB <= 2 ? Format<FORMAT>::kParts : 1;

// Bytes of LDS that a line takes with its columns.
template <int FORMAT, int RT, int NB, bool HALF = false>
constexpr int kLineBytes = RT * (HALF ? 1024 : 2048) + NB * kHeld<FORMAT, NB> * 1024;

// HALF: rows 8 .. 15 of the tiles do not exist, and what the product has in their
// places is dropped.
template <int FORMAT, int RT, int NB, bool HALF = false>
struct Product {
    using P = Format<FORMAT>;
    static constexpr int G = (NB + 1) / 2;  // groups of 16 columns
    // lines in flight: 8 KB of weights where the columns leave the registers for it
    static constexpr int CH = std::max(1, std::min((HALF ? 8 : 4) / RT, 8 / (NB * kHeld<FORMAT, NB>)));
    static constexpr int kParts = kHeld<FORMAT, NB>;
    struct Line {
        u32x4 w[RT][HALF ? 1 : 2], x[NB][kParts];
    };

    const Tiles& tiles;
    const char* const (&x)[NB];  // this lane's unit of part 0 of column 8 j + lane / 8
    int columns, l0, l1, lines;
    char* lds;
    int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, i8 = lane >> 3, p8 = lane & 7;

    // the last line of a row is half a line: units 4 .. 7 of it would be the next row's
    __device__ __forceinline__ bool half(int l) const { return P::kOdd && l == lines - 1; }

    __device__ __forceinline__ static u32x4 load_unit(const char* p) {
        const u32x4* u = reinterpret_cast<const u32x4*>(p);
        if constexpr (P::kOdd)
            return *u;
        else
            return __builtin_nontemporal_load(u);
    }

    __device__ __forceinline__ void load_weights(Line& v, int l) const {
        const int64_t at = i8 * tiles.pitch + (int64_t)l * 128 + (half(l) ? p8 & 3 : p8) * 16;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            v.w[t][0] = load_unit(tiles.w0 + t * tiles.next + at);
            if (!HALF) v.w[t][HALF ? 0 : 1] = load_unit(tiles.w1 + t * tiles.next + at);
        }
    }
    // part k of the columns
    __device__ __forceinline__ void load_columns(Line& v, int l, int k) const {
        const int64_t at = ((int64_t)l * P::kParts + (half(l) ? 0 : k)) * 128;
#pragma unroll
        for (int j = 0; j < NB; ++j) v.x[j][k % kParts] = *reinterpret_cast<const u32x4*>(x[j] + at);
    }

    // lane 4 i + p loads the four scales of row i and pair p, a (tile, line) of a
    // batch of CH lines from l: the lanes of a row's neighbouring lines share a lookup
    __device__ __forceinline__ uint32_t load_scales(int l) const {
        if constexpr (!P::kScaled) return 0;
        static_assert(!P::kScaled || (CH * RT <= 4 && !HALF), "four pairs of whole tiles at most");
        const int t = min((lane & 3) / CH, RT - 1), at = min(l + (lane & 3) % CH, l1 - 1);
        const uint8_t* p = (lane < 32 ? tiles.s0 : tiles.s1) + ((lane >> 2) & 7) * (tiles.pitch / 32) + t * (tiles.next / 32) + 4 * at;
        if constexpr (!P::kOdd) return *reinterpret_cast<const uint32_t*>(p);
        const uint16_t *lo = reinterpret_cast<const uint16_t*>(p), *hi = lo + (at == lines - 1 ? 0 : 1);
        return *lo | (uint32_t)*hi << 16;
    }

    // The products of line l, held in v and number i of its batch; v then holds
    // line `next` if there is one (a wavefront's LDS accesses stay in order).
    __device__ __forceinline__ void step(Line& v, int l, int i, uint32_t scales, int next, f32x4 (&acc)[RT][G]) const {
        char* to = lds + i8 * 128 + (p8 ^ i8) * 16;
        constexpr int kColumns = RT * (HALF ? 1024 : 2048);  // their place behind the weights
        const char *row = lds + (HALF ? 0 : r >> 3) * 1024 + (r & 7) * 128, *column = lds + kColumns;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            *reinterpret_cast<u32x4*>(to + t * 2048) = v.w[t][0];
            if (!HALF) *reinterpret_cast<u32x4*>(to + t * 2048 + 1024) = v.w[t][HALF ? 0 : 1];
        }
        uint32_t four[RT] = {};
        if constexpr (P::kScaled)
#pragma unroll
            for (int t = 0; t < RT; ++t) four[t] = (uint32_t)__shfl((int)scales, 4 * r + t * CH + i);
        // halves of the line: both at once, or one after the other
        constexpr int kAtOnce = kParts == P::kParts ? 2 : 1;
#pragma unroll
        for (int k0 = 0; k0 < 2; k0 += kAtOnce) {
#pragma unroll
            for (int k = 0; k < kParts; ++k)
#pragma unroll
                for (int j = 0; j < NB; ++j) *reinterpret_cast<u32x4*>(to + kColumns + (j * kParts + k) * 1024) = v.x[j][k];
            // loads arrive in the order asked for: what this line still needs comes first
            if (kAtOnce == 1 && k0 == 0) load_columns(v, l, 1);
            if (k0 == 0 && next >= 0) load_weights(v, next);
            if (kAtOnce == 2) {
                if (next >= 0)
#pragma unroll
                    for (int k = 0; k < kParts; ++k) load_columns(v, next, k);
            } else if (k0 == 1 && next >= 0) {
                load_columns(v, next, 0);
            }
            __builtin_amdgcn_wave_barrier();
            if (k0 == 1 && half(l)) break;
            u32x4 b[kAtOnce][G][P::kReads], w[RT][kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const int c = min(16 * g + r, columns - 1);  // columns past the last repeat it, and are dropped
#pragma unroll
                    for (int j = 0; j < P::kReads; ++j)
                        b[k][g][j] = *reinterpret_cast<const u32x4*>(column + ((c >> 3) * kParts + k % kParts) * 1024 + (c & 7) * 128 +
                                                                     (P::unit(k0 + k, j, q) ^ (c & 7)) * 16);
                }
#pragma unroll
                for (int t = 0; t < RT; ++t)
                    w[t][k] = *reinterpret_cast<const u32x4*>(row + t * 2048 + ((q + 4 * (k0 + k)) ^ (r & 7)) * 16);
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (k == 1 && half(l)) break;
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int g = 0; g < G; ++g) acc[t][g] = P::mul(w[t][k], four[t], k0 + k, b[k][g], acc[t][g]);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }

    // acc[t][g] += lines l0 .. l1 of `lines` of tile t times columns 16 g .. of
    // `columns` (at least 1).
    __device__ __forceinline__ void run(f32x4 (&acc)[RT][G]) const {
        if (l0 >= l1) return;
        Line v[CH];
        uint32_t scales = load_scales(l0);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int l = min(l0 + i, l1 - 1);
            load_weights(v[i], l);
#pragma unroll
            for (int k = 0; k < kParts; ++k) load_columns(v[i], l, k);
        }
        int l = l0;
        for (; l + 2 * CH <= l1; l += CH) {
            const uint32_t next = load_scales(l + CH);
#pragma unroll
            for (int i = 0; i < CH; ++i) step(v[i], l + i, i, scales, l + i + CH, acc);
            scales = next;
        }
        const uint32_t next = l + CH < l1 ? load_scales(l + CH) : 0;
#pragma unroll
        for (int i = 0; i < 2 * CH - 1; ++i)
            if (l + i < l1) step(v[i % CH], l + i, i % CH, i < CH ? scales : next, l + i + CH < l1 ? l + i + CH : -1, acc);
    }
};

__device__ inline float silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// fp32 as the sum of three bf16 numbers, exactly but for its last bit or two:
// the intermediate loses nothing on the bf16 matrix core.  Rounded to bf16, the
// tiles would take a third of the columns; its error, 2^-9 of each product, would be
// the largest of the whole layer.
__device__ inline void split3(float v, __bf16* p) {
    p[0] = (__bf16)v;
    const float r = fabsf((float)p[0]) < INFINITY ? v - (float)p[0] : 0.0f;
    p[1] = (__bf16)r;
    p[2] = (__bf16)(r - (float)p[1]);
}

template <int FORMAT, int RT, int NB>
__device__ __forceinline__ void up_product(const MoeArgs& a, const uint8_t* token, int first, int n, const Tiles& tiles, int l0, int l1, int lines,
                                           char* lds, f32x4 (*red)[64]) {
    using P = Format<FORMAT>;
    const int lane = threadIdx.x & 63, i8 = lane >> 3;
    const char* x[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j)
        x[j] = (a.h8 ? reinterpret_cast<const char*>(a.x) : static_cast<const char*>(a.h)) +
               (token ? token[8 * j + i8] : first) * (a.h8 ? (int64_t)a.d : a.h_stride) * P::kBytes + (lane & 7) * 16;
    f32x4 acc[RT][1] = {};
    Product<FORMAT, RT, NB>{tiles, x, n, l0, l1, lines, lds}.run(acc);
#pragma unroll
    for (int t = 0; t < RT; ++t) red[t][lane] = acc[t][0];
}

// Gate and up projections and the SwiGLU product: a tile is eight rows of W_gate
// and the same eight of W_up; a workgroup takes RT of them, its wavefronts a
// quarter of the sum each.  EACH: every (token, selected expert) is a unit of its
// own: each wavefront finds its expert from the token's logits, which takes less
// than the plan's launch, and one per token leaves the units for the down
// projection.
// Bound by HBM from some 200 MB on, by the start and the end of the stream below.
// Split over the sum, so that one token's experts too (eight of 96 tiles at F = 768)
// give every CU three workgroups.
// grid: x = F / (8 RT), y = units
template <int FORMAT, int RT, bool EACH>
__global__ __launch_bounds__(kThreads, 4) void moe_up_kernel(MoeArgs a) {
    using P = Format<FORMAT>;
    __shared__ __align__(16) char lds[kWaves][kLineBytes<FORMAT, RT, EACH ? 1 : 2>];
    __shared__ f32x4 red[kWaves][RT][64];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    MoeUnit* unit = a.plan->unit + blockIdx.y;
    int expert, n, row0, first = 0;  // first: its token, where there is no plan
    if constexpr (EACH) {
        const int k = blockIdx.y % a.K;
        first = blockIdx.y / a.K;
        if (first >= live_tokens(a)) return;
        const bool write = blockIdx.x == 0 && k == 0 && wv == 0;
        const int e = select_experts(a, first, lane, write ? a.K : k + 1, write);
        if (write && lane < a.K) {
            unit[lane].expert = e;
            unit[lane].n = e >= 0;
        }
        expert = __builtin_amdgcn_readlane(e, k);
        n = expert >= 0;
        row0 = blockIdx.y;
    } else {
        expert = unit->expert;
        n = unit->n;
        row0 = unit->row;
    }
    if (n == 0) return;
    const int64_t pitch = (int64_t)a.d * 128 / P::kLine;  // bytes of a weight row
    const int64_t row = (int64_t)expert * 3 * a.F + blockIdx.x * (8 * RT);
    Tiles tiles;
    tiles.w0 = static_cast<const char*>(a.experts) + row * pitch;
    tiles.w1 = tiles.w0 + a.F * pitch;
    tiles.s0 = P::kScaled ? a.scales + row * (pitch / 32) : nullptr;
    tiles.s1 = P::kScaled ? tiles.s0 + a.F * (pitch / 32) : nullptr;
    tiles.pitch = pitch;
    tiles.next = 8 * pitch;
    const int lines = (a.d + P::kLine - 1) / P::kLine, l0 = wv * lines / kWaves, l1 = (wv + 1) * lines / kWaves;
    if constexpr (EACH)
        up_product<FORMAT, RT, 1>(a, nullptr, first, 1, tiles, l0, l1, lines, lds[wv], red[wv]);
    else if (n <= 8)
        up_product<FORMAT, RT, 1>(a, unit->token, 0, n, tiles, l0, l1, lines, lds[wv], red[wv]);
    else
        up_product<FORMAT, RT, 2>(a, unit->token, 0, n, tiles, l0, l1, lines, lds[wv], red[wv]);
    __syncthreads();
    // lane (c, q) of a product holds rows 4 q .. of column c: q = 0, 1 W_gate's, 2, 3 W_up's
    if (wv >= RT || lane >= 32 || r >= n) return;
    f32x4 g = red[0][wv][lane], u = red[0][wv][lane + 32];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) {
        g += red[k][wv][lane];
        u += red[k][wv][lane + 32];
    }
    const int64_t at = row0 + r;
    const int f = (blockIdx.x * RT + wv) * 8 + (lane >> 4) * 4;
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
            *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.act) + (at * 3 + i) * a.F + f) = bf16x4{p[0][i], p[1][i], p[2][i], p[3][i]};
    }
}

// y: the gated sum over a token's experts in descending logit.  A launch's 4.5 us:
// what it reads was just written.  The order of the sum is fixed, which atomics in the
// down projection would not give.
// grid: x = d / (4 kThreads) rounded up, y = tokens
__global__ __launch_bounds__(kThreads) void moe_sum_kernel(MoeArgs a) {
    const int t = blockIdx.y, j = (blockIdx.x * kThreads + threadIdx.x) * 4;
    if (t >= live_tokens(a) || j >= a.d) return;
    constexpr int kBatch = 8;  // experts whose outputs are loaded together
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < a.K; k0 += kBatch) {
        f32x4 o[kBatch];
        float g[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = t * a.K + min(k0 + k, a.K - 1);
            g[k] = k0 + k < a.K ? a.gate[i] : -1.0f;
            o[k] = *reinterpret_cast<const f32x4*>(a.out + (int64_t)i * a.d + j);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (!(g[k] < 0.0f)) y += g[k] * o[k];  // what is not selected was not written either
    }
    *reinterpret_cast<f32x4*>(a.y + (int64_t)t * a.y_stride + j) = y;
}

// The down product of a unit in NB blocks of 8 columns: column i is bf16 number
// i / n of token i % n's intermediate, so that up to five tokens take one group
// of 16.
template <int FORMAT, int RT, int NB>
__device__ __forceinline__ void down_product(const MoeArgs& a, int row, int n, const Tiles& tiles, int l0, int l1, int lines,
                                             char* lds, f32x4 (*red)[Format<FORMAT>::kPlanes][64]) {
    using P = Format<FORMAT>;
    constexpr int G = (NB + 1) / 2;
    const int lane = threadIdx.x & 63, i8 = lane >> 3, columns = P::kPlanes * n;
    const char* x[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int i = min(8 * j + i8, columns - 1), plane = (i >= n) + (i >= 2 * n);
        x[j] = static_cast<const char*>(a.act) + ((int64_t)(row + i - plane * n) * P::kPlanes + plane) * a.F * P::kBytes + (lane & 7) * 16;
    }
    f32x4 acc[RT][G] = {};
    Product<FORMAT, RT, NB>{tiles, x, columns, l0, l1, lines, lds}.run(acc);
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int g = 0; g < G; ++g) red[t][g][lane] = acc[t][g];
}

// The weights of W_down's rows row0 .. of an expert.
template <int FORMAT>
__device__ __forceinline__ Tiles down_tiles(const MoeArgs& a, int expert, int row0) {
    using P = Format<FORMAT>;
    const int64_t pitch = (int64_t)a.F * 128 / P::kLine;
    const int64_t before = ((int64_t)expert * 3 + 2) * a.F * ((int64_t)a.d * 128 / P::kLine) + row0 * pitch;
    Tiles t;
    t.w0 = static_cast<const char*>(a.experts) + before;
    t.w1 = t.w0 + 8 * pitch;
    t.s0 = P::kScaled ? a.scales + before / 32 : nullptr;
    t.s1 = P::kScaled ? t.s0 + 8 * (pitch / 32) : nullptr;
    t.pitch = pitch;
    t.next = 16 * pitch;
    return t;
}

// Down projection and gated sum of a token: a workgroup takes a tile of outputs,
// its wavefronts a part of an expert's sum each, `split` parts.  HALF: half tiles,
// where whole ones leave many CUs without a workgroup (half_tiles).
// grid: x = d / kTile, y = tokens
template <bool HALF>
struct One {
    static constexpr int kTile = HALF ? 8 : 16, kThreads = HALF ? 512 : 1024, kWaves = kThreads / 64;
};

template <int FORMAT, bool HALF>
__global__ __launch_bounds__(One<HALF>::kThreads) void moe_down_one_kernel(MoeArgs a, int split) {
    using P = Format<FORMAT>;
    using O = One<HALF>;
    __shared__ __align__(16) char lds[O::kWaves][kLineBytes<FORMAT, 1, 1, HALF>];
    __shared__ __align__(16) float red[kMaxK][O::kTile];  // K split is at most kWaves, or K
    __shared__ float gate[kMaxK];                         // its product of an expert that is not selected is 0
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lines = (a.F + P::kLine - 1) / P::kLine;
    const int first = blockIdx.y * a.K;  // the token's first unit
    if ((int)blockIdx.y >= live_tokens(a)) return;
    if (threadIdx.x < a.K) gate[threadIdx.x] = a.gate[first + threadIdx.x];
    for (int job = wv; job < a.K * split; job += O::kWaves) {
        const int k = job / split, part = job % split;
        const MoeUnit& unit = a.plan->unit[first + k];
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (unit.n != 0) {
            const char* x[1] = {static_cast<const char*>(a.act) +
                                ((int64_t)(first + k) * P::kPlanes + min(lane >> 3, P::kPlanes - 1)) * a.F * P::kBytes + (lane & 7) * 16};
            f32x4 acc[1][1] = {};
            const Tiles tiles = down_tiles<FORMAT>(a, unit.expert, blockIdx.x * O::kTile);
            Product<FORMAT, 1, 1, HALF>{tiles, x, P::kPlanes, part * lines / split, (part + 1) * lines / split, lines, lds[wv]}.run(acc);
            v = acc[0][0];
            if constexpr (P::kPlanes == 3)  // columns 0, 1, 2, the smallest first
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = (__shfl(v[j], lane + 2) + __shfl(v[j], lane + 1)) + v[j];
        }
        const int i = 4 * (lane >> 4);
        if ((lane & 15) == 0 && i < O::kTile) *reinterpret_cast<f32x4*>(&red[job][i]) = v;
    }
    __syncthreads();
    if (threadIdx.x >= O::kTile) return;
    float y = 0.0f;
    for (int k = 0; k < a.K; ++k) {
        float o = 0.0f;
        for (int p = 0; p < split; ++p) o += red[k * split + p][threadIdx.x];
        y += gate[k] * o;
    }
    a.y[blockIdx.y * a.y_stride + blockIdx.x * O::kTile + threadIdx.x] = y;
}

// Down projection: the workgroup's wavefronts take RT tiles of 16 rows and a part
// of the sum each, `split` parts (1, 2 and 4 parts take 63 to 65 us at 61 tokens of
// 128 x 2048 x 768; at 61 tokens the rule takes 1).  Bound by HBM and by the
// columns, three for each token: read through the caches, into LDS and out again.
// Without their loads (61 tokens bf16, 64 tokens 8 bits) it takes 58 and 135
// instead of 63 and 161 us.  Six and more tokens of an expert with 8-bit weights
// hold one half of a line's columns at a time; both at once spill: 221 us.
// grid: x = d / 16 / (RT kWaves / split) rounded up, y = units
template <int FORMAT, int RT>
__global__ __launch_bounds__(kThreads, 3) void moe_down_kernel(MoeArgs a, int split) {
    using P = Format<FORMAT>;
    constexpr int kGroups = P::kPlanes, kBlocks = 2 * kGroups;
    // a line with its columns, then the products
    __shared__ __align__(16) char lds[kWaves][std::max(kLineBytes<FORMAT, RT, kBlocks>, RT * kGroups * 1024)];
    auto red = [&](int w) { return reinterpret_cast<f32x4(*)[kGroups][64]>(lds[w]); };
    const MoeUnit& unit = a.plan->unit[blockIdx.y];
    const int n = unit.n;
    if (n == 0) return;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int part = wv % split, tile0 = (blockIdx.x * (kWaves / split) + wv / split) * RT, all = a.d / 16;
    if (tile0 < all) {  // d / 16 is a multiple of RT
        const Tiles tiles = down_tiles<FORMAT>(a, unit.expert, tile0 * 16);
        const int lines = (a.F + P::kLine - 1) / P::kLine, l0 = part * lines / split, l1 = (part + 1) * lines / split;
        const int columns = P::kPlanes * n;
        if (columns <= 8)
            down_product<FORMAT, RT, 1>(a, unit.row, n, tiles, l0, l1, lines, lds[wv], red(wv));
        else if (columns <= 16)
            down_product<FORMAT, RT, 2>(a, unit.row, n, tiles, l0, l1, lines, lds[wv], red(wv));
        else if constexpr (kGroups > 1) {
            if (columns <= 32)
                down_product<FORMAT, RT, 4>(a, unit.row, n, tiles, l0, l1, lines, lds[wv], red(wv));
            else
                down_product<FORMAT, RT, 6>(a, unit.row, n, tiles, l0, l1, lines, lds[wv], red(wv));
        }
    }
    __syncthreads();
    // one wavefront per tile from here
    for (int t = part; t < RT; t += split) {
        const int tile = tile0 + t;
        if (tile >= all) return;
        if (r < n) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = P::kPlanes - 1; p >= 0; --p) {  // the smallest first
                const int i = p * n + r;
                for (int k = 0; k < split; ++k) v += red(wv - part + k)[t][i >> 4][16 * q + (i & 15)];
            }
            *reinterpret_cast<f32x4*>(a.out + (int64_t)unit.slot[r] * a.d + tile * 16 + 4 * q) = v;
        }
    }
}

template <bool BF16>
void launch_route(const MoeArgs& a, hipStream_t st) {
    const unsigned groups = (a.T + 7) / 8;
    if (a.T == 1)
        launch_kernel(moe_logits_kernel<BF16, 1, 1>, dim3(a.N, 1), dim3(kThreads), st, Timing{}, a);
    else if (a.T <= 16)
        launch_kernel(moe_logits_kernel<BF16, 1, 4>, dim3(a.N, (a.T + 3) / 4), dim3(kThreads), st, Timing{}, a);
    else
        launch_kernel(moe_logits_kernel<BF16, 4, 8>, dim3((a.N + 3) / 4, groups), dim3(kThreads), st, Timing{}, a);
}

// Few tokens of many experts: hardly two of them share one, and the plan's and the
// gated sum's launches take longer than reading a shared expert's weights twice, as
// long as the weights are not so many that the tiles of the joint launches stream
// them faster.  Joint / each alone, us a layer, through so many layers that every
// weight comes from HBM (MB: of the weights of all rows):
//   top-8 of 128, 2048 x 768    bf16: 1 to 4 tokens (76 to 302 MB) 28.4 / 22.5, 40.7 / 35.8, 51.6 / 52.3, 62.1 / 59.4
//                             8 bits: 1 to 4 (38 to 151 MB) 26.3 / 20.6, 32.1 / 27.6, 37.6 / 40.2, 41.7 / 47.3
//                               fp32: 1 to 4 (151 to 604 MB) 42.7 / 38.8, 63.6 / 58.8, 89.0 / 85.5, 107 / 106
//   top-6 of 256, 1024 x 512, 4 tokens  bf16 32.0 / 24.2, 8 bits 29.5 / 23.3, fp32 41.8 / 35.8 (75, 38, 151 MB)
//   top-8 of 128, 4096 x 1536   bf16: 1, 2, 4 (302, 604, 1208 MB) 62.5 / 57.7, 105 / 102, 188 / 192
//                             8 bits: 1, 2 (151, 302 MB) 44.9 / 41.4, 67.5 / 73.1; fp32: 1, 2 (604, 1208 MB) 118 / 113, 207 / 211
//   top-4 of 32, 2880 x 2880    bf16: 1, 2 (199, 398 MB) 46.2 / 42.8, 75.2 / 76.5; 8 bits: 1, 2 (100, 199 MB) 38.9 / 34.4, 56.3 / 57.3
//                               fp32: 1, 2 (398, 796 MB) 79.0 / 76.2, 135 / 151
bool each_alone(const MoeArgs& a) {
    const int64_t rows = (int64_t)a.T * a.K, values = rows * 3 * a.d * a.F;
    const int64_t bytes = a.format == kMoeMx8 ? values : a.format == kMoeBf16 ? 2 * values : 4 * values;
    return a.T == 1 || (a.T <= 4 && 4 * rows <= a.N && bytes <= (a.format == kMoeMx8 ? 96 : 512) * 1000000ll);
}

// The two products, with their variants for rows of whole lines or not.
template <int FORMAT, int RT, bool EACH>
void launch_up(const MoeArgs& a, int units, hipStream_t st) {
    launch_kernel(moe_up_kernel<FORMAT, RT, EACH>, dim3(a.F / (8 * RT), units), dim3(kThreads), st, Timing{}, a);
}

// Half tiles for weights of 16 and 32 bits and fewer than 160 whole ones.  Half / whole,
// us a layer on cold weights, bf16 and fp32: 1 token of d = 1024 (64 tiles) 15.0 / 15.6
// and 22.3 / 22.3, of 2048 (128) 22.5 / 23.8 and 37.5 / 38.7, of 2880 (180) 46.2 / 42.5 and
// 86.9 / 78.9, of 4096 (256) 59.7 / 58.1 and 116 / 109.  Half tiles of 8-bit weights put
// too few bytes in flight (2880 x 2880, four experts: the launch 14.3 us against 16.6).
bool half_tiles(const MoeArgs& a) { return a.format != kMoeMx8 && a.d / 16 * a.T < 160; }

template <int FORMAT, bool HALF>
void launch_down_one(const MoeArgs& a, hipStream_t st) {
    using O = One<HALF>;
    const int lines = (a.F + Format<FORMAT>::kLine - 1) / Format<FORMAT>::kLine;
    int split = 1;
    while (2 * split * a.K <= O::kWaves && 2 * split <= lines) split *= 2;
    launch_kernel(moe_down_one_kernel<FORMAT, HALF>, dim3(a.d / O::kTile, a.T), dim3(O::kThreads), st, Timing{}, a, split);
}

template <int FORMAT, int RT>
void launch_down(const MoeArgs& a, int units, hipStream_t st) {
    const int lines = (a.F + Format<FORMAT>::kLine - 1) / Format<FORMAT>::kLine;
    // parts of the sum: four lines at least, more parts where the tiles alone do not
    // fill the device
    int split = lines >= 32 ? 4 : lines >= 16 ? 2 : 1;
    while (split < kWaves && (int64_t)(a.d / 16) * units * split < 4096) split *= 2;
    const int tiles = RT * kWaves / split;
    launch_kernel(moe_down_kernel<FORMAT, RT>, dim3((a.d / 16 + tiles - 1) / tiles, units), dim3(kThreads), st, Timing{}, a, split);
}

// UP, DOWN: the formats of W_gate's and W_up's rows and of W_down's.
template <int UP, int DOWN>
void launch_experts(const MoeArgs& a, hipStream_t st) {
    const int rows = a.T * a.K, units = moe_max_units(rows, a.N);
    if (each_alone(a)) {
        launch_up<UP, 1, true>(a, rows, st);
        if constexpr (!Format<DOWN>::kScaled) {
            if (half_tiles(a)) {
                launch_down_one<DOWN, true>(a, st);
                return;
            }
        }
        launch_down_one<DOWN, false>(a, st);
        return;
    }
    if (a.T > 2 * kPlanThreads / 64) {
        launch_kernel(moe_select_kernel, dim3(a.T), dim3(64), st, Timing{}, a);
        launch_kernel(moe_plan_kernel<true>, dim3(1), dim3(kPlanThreads), st, Timing{}, a);
    } else {
        launch_kernel(moe_plan_kernel<false>, dim3(1), dim3(kPlanThreads), st, Timing{}, a);
    }
    if ((int64_t)(a.F / 16) * units < 1024) {  // few tiles: one for each wavefront
        launch_up<UP, 1, false>(a, units, st);
        launch_down<DOWN, 1>(a, units, st);
    } else {
        launch_up<UP, 2, false>(a, units, st);
        launch_down<DOWN, 2>(a, units, st);
    }
    launch_kernel(moe_sum_kernel, dim3((a.d / 4 + kThreads - 1) / kThreads, a.T), dim3(kThreads), st, Timing{}, a);
}

}  // namespace

hipError_t launch_moe(const MoeArgs& a, hipStream_t st) {
    if (a.bf16)
        launch_route<true>(a, st);
    else
        launch_route<false>(a, st);
    if (a.format == kMoeF32)
        launch_experts<kMoeF32, kMoeF32>(a, st);
    else if (a.format == kMoeBf16)
        launch_experts<kMoeBf16, kMoeBf16>(a, st);
    else if (a.d % 128 == 0)
        a.F % 128 == 0 ? launch_experts<kMoeMx8, kMoeMx8>(a, st) : launch_experts<kMoeMx8, kMoeMx8Odd>(a, st);
    else
        a.F % 128 == 0 ? launch_experts<kMoeMx8Odd, kMoeMx8>(a, st) : launch_experts<kMoeMx8Odd, kMoeMx8Odd>(a, st);
    return hipGetLastError();
}

}  // namespace cmoe
