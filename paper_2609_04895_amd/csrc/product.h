// product.h - matrix products grouped by expert: rows first[e] .. first[e + 1] of y
// are W_e times as many rows of x,
//
//   y[i] = W_e x[r(i)],  or with SwiGLU  y[i] = silu(G_e x[r(i)]) * (U_e x[r(i)]),
//
// r(i) the row itself or x_row[i].  Compiled once for each kind of x
// (product_f32.hip, product_bf16.hip, product_mx8.hip).
#pragma once

#include <type_traits>
#include <utility>

#include "cmoe_internal.h"
#include "mx4.h"

namespace cmoe {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- weights' forms
// Sixteen 8-bit values of one block as bf16, exact from 2^-126 on.
__device__ inline void widen8(const u32x4& q, uint32_t byte, u32x4 (&to)[2]) {
    const float s = mx_scale(byte);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        to[j / 2][2 * (j % 2)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[j], s, false));
        to[j / 2][2 * (j % 2) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[j], s, true));
    }
}

// Eight 4-bit values as bf16.
__device__ inline u32x4 widen4(uint32_t q, float s) {
    u32x4 v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 0));
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 1));
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 2));
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, s, 3));
    return v;
}

// f(0) .. f(N - 1) as constants, in straight code however long it gets: registers have no
// index at run time.
template <typename F, int... I>
__device__ __forceinline__ void repeat(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void repeat(F&& f) {
    repeat(f, std::make_integer_sequence<int, N>{});
}

// Halves of 32 values that share a power of two, for outputs that are only added up
// once more: 11 bits of each, so off by at most 2^-11 of its value (2^-39 of the block's
// largest where that is more) against 2^-8 for bf16, at the same bytes; infinities and NaN
// stay for themselves.  byte: the exponent field of the largest finite value, which
// becomes 2^14 .. 2^15.
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
constexpr uint32_t kHalfLeast = 15;
__device__ inline float half_inverse(uint32_t byte) { return __uint_as_float((268u - byte) << 23); }

__device__ inline float silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// ---------------------------------------------------------------- outputs
// Scale byte of a row's 32 values as halves: the exponent of the largest finite one.
__device__ __forceinline__ uint32_t half_scale(const f32x4 (&v)[2]) {
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t e = __float_as_uint(v[p][k]) >> 23 & 255u;
            top = max(top, e == 255 ? 0u : e);
        }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    return max(top, kHalfLeast);
}

// Columns col .. col + 3 and 16 behind them of row `at` of y; the four lanes of a row hold
// 32 columns.
__device__ __forceinline__ void put32(const ProductArgs& a, const f32x4 (&v)[2], int64_t at, int col, bool live) {
    const int q = (threadIdx.x & 63) >> 4;
    if (a.y_kind == kProductMx8) {
        float top = 0.0f;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int k = 0; k < 4; ++k) top = mx_max(top, v[p][k]);
        top = mx_max(top, __shfl_xor(top, 16));
        top = mx_max(top, __shfl_xor(top, 32));
        const uint32_t byte = mx_scale_byte(top);
        const float inv = mx_inverse(byte);
        if (live && col < a.m) {
            uint8_t* y = static_cast<uint8_t*>(a.y) + at * a.y_stride + col;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const uint32_t e = byte == kMxBad ? kMxNaN2 * 0x10001u
                                                  : mx_pair<true>(v[p][2], v[p][3], inv, mx_pair<false>(v[p][0], v[p][1], inv, 0));
                *reinterpret_cast<uint32_t*>(y + 16 * p) = e;
            }
            if (q == 0) a.y_scale[at * a.y_scale_stride + col / 32] = (uint8_t)byte;
        }
    } else if (a.y_kind == kProductHalf) {
        const uint32_t byte = half_scale(v);
        const float inv = half_inverse(byte);
        if (live && col < a.m) {
            _Float16* y = static_cast<_Float16*>(a.y) + at * a.y_stride + col;
#pragma unroll
            for (int p = 0; p < 2; ++p)
                *reinterpret_cast<half4*>(y + 16 * p) =
                    half4{(_Float16)(v[p][0] * inv), (_Float16)(v[p][1] * inv), (_Float16)(v[p][2] * inv), (_Float16)(v[p][3] * inv)};
            if (q == 0) a.y_scale[at * a.y_scale_stride + col / 32] = (uint8_t)byte;
        }
    } else if (live) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int c = col + 16 * p;
            if (a.y_kind == kProductBf16) {
                __bf16* y = static_cast<__bf16*>(a.y) + at * a.y_stride + c;
                if (a.y_aligned && c + 3 < a.m)
                    *reinterpret_cast<bf16x4*>(y) = bf16x4{(__bf16)v[p][0], (__bf16)v[p][1], (__bf16)v[p][2], (__bf16)v[p][3]};
                else
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (c + k < a.m) y[k] = (__bf16)v[p][k];
            } else {
                float* y = static_cast<float*>(a.y) + at * a.y_stride + c;
                if (a.y_aligned && c + 3 < a.m)
                    *reinterpret_cast<f32x4*>(y) = v[p];
                else
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (c + k < a.m) y[k] = v[p][k];
            }
        }
    }
}

// ---------------------------------------------------------------- the kernel
// A workgroup computes BM rows by BN weight rows, its WM x WN wavefronts a part each,
// in steps of 128 bytes of a row of x.  Operands go straight from memory into LDS as they
// are.  Weights of fewer bits than x come 128 bytes of a row at a time too, which last
// two steps or four, and are widened to bf16 as they are read from LDS; with 8-bit x the
// matrix core takes 4 bits as they are.  A row's 128 bytes are eight units of 16; unit p
// of row i lies at place p ^ (i & 7), so that the reads of the operands (lane (r, q) =
// 16 q + r reads a unit of row r) meet no LDS bank twice.
//
// What bounds it: matrix instructions where a group has many rows, the weights' way from
// HBM where it has few, and in between the two do not overlap in full: a tile's first
// loads and its stores stand alone, with one workgroup on a CU.  One group of 8192 cubed
// runs at 1184 TFLOP/s in bf16 (a library product: 1370), 1660 to 1914 in 8 bits and 1271
// with 4-bit weights; 128 groups of 256 rows by 1536 x 2048, every weight out of HBM,
// at 911 and 1373 in bf16 and 8 bits.  Found on the way there, at these two shapes in
// bf16: operands through registers, two steps of LDS, 930 us and 245; straight into LDS,
// weights asked for two steps ahead and not one, 867 and 239; whole lines of y, by way
// of LDS, 942 and 232; workgroups that go on from tile to tile with the next one's loads
// in flight 1069 and 311 (their stores of y are then waited for with the loads).  Eight
// wavefronts of 128 x 64, not four of 128 x 128: 931 against 1178 us.  Packed weights in
// pieces of a step, 32 or 64 bytes of a row, not 128 at a time: 8 bits, 128 x (1536 x
// 2048), 1024 rows 98 / 81 us, 4000 rows 114 / 94; 4 bits with 8-bit rows, 32 x (2880 x
// 2880), 256 rows 90 / 77.  With 4-bit weights and bf16 rows, 32 x 125 rows by 5760 x 2880,
// in 209 us, the products and the widening alone take 159 and the loads alone 162.
//
// In 8 bits the instruction adds the 32 products of a pair of scales with 13 bits below
// the largest (1 + 2^-12 is kept, 1 + 2^-14 is 1), and what it gives for each 32 in
// fp32.  With e4m3 values of normal rows that is 1.5e-5 of the result, rms, a hundredth
// of the rounding to bf16 that follows, at twice the rate of the bf16 core, on which
// the same products would be exact.
//
// SWIGLU: a tile's weight rows alternate, 32 of G and the same 32 of U, so that a lane
// holds both factors of its outputs.
//
// EXACT, for 8-bit rows: both operands become bf16 as they are read, and the bf16 core
// multiplies.  Where y is in 8 bits a value next to the middle of a step would else go to
// either side, a sixteenth of itself away, for a sum that is off by 1e-5.
template <int KIND, int HELD, int BM, int BN, int WM, int WN, bool SWIGLU, bool EXACT>
struct ProductTile {
    static constexpr int NT = 64 * WM * WN, TM = BM / 16 / WM, TN = BN / 16 / WN;
    static constexpr bool kScaled = KIND == kProductMx8;
    static constexpr int kValues = KIND == kProductF32 ? 32 : KIND == kProductBf16 ? 64 : 128;  // of a step
    // bytes of a weight row per step, 16-byte units of them, and units per thread
    static constexpr int kWBytes = HELD == kHeldSame ? 128 : HELD == kHeld8 ? kValues : kValues / 2;
    static constexpr int kWUnits = kWBytes / 16;
    static constexpr int G = 8 / kWUnits;  // steps that 128 bytes of a weight row last, which are loaded together
    static constexpr int XI = BM * 8 / NT, WI = BN * 8 / NT;
    static constexpr bool kPacked = HELD != kHeldSame;  // weights of fewer bits than x
    static constexpr bool kWiden = kPacked && !kScaled;  // that become bf16
    // rows whose scales a thread keeps, 16 bytes of each at a time, and the steps they last
    static constexpr int SI = ((kScaled ? BM : 0) + BN + NT - 1) / NT;
    static constexpr int kBatch = kWiden ? 8 : 4;
    static_assert(XI * NT == BM * 8 && WI * NT == BN * 8, "whole loads");
    static_assert(!SWIGLU || TN % 4 == 0, "G and U in one wavefront");
    static_assert(TN % 2 == 0, "blocks of 32 outputs in one wavefront");

    // LDS: rows of x of two steps; 128 bytes of the weight rows three times, or
    // twice where they last several steps; two steps' scales, four bytes of each row, of x
    // first, or two of each weight row.
    static constexpr int kXSlots = 2, kWSlots = kPacked ? 2 : 3;
    static constexpr int kAtW = kXSlots * BM * 128, kAtScale = kAtW + kWSlots * BN * 128;
    static constexpr int kScaleBytes = kScaled ? (BM + BN) * 4 : kWiden ? BN * 2 : 0;
    static constexpr int kBytes = kAtScale + 2 * kScaleBytes;

    const ProductArgs& a;
    const char* px[XI];
    const char* pw[WI];
    const uint8_t* ps[kPacked || kScaled ? SI : 1];
    int steps;
    bool tail;  // the last step is half of one (8 bits only)
    int tid = threadIdx.x, lane = tid & 63, r = lane & 15, q = lane >> 4;
    int wv = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wv / WN, wn = wv % WN;

    // Row of W that row j of the tile holds; outputs behind the last one repeat it.
    __device__ __forceinline__ static int64_t weight_row(const ProductArgs& a, int c0, int j) {
        if constexpr (SWIGLU)
            return (int64_t)((j >> 5) & 1) * a.m + min(c0 + (j >> 6) * 32 + (j & 31), a.m - 1);
        else
            return min(c0 + j, a.m - 1);
    }
    // Row of x for row i of y.
    __device__ __forceinline__ static int64_t source_row(const ProductArgs& a, int i) {
        if (!a.x_row) return i;
        const int s = a.x_row[i];
        return (unsigned)s < (unsigned)a.x_rows ? s : 0;
    }
    // The unit that goes to place p of row j.
    __device__ __forceinline__ static int swizzle(int p, int j) { return p ^ (j & 7); }

    __device__ __forceinline__ ProductTile(const ProductArgs& args, int expert, int r0, int n, int c0) : a(args) {
        steps = (a.d + kValues - 1) / kValues;
        tail = kScaled && a.d % kValues != 0;
#pragma unroll
        for (int i = 0; i < XI; ++i) {
            const int j = i * (NT / 8) + (tid >> 3);
            px[i] = a.x + source_row(a, r0 + min(j, n - 1)) * a.x_pitch + swizzle(tid & 7, j) * 16;
        }
        const int64_t pitch = (int64_t)a.d / kValues * kWBytes + (kScaled ? a.d % kValues / (kValues / kWBytes) : 0);
        const char* w = a.w + expert * a.w_matrix;
        const uint8_t* ws = a.w_scale ? a.w_scale + expert * a.w_scale_matrix : nullptr;
#pragma unroll
        for (int i = 0; i < WI; ++i) {
            pw[i] = w + weight_row(a, c0, i * (NT / 8) + (tid >> 3)) * pitch;
        }
        if constexpr (kWiden)
#pragma unroll
            for (int i = 0; i < SI; ++i) ps[i] = ws + weight_row(a, c0, min(i * NT + tid, BN - 1)) * (a.d / 32);
        if constexpr (kScaled)
#pragma unroll
            for (int i = 0; i < SI; ++i) {
                const int j = min(i * NT + tid, BM + BN - 1);
                ps[i] = j < BM ? a.x_scale + source_row(a, r0 + min(j, n - 1)) * a.x_scale_pitch
                               : ws + weight_row(a, c0, j - BM) * (a.d / 32);
            }
    }

    // 16 bytes of each lane into LDS at byte `to`, one lane's behind the other's.  It has no
    // output register; arrive() waits for it.  As a builtin it would have every read of
    // LDS wait for all such loads, those of later steps too.  m0 is reserved: nothing else
    // here uses it, and a builtin that did would set it for itself.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    // ONCE: nontemporal.
    template <bool ONCE>
    __device__ __forceinline__ static void direct(const char* from, uint32_t to) {
        if constexpr (ONCE)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
                         : "m0");
        else
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from)
                         : "m0");
    }
#pragma clang diagnostic pop
    // All wavefronts have read what they need and their loads but the last LEFT have arrived.
    template <int LEFT>
    __device__ __forceinline__ static void arrive() {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
    }

    // Rows of x of step k, straight into LDS.  Of half a step, the units behind it are read
    // from its front, so that nothing behind the rows' ends is; their scales are 2^-127
    // each and make nothing of them.
    __device__ __forceinline__ void load_x(uint32_t lds, int k, int slot) const {
        const bool half = kScaled && tail && k == steps - 1;
        const uint32_t to = lds + slot * (BM * 128) + wv * 1024;
#pragma unroll
        for (int i = 0; i < XI; ++i) {
            const int at = half && swizzle(tid & 7, i * (NT / 8) + (tid >> 3)) >= 4 ? k * 128 - 64 : k * 128;
            direct<false>(px[i] + at, to + i * NT * 16);
        }
    }
    // Stretch g of 128 bytes of the weight rows, as they lie in memory.  What would lie behind
    // a row's end is read from its last unit, and not used or made nothing of.
    template <bool ONCE>
    __device__ __forceinline__ void load_w(uint32_t lds, int g, int slot) const {
        const uint32_t to = lds + kAtW + slot * (BN * 128) + wv * 1024;
        const int last = a.d / kValues * kWUnits + a.d % kValues * kWUnits / kValues - 1;
#pragma unroll
        for (int i = 0; i < WI; ++i) direct<ONCE>(pw[i] + min(g * 8 + swizzle(tid & 7, i * (NT / 8) + (tid >> 3)), last) * 16, to + i * NT * 16);
    }
    // Nontemporally where a group has one tile of rows, so that each weight is read once and
    // need not push rows of x out of the L2.  With and without, us: 128 groups of 256 rows
    // by 1536 x 2048 bf16 204 / 227, 8 bits 138 / 149, of 128 rows 158 / 185 and 91 / 108; one
    // group of 8192 cubed 948 / 924 and 624 / 574.
    __device__ __forceinline__ void load_w(uint32_t lds, int g, int slot) const {
        if (a.once)
            load_w<true>(lds, g, slot);
        else
            load_w<false>(lds, g, slot);
    }

    // Sixteen bytes of a row's scales, zeros behind its end.  They are waited for at once:
    // left open, the compiler, which does not see the loads into LDS, would wait for all of
    // those too in every step that might be the next to use a scale.
    __device__ __forceinline__ void load_scales(u32x4 (&s)[SI], int k) const {
        const int at = k / kBatch * 16, all = a.d / 32;
#pragma unroll
        for (int i = 0; i < SI; ++i) {
            if (at + 16 <= all) {
                __builtin_memcpy(&s[i], ps[i] + at, 16);
            } else {  // by twos, as d / 32 is even, and all at once
                uint16_t two[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) __builtin_memcpy(&two[j], ps[i] + min(at + 2 * j, all - 2), 2);
                s[i] = u32x4{};
#pragma unroll
                for (int j = 0; j < 8; ++j) s[i][j / 2] |= at + 2 * j < all ? (uint32_t)two[j] << (16 * (j & 1)) : 0;
            }
        }
#pragma unroll
        for (int i = 0; i < SI; ++i) asm volatile("" : "+v"(s[i]));
    }
    __device__ __forceinline__ static uint32_t word(const u32x4& s, int i) { return i == 0 ? s[0] : i == 1 ? s[1] : i == 2 ? s[2] : s[3]; }

    // Scales of step k into LDS.
    __device__ __forceinline__ void store_scales(const u32x4 (&s)[SI], char* lds, int k) const {
#pragma unroll
        for (int i = 0; i < SI; ++i) {
            const int j = i * NT + tid;
            char* to = lds + (kAtScale + (k & 1) * kScaleBytes + j * (kScaled ? 4 : 2));
            if constexpr (kScaled) {
                if (j < BM + BN) *reinterpret_cast<uint32_t*>(to) = word(s[i], k & 3);
            } else {
                if (j < BN) *reinterpret_cast<uint16_t*>(to) = (uint16_t)(word(s[i], (k >> 1) & 3) >> (16 * (k & 1)));
            }
        }
    }

    // 8-bit rows on the bf16 core: lane (r, q) has values 32 q .. of both operands, half of
    // them at a time.
    __device__ __forceinline__ void multiply_exact(f32x4 (&acc)[TN][TM], const char* from, int x, int sx, int w, int sw, int u0) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = swizzle(2 * q + h, r) << 4;
            u32x4 vx[TM][2];
#pragma unroll
            for (int i = 0; i < TM; ++i)
                widen8(*reinterpret_cast<const u32x4*>(from + (x + i * 2048 + at)), *reinterpret_cast<const uint8_t*>(from + (sx + i * 64)), vx[i]);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const uint32_t byte = *reinterpret_cast<const uint8_t*>(from + (sw + j * 64));
                u32x4 vw[2];
                if constexpr (kPacked) {
                    const u32x2 v = *reinterpret_cast<const u32x2*>(from + (w + j * 2048 + (swizzle(u0 + q, r) << 4) + h * 8));
                    const float f = mx_scale(byte);
                    vw[0] = widen4(v[0], f);
                    vw[1] = widen4(v[1], f);
                } else {
                    widen8(*reinterpret_cast<const u32x4*>(from + (w + j * 2048 + at)), byte, vw);
                }
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int i = 0; i < TM; ++i)
                        acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vw[p]), __builtin_bit_cast(bf16x8, vx[i][p]),
                                                                            acc[j][i], 0, 0, 0);
            }
        }
    }

    // acc[j][i] += weight tile j times row tile i over step k, its weights in `slot`.
    __device__ __forceinline__ void multiply(f32x4 (&acc)[TN][TM], const char* from, int k, int slot) const {
        const int x = (k & 1) * (BM * 128) + (wm * TM * 16 + r) * 128, w = kAtW + slot * (BN * 128) + (wn * TN * 16 + r) * 128;
        const int u0 = k % G * kWUnits;  // of the weight rows' 128 bytes, the step's first unit
        if constexpr (kScaled) {
            // the instruction takes values 16 q .. and 64 + 16 q .. of a row from lane (r, q),
            // and from the same lane the scale of values 32 q ..
            const int sx = kAtScale + (k & 1) * kScaleBytes + (wm * TM * 16 + r) * 4 + q, sw = kAtScale + (k & 1) * kScaleBytes + (BM + wn * TN * 16 + r) * 4 + q;
            auto operand = [&](int p, int t) {
                const u32x4 lo = *reinterpret_cast<const u32x4*>(from + (p + t * 2048 + ((q ^ (r & 7)) << 4)));
                u32x4 hi = *reinterpret_cast<const u32x4*>(from + (p + t * 2048 + (((q + 4) ^ (r & 7)) << 4)));
                return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
            };
            if constexpr (EXACT) {
                multiply_exact(acc, from, x, sx, w, sw, u0);
                return;
            }
            i32x8 vx[TM], vw[3];
            int cx[TM], cw[3];
            auto weights = [&](int j) {
                if constexpr (kPacked) {  // the instruction takes 4 bits as they are, values 32 q .. from lane (r, q)
                    const u32x4 v = *reinterpret_cast<const u32x4*>(from + (w + j * 2048 + (swizzle(u0 + q, r) << 4)));
                    vw[j % 3] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
                } else {
                    vw[j % 3] = operand(w, j);
                }
                cw[j % 3] = *reinterpret_cast<const uint8_t*>(from + (sw + j * 64));
            };
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                vx[i] = operand(x, i);
                cx[i] = *reinterpret_cast<const uint8_t*>(from + (sx + i * 64));
            }
            weights(0);
            weights(1);
            // weights are read two tiles ahead of their products; left to itself, the compiler
            // reads all of them first and runs out of registers
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                if (j + 2 < TN) weights(j + 2);
#pragma unroll
                for (int i = 0; i < TM; ++i)
                    acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(vw[j % 3], vx[i], acc[j][i], kPacked ? 4 : 0, 0, 0, cw[j % 3], 0, cx[i]);
#pragma unroll
                for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(acc[j][i])::"memory");
            }
        } else if constexpr (kWiden) {
            // lane (r, q) has values 16 q .. of a weight row and widens them for two products,
            // each of which takes eight; of x it reads the same values, units 2 q and 2 q + 1
            u32x4 vx[2][TM];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < TM; ++i) vx[h][i] = *reinterpret_cast<const u32x4*>(from + (x + i * 2048 + (swizzle(2 * q + h, r) << 4)));
            const int sw = kAtScale + (k & 1) * kScaleBytes + (wn * TN * 16 + r) * 2 + (q >> 1);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const uint32_t byte = *reinterpret_cast<const uint8_t*>(from + (sw + j * 32));
                u32x4 vw[2];
                if constexpr (HELD == kHeld8) {
                    widen8(*reinterpret_cast<const u32x4*>(from + (w + j * 2048 + (swizzle(u0 + q, r) << 4))), byte, vw);
                } else {
                    const u32x2 v = *reinterpret_cast<const u32x2*>(from + (w + j * 2048 + (swizzle(u0 + (q >> 1), r) << 4) + (q & 1) * 8));
                    const float f = mx_scale(byte);
                    vw[0] = widen4(v[0], f);
                    vw[1] = widen4(v[1], f);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < TM; ++i)
                        acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vw[h]), __builtin_bit_cast(bf16x8, vx[h][i]),
                                                                            acc[j][i], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = ((q + 4 * h) ^ (r & 7)) << 4;
                u32x4 vx[TM], vw[TN];
#pragma unroll
                for (int i = 0; i < TM; ++i) vx[i] = *reinterpret_cast<const u32x4*>(from + (x + i * 2048 + at));
#pragma unroll
                for (int j = 0; j < TN; ++j) vw[j] = *reinterpret_cast<const u32x4*>(from + (w + j * 2048 + at));
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int i = 0; i < TM; ++i) {
                        if constexpr (KIND == kProductBf16) {
                            acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vw[j]),
                                                                                __builtin_bit_cast(bf16x8, vx[i]), acc[j][i], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vw[j][k]), __uint_as_float(vx[i][k]),
                                                                                 acc[j][i], 0, 0, 0);
                        }
                    }
            }
        }
    }

    // Two tiles of 16 outputs, of pair o, for row tile i: lane (r, q) has columns 4 q .. of
    // each for row r.
    template <int O, int I>
    __device__ __forceinline__ static void outputs(const f32x4 (&acc)[TN][TM], bool zero, f32x4 (&v)[2]) {
        if constexpr (SWIGLU) {
            repeat<4>([&](auto k) {
                constexpr int K = decltype(k)::value;
                v[0][K] = silu_mul(acc[2 * O][I][K], acc[2 * O + 2][I][K]);
                v[1][K] = silu_mul(acc[2 * O + 1][I][K], acc[2 * O + 3][I][K]);
            });
        } else {
            v[0] = acc[O][I];
            v[1] = acc[O + 1][I];
        }
        if (zero) v[0] = v[1] = f32x4{};
    }

    // bf16 outputs whose rows take 16-byte stores, and halves with scales: through the
    // wavefront's part of LDS, so that whole lines are stored.
    __device__ __forceinline__ void write_lines(const f32x4 (&acc)[TN][TM], char* lds, int r0, int n, int c0) const {
        constexpr int TO = SWIGLU ? TN / 2 : TN, kUnits = TO * 2, kRow = kUnits * 16;  // 16-byte units of a row
        constexpr int kMask = kUnits < 8 ? kUnits - 1 : 7;
        char* const mine = lds + wv * (TM * 16 * kRow);
        repeat<TM>([&](auto i) {
            constexpr int I = decltype(i)::value;
            const int row = I * 16 + r, in_tile = wm * TM * 16 + row;
            const bool zero = a.x_row && in_tile < n && (unsigned)a.x_row[r0 + in_tile] >= (unsigned)a.x_rows;
            repeat<TO / 2>([&](auto o) {
                constexpr int O = 2 * decltype(o)::value;
                f32x4 v[2];
                outputs<O, I>(acc, zero, v);
                u32x2 e[2];
                if (a.y_kind == kProductHalf) {
                    const uint32_t byte = half_scale(v);
                    const float inv = half_inverse(byte);
                    const int col = c0 + (wn * TO + O) * 16;
                    if (q == 0 && in_tile < n && col < a.m) a.y_scale[(int64_t)(r0 + in_tile) * a.y_scale_stride + col / 32] = (uint8_t)byte;
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        e[p] = __builtin_bit_cast(u32x2, half4{(_Float16)(v[p][0] * inv), (_Float16)(v[p][1] * inv), (_Float16)(v[p][2] * inv),
                                                               (_Float16)(v[p][3] * inv)});
                } else {
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        e[p] = __builtin_bit_cast(u32x2, bf16x4{(__bf16)v[p][0], (__bf16)v[p][1], (__bf16)v[p][2], (__bf16)v[p][3]});
                }
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    *reinterpret_cast<u32x2*>(mine + row * kRow + (((2 * (O + p) + (q >> 1)) ^ (row & kMask)) << 4) + (q & 1) * 8) = e[p];
            });
        });
        __builtin_amdgcn_wave_barrier();
        constexpr int kRows = 64 / kUnits;  // of an instruction
        const int row0 = lane / kUnits, u = lane % kUnits, col = c0 + wn * TO * 16 + u * 8;
        const int left = col < a.m ? n - wm * TM * 16 - row0 : 0;  // rows from row0 on
        uint16_t* y = static_cast<uint16_t*>(a.y) + (int64_t)(r0 + wm * TM * 16 + row0) * a.y_stride + col;
        const int64_t next = kRows * a.y_stride;
        repeat<TM * 16 / kRows>([&](auto i) {
            constexpr int I = decltype(i)::value;
            const u32x4 v = *reinterpret_cast<const u32x4*>(mine + (I * kRows + row0) * kRow + ((u ^ ((I * kRows + row0) & kMask)) << 4));
            if (I * kRows < left) *reinterpret_cast<u32x4*>(y) = v;
            y += next;
        });
    }

    // Outputs of any other kind, as the lanes hold them.
    __device__ __forceinline__ void write(const f32x4 (&acc)[TN][TM], int r0, int n, int c0) const {
        constexpr int TO = SWIGLU ? TN / 2 : TN;
        repeat<TM>([&](auto i) {
            constexpr int I = decltype(i)::value;
            const int row = (wm * TM + I) * 16 + r;
            const bool live = row < n;
            const int64_t at = r0 + row;
            const bool zero = live && a.x_row && (unsigned)a.x_row[at] >= (unsigned)a.x_rows;
            repeat<TO / 2>([&](auto o) {  // a block of 32 outputs
                constexpr int O = 2 * decltype(o)::value;
                f32x4 v[2];
                outputs<O, I>(acc, zero, v);
                put32(a, v, at, c0 + (wn * TO + O) * 16 + 4 * q, live);
            });
        });
    }
    // fp32 products are added four at a time, and rounded each time: chains of 256 values,
    // which are added up in turn.  4096 values: y off by 3.0e-7 rms, in one chain by 1.15e-6,
    // both 160 us at 1000 rows by 4 x 512; 182 with a branch among the steps in place of a
    // loop for each chain.
    static constexpr int kChain = 8;  // steps
    __device__ __forceinline__ static void end_chain(f32x4 (&acc)[TN][TM], f32x4 (&sum)[KIND == kProductF32 ? TN : 1][TM]) {
#pragma unroll
        for (int j = 0; j < (KIND == kProductF32 ? TN : 1); ++j)
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                sum[j][i] += acc[j][i];
                acc[j][i] = f32x4{};
            }
    }

    // In step k the weights of step k + 2 are asked for, or where 128 bytes of a row last G
    // steps, in the first of them the next 128; and the rows of x of step k + 1.
    __device__ __forceinline__ void run(char* lds, int r0, int n, int c0) {
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
        constexpr bool kScales = kPacked || kScaled;
        f32x4 acc[TN][TM] = {}, sum[KIND == kProductF32 ? TN : 1][TM] = {};
        u32x4 s[SI];
        load_w(base, 0, 0);
        load_x(base, 0, 0);
        if constexpr (kScales) load_scales(s, 0);  // waits for all that
        if (!kPacked && steps > 1) load_w(base, 1, 1);
        if constexpr (kScales) store_scales(s, lds, 0);
        if (!kPacked && steps > 1)
            arrive<WI>();
        else
            arrive<0>();
        int slot = 0;  // of step k, of three
        int k = 0;
        do {
            const int end = KIND == kProductF32 ? min(k + kChain, steps) : steps;
            for (; k < end; ++k) {
                if constexpr (kScales)
                    if ((k + 1) % kBatch == 0 && k + 1 < steps) load_scales(s, k + 1);
                const int free = slot == 0 ? 2 : slot - 1, g = k / G + 1;
                if (k + 1 < steps) load_x(base, k + 1, (k + 1) & 1);
                if constexpr (kPacked) {
                    if (k % G == 0 && g * G < steps) load_w(base, g, g & 1);
                } else {
                    if (k + 2 < steps) load_w(base, k + 2, free);
                }
                // behind the last step this writes what nothing reads
                if constexpr (kScales) store_scales(s, lds, k + 1);
                __builtin_amdgcn_sched_barrier(0);
                multiply(acc, lds, k, kPacked ? (g - 1) & 1 : slot);
                __builtin_amdgcn_sched_barrier(0);
                // what may be left on its way: weights that are not needed in the next step
                if (kPacked ? k % G < G - 1 && k % G == 0 && g * G < steps : k + 2 < steps)
                    arrive<WI>();
                else
                    arrive<0>();
                slot = slot == 2 ? 0 : slot + 1;
            }
            if constexpr (KIND == kProductF32) end_chain(acc, sum);
        } while (KIND == kProductF32 && k < steps);
        if constexpr (KIND == kProductF32) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[j][i] = sum[j][i];
        }
        if (a.y_lines)
            write_lines(acc, lds, r0, n, c0);
        else
            write(acc, r0, n, c0);
    }
};

// Which tile a workgroup takes: found from the offsets alone, by every wavefront for
// itself, four groups a lane.  A group's rows are cut into units of `unit` and these
// into tiles of up to `most`, as evenly as they go.  Tiles of a group follow each other,
// and each XCD takes a stretch of the whole list, so that a group's weights and rows
// come into one L2.
struct ProductPlace {
    int expert, r0, n, col;
};
__device__ inline bool product_tile_at(const ProductArgs& a, int unit, int most, int columns, int xcd, int j, ProductPlace& at) {
    const int lane = threadIdx.x & 63;
    int c[5], tiles[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 5; ++j) c[j] = min(max(a.first[min(4 * lane + j, a.N)], 0), a.rows);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        tiles[j] = c[j + 1] > c[j] ? (c[j + 1] - c[j] + unit * most - 1) / (unit * most) : 0;
        sum += tiles[j];
    }
    int end = sum;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int p = __shfl_up(end, m);
        if (lane >= m) end += p;
    }
    const int all = __builtin_amdgcn_readlane(end, 63) * columns, share = xcd < 0 ? all : (all + 7) / 8;
    const int t = (xcd < 0 ? 0 : xcd * share) + j;
    if (j >= share || t >= all) return false;
    const int mine = __ffsll(__ballot(end * columns > t)) - 1;  // the lane whose groups hold tile t
    int local = t - __builtin_amdgcn_readlane(end - sum, mine) * columns;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int nt = __builtin_amdgcn_readlane(tiles[k], mine);
        if (local < nt * columns) {
            const int from = __builtin_amdgcn_readlane(c[k], mine), to = __builtin_amdgcn_readlane(c[k + 1], mine);
            const int units = (to - from + unit - 1) / unit, i = local % nt;
            const int u0 = i * (units / nt) + min(i, units % nt), u1 = u0 + units / nt + (i < units % nt ? 1 : 0);
            at.expert = 4 * mine + k;
            at.col = local / nt;
            at.r0 = from + u0 * unit;
            at.n = min(u1 * unit, to - from) - u0 * unit;
            return true;
        }
        local -= nt * columns;
    }
    return false;
}

__device__ inline bool product_place(const ProductArgs& a, int unit, int most, int columns, ProductPlace& at) {
    return product_tile_at(a, unit, most, columns, blockIdx.x & 7, blockIdx.x >> 3, at);
}
// Unit i of 16 rows.
__device__ inline bool product_unit(const ProductArgs& a, int i, ProductPlace& at) { return product_tile_at(a, 16, 1, 1, -1, i, at); }

// MOST: units of the largest tile.  A tile of fewer has code of its own,
// so that rows which are not there are not multiplied.
template <int KIND, int HELD, int UNIT, int MOST, int BN, int WM, int WN, int PER_CU, bool SWIGLU, bool EXACT>
__global__ __launch_bounds__(64 * WM * WN, PER_CU) void product_kernel(ProductArgs a) {
    constexpr int kUnit = UNIT, kOut = SWIGLU ? BN / 2 : BN;
    using Largest = ProductTile<KIND, HELD, kUnit * MOST, BN, WM, WN, SWIGLU, EXACT>;
    __shared__ __align__(16) char lds[Largest::kBytes];
    ProductPlace at;
    if (!product_place(a, kUnit, MOST, (a.m + kOut - 1) / kOut, at)) return;
    auto go = [&](auto units) {
        using Tile = ProductTile<KIND, HELD, kUnit * decltype(units)::value, BN, WM, WN, SWIGLU, EXACT>;
        Tile tile(a, at.expert, at.r0, at.n, at.col * kOut);
        tile.run(lds, at.r0, at.n, at.col * kOut);
    };
    const int units = (at.n + kUnit - 1) / kUnit;
    if constexpr (MOST >= 4)
        if (units == 4) return go(std::integral_constant<int, 4>{});
    if constexpr (MOST >= 3)
        if (units == 3) return go(std::integral_constant<int, 3>{});
    if constexpr (MOST >= 2)
        if (units == 2) return go(std::integral_constant<int, 2>{});
    go(std::integral_constant<int, 1>{});
}

template <int KIND, int HELD, int UNIT, int MOST, int BN, int WM, int WN, int PER_CU>
void launch_product_tile(const ProductArgs& args, hipStream_t st) {
    const int out = args.swiglu ? BN / 2 : BN;
    const int64_t columns = (args.m + out - 1) / out;
    // row tiles, at most: one for every whole one's rows and one more for each group
    const int64_t tiles = std::min<int64_t>(args.rows, args.rows / (UNIT * MOST) + std::min(args.N, args.rows)) * columns;
    const dim3 grid((unsigned)((tiles + 7) / 8 * 8)), block(64 * WM * WN);
    using Tile = ProductTile<KIND, HELD, UNIT * MOST, BN, WM, WN, false, false>;
    ProductArgs a = args;
    // not where a row's 128 bytes are parts of two lines, which the caches have to keep
    a.once = (int64_t)a.rows * 4 <= (int64_t)a.N * UNIT * MOST * 3 && a.d % (Tile::kValues * 128 / Tile::kWBytes) == 0;
    auto go = [&](auto exact) {
        constexpr bool EXACT = decltype(exact)::value;
        launch_kernel(a.swiglu ? product_kernel<KIND, HELD, UNIT, MOST, BN, WM, WN, PER_CU, true, EXACT>
                               : product_kernel<KIND, HELD, UNIT, MOST, BN, WM, WN, PER_CU, false, EXACT>,
                      grid, block, st, Timing{}, a);
    };
    if constexpr (KIND == kProductMx8)
        if (a.exact) return go(std::true_type{});
    go(std::false_type{});
}

// ---------------------------------------------------------------- few rows of a group
// A workgroup takes up to 16 rows of a group and 32 outputs, its wavefronts share the sum:
// each takes every so many-th line, 128 bytes of a weight row, lane (r, q) units q and q + 4
// of it and the same values of row r of x, straight into the matrix core's registers, DEPTH
// lines under way.  Values of 8 and 4 bits become bf16, which holds them exactly, so the
// products are too.
// grid: x = units of 16 rows, which share weights where they are of one group, y = outputs
// / 32 rounded up
constexpr int kFewWaves = 4;
template <int KIND, int HELD, bool SWIGLU>
struct FewRows {
    static constexpr bool kF32 = KIND == kProductF32, kX8 = KIND == kProductMx8;
    static constexpr int kW = HELD == kHeld4 ? 4 : HELD == kHeld8 || kX8 ? 8 : kF32 ? 32 : 16;  // bits of a weight
    static constexpr int kX = kX8 ? 8 : kF32 ? 32 : 16;
    static constexpr int V = 128 / kW, XU = V * kX / 128;  // values of a unit, and units of x that hold as many
    static constexpr int RT = SWIGLU ? 4 : 2;              // tiles of 16 weight rows
    static constexpr int DEPTH = RT * XU <= 2 ? 4 : 2;
    static constexpr int kWaves = kFewWaves;

    struct Line {
        u32x4 w[2][RT], x[2][XU];
        uint8_t ws[2][RT], xs[2];
    };

    // Eight values, number j of a unit, as bf16.
    __device__ static bf16x8 weight(const u32x4& w, uint32_t byte, int j) {
        if constexpr (kW == 4) return __builtin_bit_cast(bf16x8, widen4(w[j], mx_scale(byte)));
        if constexpr (kW == 8) return eight(w, byte, j);
        return __builtin_bit_cast(bf16x8, w);
    }
    __device__ static bf16x8 eight(const u32x4& q, uint32_t byte, int j) {
        u32x4 v[2];
        widen8(q, byte, v);
        return __builtin_bit_cast(bf16x8, v[j]);
    }

    const ProductArgs& a;
    const char *w[RT], *x;
    const uint8_t *ws[RT], *xs;
    bool live;  // this lane has a row of x
    int units;
    int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;

    __device__ FewRows(const ProductArgs& args, const ProductPlace& at, int c0) : a(args) {
        units = a.d / V;
        const int64_t pitch = (int64_t)a.d * kW / 8;
        const char* we = a.w + at.expert * a.w_matrix;
        const uint8_t* se = kW < 16 ? a.w_scale + at.expert * a.w_scale_matrix : nullptr;
#pragma unroll
        for (int t = 0; t < RT; ++t) {  // with SwiGLU two tiles of G and the same two of U
            const int64_t row = (SWIGLU && t >= 2 ? a.m : 0) + min(c0 + (t & 1) * 16 + r, a.m - 1);
            w[t] = we + row * pitch;
            ws[t] = kW < 16 ? se + row * (a.d / 32) : nullptr;
        }
        live = r < at.n;
        int64_t s = at.r0 + (live ? r : 0);
        if (a.x_row) {
            const int i = a.x_row[s];
            s = (unsigned)i < (unsigned)a.x_rows ? i : 0;
        }
        x = a.x + s * a.x_pitch;
        xs = kX8 ? a.x_scale + s * a.x_scale_pitch : nullptr;
    }

    __device__ __forceinline__ void load(Line& v, int l) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int u = l * 8 + 4 * h + q;
            const bool in = u < units;  // zeros behind the row's end
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                v.w[h][t] = in ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(w[t] + (int64_t)u * 16)) : u32x4{};
                v.ws[h][t] = kW < 16 && in ? ws[t][u * V / 32] : 0;
            }
#pragma unroll
            for (int i = 0; i < XU; ++i) v.x[h][i] = in && live ? *reinterpret_cast<const u32x4*>(x + ((int64_t)u * XU + i) * 16) : u32x4{};
            v.xs[h] = kX8 && in && live ? xs[u * V / 32] : 0;
        }
    }
    __device__ __forceinline__ void step(const Line& v, f32x4 (&acc)[RT]) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (kF32) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v.w[h][t][j]), __uint_as_float(v.x[h][0][j]), acc[t], 0, 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < V / 8; ++j) {
                    bf16x8 b;
                    if constexpr (kX8)
                        b = eight(v.x[h][j / 2], v.xs[h], j & 1);
                    else
                        b = __builtin_bit_cast(bf16x8, v.x[h][j]);
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(weight(v.w[h][t], v.ws[h][t], j), b, acc[t], 0, 0, 0);
                }
            }
        }
    }
    __device__ __forceinline__ void run(f32x4 (&red)[kWaves][RT][64], const ProductPlace& at, int c0) const {
        const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lines = (units + 7) / 8;
        f32x4 acc[RT] = {}, sum[kF32 ? RT : 1] = {};
        Line v[DEPTH];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) load(v[i], wv + i * kWaves);  // zeros behind the last line
        for (int l = wv; l < lines; l += DEPTH * kWaves) {
#pragma unroll
            for (int i = 0; i < DEPTH; ++i) {
                step(v[i], acc);
                load(v[i], l + (i + DEPTH) * kWaves);
            }
            // chains as in the tiles, of 128 values, or 64 with SwiGLU.  y off by, rms, for 4096
            // values 2.2e-7, in one chain a wavefront 5.7e-7; for 65536, 2.9e-7 and 2.2e-6; at no
            // cost: 8 rows by 4096 x 4096, 32 us
            if constexpr (kF32)
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    sum[t] += acc[t];
                    acc[t] = f32x4{};
                }
        }
        if constexpr (kF32)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t] = sum[t];
#pragma unroll
        for (int t = 0; t < RT; ++t) red[wv][t][lane] = acc[t];
        __syncthreads();
        if (wv) return;
#pragma unroll
        for (int k = 1; k < kWaves; ++k)
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t] += red[k][t][lane];
        const bool zero = live && a.x_row && (unsigned)a.x_row[at.r0 + r] >= (unsigned)a.x_rows;
        f32x4 y[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            if constexpr (SWIGLU) {
#pragma unroll
                for (int k = 0; k < 4; ++k) y[p][k] = silu_mul(acc[p][k], acc[2 + p][k]);
            } else {
                y[p] = acc[p];
            }
            if (zero) y[p] = f32x4{};
        }
        put32(a, y, at.r0 + r, c0 + 4 * q, live);
    }
};

template <int KIND, int HELD, bool SWIGLU>
__global__ __launch_bounds__(64 * kFewWaves) void product_few_kernel(ProductArgs a) {
    using Few = FewRows<KIND, HELD, SWIGLU>;
    __shared__ f32x4 red[Few::kWaves][Few::RT][64];
    ProductPlace at;
    if (!product_unit(a, blockIdx.x, at)) return;
    Few(a, at, blockIdx.y * 32).run(red, at, blockIdx.y * 32);
}

template <int KIND, int HELD>
void launch_product_few(const ProductArgs& a, hipStream_t st) {
    const int units = std::min(a.rows, a.rows / 16 + std::min(a.N, a.rows));
    launch_kernel(a.swiglu ? product_few_kernel<KIND, HELD, true> : product_few_kernel<KIND, HELD, false>,
                  dim3((unsigned)units, (unsigned)((a.m + 31) / 32)), dim3(64 * kFewWaves), st, Timing{}, a);
}

template <int KIND, int HELD>
void launch_product_held(const ProductArgs& a, hipStream_t st) {
    // By the rows of a group that has some, on average, and by how many tiles of 128 x 128 and
    // of 256 x 256 outputs that makes.
    const int64_t groups = std::min(a.N, a.rows), rows = (a.rows + groups - 1) / groups, weights = (int64_t)a.m * (a.swiglu ? 2 : 1);
    const int64_t middle = groups * ((rows + 127) / 128) * ((weights + 127) / 128);
    const int64_t large = groups * ((rows + 255) / 256) * ((weights + 255) / 256);
    const bool fills = large * 10 >= (large + 255) / 256 * 256 * 8 || large >= 1024;  // the device's CUs, to 80 %
    // Few rows of few groups leave most of the device without a tile.  us, tiles of 128 x 128
    // against few rows: 2048 x 2048 bf16, 1 group of 16 rows 21 / 12, 8 of 1 20 / 17, of 16 22 /
    // 36; 1536 x 2048, 64 groups of one row 71 / 83, 128 of 8 132 / 212; 8-bit weights 61 / 55
    // and 104 / 136.  How rows spread over the groups is known on the device only: of 128 groups
    // all 1000 rows in one, by 64 x 2048, bf16 23.2 / 12.5, 8-bit weights 27.0 / 10.6, but by 768
    // x 2048, 8-bit weights 25.4 / 48.4, 4-bit ones 25.4 / 39.0.
    const int64_t scarce = HELD == kHeldSame ? 1 : 2;
    if ((rows <= 8 && middle < 512 * scarce) || (rows <= 32 && middle < 128 * scarce)) {
        launch_product_few<KIND, HELD>(a, st);
    } else if constexpr (KIND == kProductF32) {
        if (middle < 1024)
            launch_product_tile<KIND, HELD, 16, 2, 128, 1, 2, 1>(a, st);
        else
            launch_product_tile<KIND, HELD, 32, 4, 128, 2, 2, 2>(a, st);
    } else {
        constexpr int kMost = KIND == kProductMx8 && HELD == kHeldSame ? 3 : 4;  // units that leave room in LDS
        // The large tile reads the rows of x half as often, two of the small one on a CU start
        // and store beside each other's products.  us, large / small, rows of a group ragged by a
        // tenth: bf16 128 x (1536 x 2048), 100 rows 143 / 144, 192 172 / 209, 1024 751 / 868; 32 x
        // (2880 x 2880), 100 rows 104 / 91, 192 138 / 130, 1024 517 / 591; 8 bits, the same, 87 / 85,
        // 126 / 142, 493 / 591, and 67 / 66, 104 / 100, 365 / 416; 8-bit rows with 4-bit weights 76 /
        // 67, 96 / 116, 421 / 465, and 62 / 51, 87 / 74, 314 / 320.  Where every wavefront widens
        // 4-bit weights, 134 / 114, 176 / 192, 512 rows 415 / 428, 1024 758 / 827, and 117 / 86, 160 /
        // 132, 319 / 300, 547 / 572; of 32 x (5760 x 2880), 128 rows 203 / 201, 512 605 / 562: the
        // small tile up to 768 rows there, which loses a tenth at most (192 rows of 2048 values)
        // where the large one loses a fifth (192 of 2880).
        constexpr int64_t kLargeFrom = KIND == kProductBf16 && HELD == kHeld4 ? 768 : 28 * kMost;  // 7/8 of the small tile
        if (rows >= kLargeFrom && fills)
            launch_product_tile<KIND, HELD, 64, kMost, 256, 2, 4, 1>(a, st);
        else
            launch_product_tile<KIND, HELD, 32, kMost, 128, 2, 2, 2>(a, st);
    }
}

}  // namespace cmoe
