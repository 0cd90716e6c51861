// mx8.h - values in 8 bits: e4m3 numbers with one power-of-two scale for every
// 32 consecutive values of a row, kept as the byte E + 127.
//
// E is the smallest exponent (at least -127) with max |v| <= 448 2^E, 448 being
// the largest e4m3 number, so no value saturates and each is rounded once, to
// nearest even.  A block that holds an infinity or a NaN gets the byte 255 and
// NaN in all its places.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cmoe {

constexpr int kMxBlock = 32;         // values that share a scale
constexpr uint32_t kMxBad = 255;     // scale byte of a block with a non-finite value
constexpr uint32_t kMxNaN2 = 0x7F7F; // two e4m3 NaN

// Scale byte of a block whose largest magnitude is amax (NaN if it holds one).
// 448 = 1.75 2^8: with amax = m 2^x, 1 <= m < 2, E is x - 8, or x - 7 for m > 1.75.
__device__ inline uint32_t mx_scale_byte(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return b >= 0x7F800000u ? kMxBad : (uint32_t)max(e, 0);
}

// 2^-E: the byte of a finite block is at most 247, so the product with a value
// is exact unless it falls below e4m3's range anyway.
__device__ inline float mx_inverse(uint32_t byte) { return __uint_as_float((254u - min(byte, 253u)) << 23); }

// Two values over their scale as e4m3, in the low half or the high half of old.
template <bool HIGH>
__device__ inline uint32_t mx_pair(float a, float b, float inverse, uint32_t old) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, (int)old, HIGH);
}

// Eight values of one block in 8 bits.
__device__ inline uint2 mx_pack8(const float* v, uint32_t byte) {
    if (byte == kMxBad) return make_uint2(kMxNaN2 * 0x10001u, kMxNaN2 * 0x10001u);
    const float inv = mx_inverse(byte);
    uint2 q;
    q.x = mx_pair<true>(v[2], v[3], inv, mx_pair<false>(v[0], v[1], inv, 0));
    q.y = mx_pair<true>(v[6], v[7], inv, mx_pair<false>(v[4], v[5], inv, 0));
    return q;
}

// max of two magnitudes; a NaN wins
__device__ inline float mx_max(float a, float b) {
    const uint32_t x = __float_as_uint(a) & 0x7FFFFFFFu, y = __float_as_uint(b) & 0x7FFFFFFFu;
    return __uint_as_float(max(x, y));
}

}  // namespace cmoe
