// Device functions of the 4-bit format (include/ags_mx.h): a block's scale
// and its elements' codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ags_mx.h"

namespace ags {
namespace mx {

// Where the scale of (row, column c) stands.
__device__ __forceinline__ int64_t scale_at(int64_t rows, int64_t row, int64_t c) {
    const int64_t rp = (rows + AGS_MX_ROWS - 1) / AGS_MX_ROWS * AGS_MX_ROWS;
    return ((c >> 8) * rp + row) * 8 + ((c >> 5) & 7);
}

// The scale byte (e + 127) of a block whose largest magnitude has these fp32
// bits.  The bits of magnitudes order like their values, infinities and NaN
// above all others.
template <bool STOCHASTIC>
__device__ __forceinline__ unsigned scale_byte(unsigned amax_bits) {
    if (amax_bits >= 0x7f800000u) return 255u;
    int b = (int)(amax_bits >> 23) - 2;  // floor(log2) - 2 + 127
    if (STOCHASTIC) b += (amax_bits & 0x7fffffu) > 0x400000u ? 1 : 0;  // above 1.5: 6 would be too little
    return (unsigned)min(max(b, 0), 252);
}

// 2^e for scale bytes 0 .. 252 (2^-127 is denormal).
__device__ __forceinline__ float scale_value(unsigned byte) {
    return __uint_as_float(byte ? byte << 23 : 0x400000u);
}

// 2^-e, exact: 2^127 .. 2^-125.
__device__ __forceinline__ float scale_inverse(unsigned byte) {
    return __uint_as_float((254u - byte) << 23);
}

// Codes of 8 elements in one dword, to nearest: the converter instruction
// divides by the scale, rounds ties to even and saturates at 6.
__device__ __forceinline__ unsigned codes_nearest(const float* x, unsigned byte) {
    const float s = scale_value(byte);
    unsigned r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
    return r;
}

// One code with a random byte, in integers.  y = |x| 2^-e is exact and below
// 8.  From 1 up the grid has one bit after the leading one, so adding
// (r + 1/2) / 256 of that bit to the fp32 pattern carries into it, and over
// the binade's end, as the rule asks; below 1 the grid is 1/2 and y a
// fixed-point number with 24 bits after the point (its lower bits cannot
// reach a threshold, all of which are multiples of 2^-10).
__device__ __forceinline__ unsigned code_stochastic(float x, float inv, unsigned r) {
    const unsigned sign = (__float_as_uint(x) >> 28) & 8u;
    const float y = fabsf(x) * inv;
    const unsigned up = (__float_as_uint(y) + ((2u * r + 1u) << 13)) >> 22;  // code + 252
    const unsigned low = ((unsigned)(y * 0x1p24f) + ((2u * r + 1u) << 14)) >> 23;
    return sign | (y >= 1.0f ? min(up - 252u, 7u) : low);
}

__device__ __forceinline__ unsigned codes_stochastic(const float* x, unsigned byte, const unsigned char* r) {
    const float inv = scale_inverse(byte);
    unsigned c = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) c |= code_stochastic(x[i], inv, r[i]) << (4 * i);
    return c;
}

__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// A code's value times 2: 0, 1, 2, 3, 4, 6, 8, 12, with its sign.
__device__ __forceinline__ float code_value(unsigned c) {
    const unsigned m = c & 7u;
    const unsigned v = m < 4 ? m : (2u + (m & 1u)) << ((m >> 1) - 1);
    const float f = 0.5f * (float)v;
    return c & 8u ? -f : f;
}

}  // namespace mx
}  // namespace ags
