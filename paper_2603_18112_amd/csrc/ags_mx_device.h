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

// |x| 2^-e taken to a neighbour on the grid by a random byte r, with x's sign.
// y = |x| 2^-e is exact and below 8.  From 1 up the grid has one bit after the
// leading one, so adding (r + 1/2) / 256 of that bit to the fp32 pattern
// carries into it, and over the binade's end, as the rule asks; what is below
// the bit is then cut off.  Below 1 the grid is 1/2, that of the binade of
// 1 + y.  That sum may round: y keeps 11 significant bits first (no threshold,
// all multiples of 2^-10, lies between y and what is left of it), so the sum is
// exact down to y = 2^-13, below which no byte rounds up.  bf16 values have 8.
template <bool BF16>
__device__ __forceinline__ float round_stochastic(float x, float inv, unsigned r) {
    unsigned u = __float_as_uint(fabsf(x) * inv);
    if (!BF16) u &= 0xffffe000u;
    const float y = __uint_as_float(u), one = y < 1.0f ? 1.0f : 0.0f;
    const unsigned up = (__float_as_uint(y + one) + ((r << 14) | 0x2000u)) & 0xffc00000u;
    return copysignf(__uint_as_float(up) - one, x);
}

// Codes of 8 elements and their random bytes; the converter has nothing left
// to round, 8 becomes 6.
template <bool BF16>
__device__ __forceinline__ unsigned codes_stochastic(const float* x, unsigned byte, const unsigned* r) {
    const float inv = scale_inverse(byte);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = round_stochastic<BF16>(x[i], inv, r[i]);
    return codes_nearest(v, 127u);
}

__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

template <typename T, int N, int ALIGN>
struct __attribute__((packed, aligned(ALIGN))) Unaligned {
    T v[N];
};

// 8 elements as fp32 from p; `left` of them lie inside the row, the rest read
// as zero.
__device__ __forceinline__ void load8(const unsigned short* p, int64_t left, float* x) {
    if (left >= 8) {
        const auto w = *reinterpret_cast<const Unaligned<unsigned, 4, 2>*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w.v[i] << 16);
            x[2 * i + 1] = __uint_as_float(w.v[i] & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < left ? __uint_as_float((unsigned)p[i] << 16) : 0.0f;
}
__device__ __forceinline__ void load8(const float* p, int64_t left, float* x) {
    if (left >= 8) {
        const auto w = *reinterpret_cast<const Unaligned<float, 8, 4>*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = w.v[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < left ? p[i] : 0.0f;
}
}  // namespace mx
}  // namespace ags
