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

typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// Codes of 8 elements with random bytes.  The stochastic converter takes its
// first element, on whichever step of the grid it lies, to the upper neighbour
// where the fraction f of the step has f + seed / 2^32 >= 1; a byte r becomes
// the seed of (r + 1/2) / 256.  The second element's seed is another, and the
// converter writes one byte of its register, which the compiler takes to be
// written whole: so each element is converted into a register of its own, of
// which the low four bits count.
struct Stochastic {
    unsigned c[8];
    float scale;

    __device__ __forceinline__ explicit Stochastic(unsigned byte) : scale(scale_value(byte)) {}

    // The seed of byte J of r.
    template <int J>
    static __device__ __forceinline__ unsigned seed(unsigned r) {
        return __builtin_amdgcn_perm(r, 0x00800000u, ((4u + J) << 24) | 0x00020000u);
    }
    // (The bf16 form of the converter rounds otherwise in some cases.)
    __device__ __forceinline__ void put(int i, float x, unsigned seed) {
        float any;  // the second element's result is not used
        any = __builtin_nondeterministic_value(any);
        c[i] = __builtin_amdgcn_cvt_scalef32_sr_pk_fp4_f32(0u, v2f{x, any}, seed, scale, 0);
    }
    // Bytes 0 of four registers.
    static __device__ __forceinline__ unsigned bytes(unsigned a, unsigned b, unsigned d, unsigned e) {
        const unsigned lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(e, d, 0x0c0c0400u);
        return lo | (hi << 16);
    }
    __device__ __forceinline__ unsigned codes() const {
        const unsigned even = bytes(c[0], c[2], c[4], c[6]), odd = bytes(c[1], c[3], c[5], c[7]);
        return (even & 0x0f0f0f0fu) | ((odd & 0x0f0f0f0fu) << 4);
    }
};

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
