// gfx950 kernels of the products of 4-bit operands (include/ags_mx.h).
//
// mx_product_kernel  one wave per 16 x 16 tile of the output, operands read
//                    straight from memory.
#include "ags_mx_device.h"
#include "ags_mx_internal.h"

namespace ags {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kFp4 = 4;  // operand format of the scaled matrix instruction

__device__ __forceinline__ v8i operand(uint4 v) {
    return v8i{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
}

__device__ __forceinline__ unsigned short bf16_round(float x) {
    const unsigned u = __float_as_uint(x);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (unsigned short)((u >> 16) | 0x40u);
    return (unsigned short)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

__device__ __forceinline__ void store_elem(const MxProductArgs& a, int64_t i, int64_t j, float v) {
    const int64_t at = i * a.stride + j;
    if (a.bf16) {
        unsigned short* p = static_cast<unsigned short*>(a.out) + at;
        if (a.accumulate) v += __uint_as_float((unsigned)*p << 16);
        *p = bf16_round(v);
    } else {
        float* p = static_cast<float*>(a.out) + at;
        if (a.accumulate) v += *p;
        *p = v;
    }
}

__global__ __launch_bounds__(64) void mx_product_kernel(MxProductArgs a, unsigned tiles_n) {
    const int lane = threadIdx.x, r = lane & 15, q = lane >> 4;
    const int64_t i0 = (int64_t)(blockIdx.x / tiles_n) * 16, j0 = (int64_t)(blockIdx.x % tiles_n) * 16;
    // rows past the end repeat the last one; their results are not stored
    const int64_t ia = min(i0 + r, a.m - 1), jb = min(j0 + r, a.n - 1);
    const uint8_t* pa = a.a + ia * (a.kp / 2) + q * 16;
    const uint8_t* pb = a.b + jb * (a.kp / 2) + q * 16;
    const uint8_t* psa = a.sa + ia * (a.kp / 32) + q;
    const uint8_t* psb = a.sb + jb * (a.kp / 32) + q;
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t k = 0; k < a.kp; k += 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(pa + k / 2), y = *reinterpret_cast<const uint4*>(pb + k / 2);
        const int sx = psa[k / 32], sy = psb[k / 32];
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(x), operand(y), acc, kFp4, kFp4, 0, sx, 0, sy);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i0 + q * 4 + i < a.m && j0 + r < a.n) store_elem(a, i0 + q * 4 + i, j0 + r, acc[i]);
}

}  // namespace

hipError_t launch_mx_product(const MxProductArgs& a, hipStream_t s) {
    const unsigned tiles_n = (unsigned)((a.n + 15) / 16), tiles_m = (unsigned)((a.m + 15) / 16);
    hipLaunchKernelGGL(mx_product_kernel, dim3(tiles_n * tiles_m), dim3(64), 0, s, a, tiles_n);
    return hipGetLastError();
}

}  // namespace ags
