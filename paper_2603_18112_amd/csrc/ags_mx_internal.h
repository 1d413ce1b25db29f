// Internal declarations of the 4-bit operators (include/ags_mx.h), shared by
// their host code and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ags_mx.h"

namespace ags {

constexpr int64_t mx_padded(int64_t cols) { return (cols + AGS_MX_PAD - 1) / AGS_MX_PAD * AGS_MX_PAD; }

struct MxQuantArgs {
    const void* x;
    const uint8_t* noise;  // NULL: to nearest
    int64_t rows, cols, stride, noise_stride;
    uint8_t *codes, *scales;      // [rows][padded cols / 2], NULL: not wanted
    uint8_t *codes_t, *scales_t;  // [cols][padded rows / 2]
    int32_t bf16;
    int32_t aligned;  // rows of x (and of the noise) start at 16 (8) bytes
};

struct MxDequantArgs {
    const uint8_t *codes, *scales;
    void* out;
    int64_t rows, cols, stride;
    int32_t bf16;
};

struct MxProductArgs {
    const uint8_t *a, *sa, *b, *sb;  // codes and scales, [m][kp / 2], [n][kp / 2]
    void* out;
    int64_t stride;
    int64_t m, n, kp;
    int32_t bf16, accumulate;
};

// Weak for the same reason as the clipping launchers.
__attribute__((weak)) hipError_t launch_mx_quantize(const MxQuantArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_mx_dequantize(const MxDequantArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_mx_product(const MxProductArgs&, hipStream_t);

}  // namespace ags
