// Internal declarations of the layer norm (include/ags_norm.h), shared by its
// host code and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ags_norm.h"

namespace ags {

struct NormArgs {
    const void *x, *weight, *bias;
    void* y;
    float* saved;  // [2][rows], or NULL
    int64_t rows, cols, x_stride, y_stride;
    float eps;
    int32_t bf16, w_bf16, y_bf16;
};

struct NormBackwardArgs {
    const void *dy, *x, *weight;
    const float* saved;
    void *dx, *dweight, *dbias;  // each may be NULL
    float* partials;             // [parts][2][cols]
    int64_t rows, cols, dy_stride, x_stride, dx_stride;
    int32_t parts;
    int32_t bf16, w_bf16, dw_bf16, accumulate;
};

// Rows up to this length stay in registers between the passes over them:
// forward, and backward, where a lane also keeps the sums for its columns.
constexpr int64_t kNormForwardCols = 32768, kNormBackwardCols = 16384;

// Into how many parts the rows are cut for the gradients of weight and bias.  Each part's sums
// are 8 bytes a column, written and read once more.
inline int32_t norm_parts(int64_t rows, int64_t cols) {
    if (cols > kNormBackwardCols) {
        const int64_t tiles = (cols + 511) / 512;
        return (int32_t)std::max<int64_t>(1, std::min<int64_t>((rows + 31) / 32, (2048 + tiles - 1) / tiles));
    }
    const int64_t at_once = cols <= 512 ? 8 : cols <= 1024 ? 4 : 1;  // rows of a block
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>((rows + 4 * at_once - 1) / (4 * at_once), 512));
}

// Weak for the same reason as the clipping launchers.
__attribute__((weak)) hipError_t launch_norm(const NormArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_norm_backward(const NormBackwardArgs&, hipStream_t);

}  // namespace ags
