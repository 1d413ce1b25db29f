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
    double inv_cols;  // 1 / cols
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

// Rows up to this length stay in registers between the passes over them: forward
// (half as long in fp32), and backward, where a lane also keeps the sums for its columns.
constexpr int64_t kNormForwardCols = 32768, kNormBackwardCols = 16384;

// Into how many parts the rows are cut for the gradients of weight and bias.  Each
// part's sums are 8 bytes a column, written and read once more; a part is a block, and
// of those for more than 4096 columns a CU holds one.  With up to 256 and 512 of them
// 16384 x 8192 bf16 takes 159 and 167 us, 4000 x 16000 107 and 120; with 512 and 768
// for shorter rows 8192 x 4096 48 and 53, 8192 x 2048 fp32 45 and 48; with at least two
// rows each and four 5001 x 1000 fp32 21.5 and 24, 64 x 4096 8.3 and 9.9, one row 28
// and 8.5.
inline int32_t norm_parts(int64_t rows, int64_t cols) {
    if (cols > kNormBackwardCols) {
        const int64_t tiles = (cols + 511) / 512;
        return (int32_t)std::max<int64_t>(1, std::min<int64_t>((rows + 31) / 32, (2048 + tiles - 1) / tiles));
    }
    const int64_t at_once = cols <= 512 ? 8 : cols <= 1024 ? 4 : 1;  // rows of a block
    return (int32_t)std::max<int64_t>(
        1, std::min<int64_t>((rows + 2 * at_once - 1) / (2 * at_once), cols > 4096 ? 256 : 512));
}

// Weak for the same reason as the clipping launchers.
__attribute__((weak)) hipError_t launch_norm(const NormArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_norm_backward(const NormBackwardArgs&, hipStream_t);

}  // namespace ags
