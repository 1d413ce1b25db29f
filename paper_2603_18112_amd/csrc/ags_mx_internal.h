// Internal declarations of the 4-bit operators (include/ags_mx.h), shared by
// their host code and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ags_mx.h"

namespace ags {

constexpr int64_t mx_padded(int64_t cols) { return (cols + AGS_MX_PAD - 1) / AGS_MX_PAD * AGS_MX_PAD; }

// Scales: rows rounded up, bytes between chunks of 256 columns.
constexpr int64_t mx_scale_rows(int64_t rows) { return (rows + AGS_MX_ROWS - 1) / AGS_MX_ROWS * AGS_MX_ROWS; }
constexpr int64_t mx_scale_bytes(int64_t rows, int64_t cols) { return mx_padded(cols) / 32 * mx_scale_rows(rows); }

struct MxQuantArgs {
    const void* x;
    const uint8_t* noise;  // NULL: to nearest
    int64_t rows, cols, stride, noise_stride;
    uint8_t *codes, *scales;      // of x, NULL: not wanted
    uint8_t *codes_t, *scales_t;  // of x transposed
    int32_t bf16;
};

struct MxDequantArgs {
    const uint8_t *codes, *scales;
    void* out;
    int64_t rows, cols, stride;
    int32_t bf16;
};

struct MxProductArgs {
    const uint8_t *a, *sa, *b, *sb;  // codes and scales of [m, kp] and [n, kp]
    void* out;
    int64_t stride;
    int64_t m, n, kp;
    int32_t bf16, accumulate;
    float* partials;  // [splits][m][n] sums over parts of the contracted axis, where splits > 1
    int32_t splits;
};

// How a product is cut into blocks: tiles of 64 * tm x 64 * tn outputs, the
// contracted axis into `splits` parts.
struct MxShape {
    int32_t tm, tn, splits;
};
inline MxShape mx_product_plan(int64_t m, int64_t n, int64_t kp) {
    MxShape p{1, 1, 1};
    auto tiles = [&](int64_t tm, int64_t tn) { return ((m + 64 * tm - 1) / (64 * tm)) * ((n + 64 * tn - 1) / (64 * tn)); };
    if (tiles(4, 4) >= 192) p.tm = p.tn = 4;
    else if (tiles(2, 2) >= 192) p.tm = p.tn = 2;
    const int64_t t = tiles(p.tm, p.tn), stages = kp / 256;
    if (t < 256) p.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(512 / t, stages / 4));
    return p;
}

// Weak for the same reason as the clipping launchers.
__attribute__((weak)) hipError_t launch_mx_quantize(const MxQuantArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_mx_dequantize(const MxDequantArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_mx_product(const MxProductArgs&, hipStream_t);

}  // namespace ags
