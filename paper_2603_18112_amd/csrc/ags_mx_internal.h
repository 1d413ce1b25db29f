// Internal declarations of the 4-bit operators (include/ags_mx.h), shared by
// their host code and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

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
// contracted axis into `splits` parts; or few: the kernel for few rows of a.
struct MxShape {
    int32_t tm, tn, splits, few;
};

// The kernel for few rows reads x's codes from the caches once for each 16 rows
// of w, so beyond 16 rows it is for small products only.  Against tiles of 64 x
// 64 in parts with the launch that joins them, kernels' times in us: 32 rows
// 4096 x 4096 9.8 against 14.3, 24 rows 4096 x 25088 20.3 against 21.8 (from the
// caches 19.3 against 17.6), 20 rows 16384 x 16384 45 against 42, 32 rows 51
// against 38.
inline bool mx_few(int64_t m, int64_t n, int64_t kp) { return m <= 16 || (m <= 32 && n * kp <= ((int64_t)1 << 26)); }

// Does ags_mx_linear take x to 4 bits in the product's kernel?  Every block
// does so then; it keeps x in LDS.  One launch against two, us a call bound by
// the host / in a graph: 1 row 4096 x 4096 9.0 / 3.8 against 13.1 / 5.2, 8 rows
// (32768 elements of x) 9.0 / 5.3 against 13.3 / 5.9, 16 rows (65536) 9.1 / 7.3
// against 13.4 / 6.4; 1 row 16384 x 16384 in a graph 28.0 against 30.1.
inline bool mx_linear_fused(int64_t rows, int64_t k) { return rows <= 16 && rows * k <= 32768; }

// The tile and the split with the least estimated time in us.  A stage (256
// columns) of a tile of 64, 128 or 256 squared takes 0.55, 0.68 or 1.35 on an
// idle CU (1.9 with all CUs at work, at the clock the power limit leaves);
// four small tiles on a CU take twice as long as one, two of the middle ones
// as long as one after the other; prologue and epilogue 2, 3 or 5; a split
// costs the launch that joins the parts (5) and their bytes at 4 TB/s.
// Measured against every shape and split (bf16 results, us): 64 x 4096 x 4096
// small 10.2, middle 12.7, in two parts 14.4; 64 x 16384 x 16384 small 38.2, in
// two parts 29.3, in three 30.4; 256 x 4096 x 25088 small 53.4, middle in four
// parts 30.3, large in eight 36.0; 1024 x 4096 x 4096 small 18.4, middle 16.1,
// large 25.0; 2048 x 4096 x 4096 32.5, 24.7, 28.6; 100 x 500 x 20000 small 26.7,
// in six parts 14.7.  256 x 128 tiles were not the fastest anywhere by more
// than a twentieth.
inline MxShape mx_product_plan(int64_t m, int64_t n, int64_t kp) {
    if (mx_few(m, n, kp)) return MxShape{1, 1, 1, 1};
    MxShape best{1, 1, 1, 0};
    double least = 1e30;
    const double stages = (double)(kp / 256);
    for (int t = 1; t <= 4; t *= 2) {
        const double tiles = (double)((m + 64 * t - 1) / (64 * t)) * (double)((n + 64 * t - 1) / (64 * t));
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (s > 1 && stages < 4 * s) break;
            const double load = tiles * s / 256;  // blocks of a CU
            double us = stages / s;
            if (t == 1) us = us * 0.55 * std::max(1.0, 0.5 * load) + 2 * std::max(1.0, load / 4);
            else if (t == 2) us = us * 0.68 * std::max(1.0, load) + 3 * std::max(1.0, load / 2);
            else us = (us * (load > 0.75 ? 1.9 : 1.35) + 5) * std::max(1.0, std::ceil(load));
            if (s > 1) us += 5 + 8e-6 * (double)m * (double)n / 4 * s;
            if (us < least) {
                least = us;
                best = MxShape{t, t, s, 0};
            }
        }
    }
    return best;
}

// Weak for the same reason as the clipping launchers.
__attribute__((weak)) hipError_t launch_mx_quantize(const MxQuantArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_mx_dequantize(const MxDequantArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_mx_product(const MxProductArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_mx_linear(const MxProductArgs&, const void* x, bool bf16, int64_t stride,
                                                  int64_t k, hipStream_t);

}  // namespace ags
