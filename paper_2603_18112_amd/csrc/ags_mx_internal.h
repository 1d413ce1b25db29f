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

// The kernel for few rows is one launch with no parts to join, but reads x's
// codes from the caches once for each 16 rows of w and waits for memory chunk by
// chunk; the tiles load ahead.  Against tiles of 64 squared, with the launch that
// joins their parts (in brackets) where those are faster, weights from memory,
// kernels' times in us: 8 rows 4096 x 4096 4.7 against 7.4, 16 rows 5.2 / 7.3, 32
// rows 6.5 / 7.4; 16 rows 4096 x 25088 16.0 / 12.8 (+ 2.9), 32 rows 22.3 / 13.0
// (+ 2.9); 16 rows 1000 x 4096 4.6 / 7.2, 32 rows 5.8 / 7.2; where w's rows make
// a tile for every CU, 1 row 16384 x 16384 28.5 / 32.6, 8 rows 32.9 / 32.2, 16 rows
// 35.6 / 31.8, 32 rows 50 / 32.3; 16 rows 16384 x 4096 13.7 / 9.8, 9 rows 16384 x
// 2048 7.3 / 6.8; with tiles for half of them, 9 rows 8192 x 4096 7.5 / 8.4, 16 rows
// 8.0 / 8.4.  More than 16 rows of few, long rows of w, the launch that joins
// included: 23 x 692 x 14723 11.6 / 8.5, 20 x 1970 x 9049 8.1 / 8.8, 32 x 1780 x
// 4959 6.5 / 7.5.  For up to 16 rows of few, long rows of w the rule is not the
// faster one: a block goes through its rows' whole length.  Against 16 parts, 10
// rows 256 x 25088 11.5 / 8.9, 256 x 65536 25.8 / 11.1, 256 x 2^20 398 / 81 (64 parts:
// 44); 1 row 256 x 25088 8.4 / 8.4, 512 x 65536 24.6 / 12.2, 282 x 23778 8.2 / 8.7.
inline bool mx_few(int64_t m, int64_t n, int64_t kp) {
    if (n >= 8192) return m <= 8;
    return m <= 16 || (m <= 32 && kp <= 12288 && n * kp <= ((int64_t)1 << 24));
}

// Does ags_mx_linear take x to 4 bits in the product's kernel?  Every block
// does so then; it keeps x in LDS.  One launch against two, us a call bound by
// the host / in a graph: 1 row 4096 x 4096 9.0 / 3.8 against 13.1 / 5.2, 8 rows
// (32768 elements of x) 9.0 / 5.3 against 13.3 / 5.9, 16 rows (65536) 9.1 / 7.3
// against 13.4 / 6.4; in a graph, weights from memory, 1 row 16384 x 16384 30.5
// against 32.1, 4 rows 16384 x 8192 20.6 / 20.4, 16 rows 8192 x 2048 7.4 / 7.7.  Where
// the product alone would take tiles (mx_few: more than 8 rows, wide weights) the
// rule gains on the host what it loses on the card: 9 rows 16384 x 2048 9.3 / 9.3,
// 16 rows 12.1 / 9.2; 9 rows 25088 x 3584 22.5 / 15.4, which is lost.
inline bool mx_linear_fused(int64_t rows, int64_t k) { return rows <= 16 && rows * k <= 32768; }

// The tile and the split with the least estimated time in us.  A stage (256
// columns) of a tile of 64 squared takes 0.26 on a CU, its prologue and epilogue
// 1.4, and as much again for each further one on the CU; a stage of 128 squared
// 0.34, or 0.68 for each of more than one; of 256 squared 1.3, or 1.7 with all
// CUs at work, at the clock the power limit leaves; their prologues and epilogues
// 4 and 5; a split costs the launch that joins the parts (3.2) and their bytes, 8
// a result, at 6 TB/s.  Fitted to the times of every shape and split for 320
// products, most of them drawn over 5 to 25000 a side, bf16 and fp32, aligned and
// odd; the shape this picks is 1% slower than the best one on average, 22% at
// worst. What takes under 9 in one launch stays so: two take the host that long
// (443 x 288 x 5178 of a forward pass 14.2 us a call against 16.0 in four parts).
// Some of them (us in a graph, from memory, small / middle / large, in their best
// number of parts if it is not one): 64 x 4096 x 4096 7.3 / 11.2 / 17.9 in four;
// 64 x 16384 x 16384 35.2 / 41.4 in four / 49.9 in four; 24 x 4096 x 25088 16.3
// in four / 18.5 in eight / 27.7 in sixteen; 256 x 4096 x 25088 33.6 / 32.3 in
// four / 40.5 in twelve; 500 x 500 x 20000 13.1 in four / 15.1 in eight / 24.9 in
// sixteen; 496 x 3840 x 21760 49.6 / 39.3 in two / 45.6 in eight; 512 x 4096 x
// 8192 21.6 / 22.7 / 32.9 in four; 1024 x 4096 x 4096 19.6 / 14.3 / 29.6; 1500 x
// 1500 x 6000 18.8 / 16.6 / 28.1 in four; 2048 x 4096 x 4096 39.5 / 25.7 / 35.8;
// 3000 cubed 36.2 / 33.6 / 29.2; 4096 x 4096 x 1024 28.3 / 22.5 / 19.6; 14208 x
// 15616 x 100 168.1 / 117.5 / 125.2. 256 x 128 tiles were not the fastest
// anywhere by more than a twentieth.
inline MxShape mx_product_plan(int64_t m, int64_t n, int64_t kp) {
    if (mx_few(m, n, kp)) return MxShape{1, 1, 1, 1};
    MxShape best{1, 1, 1, 0};
    double least = 1e30;
    const double stages = (double)(kp / 256);
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
        if (s > 1 && (stages < 4 * s || m * n >= (int64_t)1 << 31)) break;  // (mx_join_kernel)
        if (s == 2 && least < 9) break;
        for (int t = 1; t <= 4; t *= 2) {
            const double tiles = (double)((m + 64 * t - 1) / (64 * t)) * (double)((n + 64 * t - 1) / (64 * t));
            const double load = tiles * s / 256;  // blocks of a CU
            double us = stages / s;
            if (t == 1) us = (us * 0.26 + 1.4) * std::max(1.0, load);
            else if (t == 2) us = us * (load > 1 ? 0.68 * load : 0.34) + 4 * std::max(1.0, load / 10);
            else us = (us * (load > 0.75 ? 1.7 : 1.3) + 5) * std::max(1.0, std::ceil(load));
            if (s > 1) us += 3.2 + 1.3e-6 * (double)m * (double)n * s;
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
