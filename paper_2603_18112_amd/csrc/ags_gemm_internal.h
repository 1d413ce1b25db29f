// How products of 16-bit operands are cut into blocks (ags_gemm_device.h).
#pragma once

#include <stdint.h>

#include <algorithm>

namespace ags {

// Tiles of 64 tm x 64 tn outputs (4 x 4, 2 x 2, 2 x 1 or 1 x 1), the contracted axis in
// `splits` parts.
struct GemmShape {
    int32_t tm, tn, splits;
};

// (a positive number's, without the library's call)
inline double gemm_ceil(double x) {
    const double down = (double)(int64_t)x;
    return down < x ? down + 1 : down;
}
constexpr int64_t gemm_tiles(int64_t x, int32_t t) { return (x + 64 * t - 1) / (64 * t); }

// A launch of blocks of 256 threads holds fewer than 2^32 threads.
constexpr int64_t kGemmMaxBlocks = ((int64_t)1 << 24) - 1;

constexpr int64_t gemm_up(int64_t x, int64_t unit) { return (x + unit - 1) / unit * unit; }

// The time of a tile of 64 t squared in us, its axis `stages` stages of 64 long: by itself
// on a CU, and of each of as many as a CU holds at once.
constexpr double gemm_alone(int t, double stages) {
    return t == 1 ? stages * 0.235 + 1.6 : t == 2 ? stages * 0.38 + 2.6 : stages * 1.05 + 7.5;
}
constexpr double gemm_among(int t, double stages) {
    return t == 1 ? stages * 0.233 + 0.8 : t == 2 ? stages * 0.42 + 1.6 : stages * 1.32 + 7.5;
}

// The tile and the split with the least estimated time in us.  A split costs the
// launch that joins the parts and their bytes.  Fitted to the times of every
// tile and split (up to 16) for 4400 products of 33 .. 8192 x 128 .. 32768 over 33 ..
// 32768, all three forms, operands from the caches, in graphs (tiles of 128 x 64 to
// the picks, not the times): the pick is 1.2 % slower than the best on average, 8 % at the
// 95th percentile, 40 % at worst (153 x 8064 over 32352: 194 us where tiles of 256
// in eight parts take 138); without tiles of 128 x 64 1.9 and 12 %.
inline GemmShape gemm_plan(int64_t m, int64_t n, int64_t k) {
    constexpr GemmShape kShapes[] = {{1, 1, 1}, {2, 1, 1}, {2, 2, 1}, {4, 4, 1}};
    int64_t tiles[4];
    for (int i = 0; i < 4; ++i) tiles[i] = gemm_tiles(m, kShapes[i].tm) * gemm_tiles(n, kShapes[i].tn);
    GemmShape best = kShapes[0];
    double least = 1e30;
    const int64_t all = (k + 63) / 64;
    for (int32_t s : {1, 2, 3, 4, 6, 8, 12, 16}) {
        if (s > 1 && (all < 2 * s || m * n >= (int64_t)1 << 31)) break;
        const double stages = (double)((all + s - 1) / s);
        const double join = s > 1 ? 3.2 + 0.21 * s + 1.58e-6 * (double)m * (double)n * s : 0.0;
        for (int i = 0; i < 4; ++i) {
            const GemmShape& p = kShapes[i];
            if (p.tm < 4 && tiles[i] * s > kGemmMaxBlocks) continue;
            const double load = (double)(tiles[i] * s) * (1.0 / 256);  // blocks of a CU
            double us = join;
            if (p.tm == 1) us += load <= 1.2 ? gemm_alone(1, stages) : gemm_among(1, stages) * gemm_ceil(load * 4) * 0.25;
            else if (p.tn == 1)
                us += load <= 1 ? stages * 0.231 + 1.84 : (stages * 0.381 + 1.25) * std::max(1.225, gemm_ceil(load * 2) * 0.5);
            else if (p.tm == 2) us += load <= 1 ? gemm_alone(2, stages) : gemm_among(2, stages) * std::max(1.85, gemm_ceil(load));
            else us += load <= 0.75 ? gemm_alone(4, stages) : gemm_among(4, stages) * gemm_ceil(load);
            if (us < least) {
                least = us;
                best = GemmShape{p.tm, p.tn, s};
            }
        }
    }
    return best;
}

}  // namespace ags
