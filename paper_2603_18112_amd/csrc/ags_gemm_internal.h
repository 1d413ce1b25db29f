// How products of 16-bit operands are cut into blocks (ags_gemm_device.h).
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace ags {

// Tiles of 64 t x 64 t outputs, the contracted axis in `splits` parts.
struct GemmShape {
    int32_t t, splits;
};

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
// tile and split (up to 16) for 4428 products of 33 .. 8192 x 128 .. 32768 over 33 ..
// 32768, all three forms, operands from the caches, in graphs: the pick is 1.1 %
// slower than the best on average, 9 % at the 95th percentile, 35 % at worst (35 x
// 5888 over 25152: 86 us where tiles of 128 in four parts take 64).
inline GemmShape gemm_plan(int64_t m, int64_t n, int64_t k) {
    GemmShape best{1, 1};
    double least = 1e30;
    const double all = (double)gemm_up(k, 64) / 64;
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
        if (s > 1 && (all < 2 * s || m * n >= (int64_t)1 << 31)) break;
        const double stages = std::ceil(all / s);
        for (int t = 1; t <= 4; t *= 2) {
            const int64_t blocks = ((m + 64 * t - 1) / (64 * t)) * ((n + 64 * t - 1) / (64 * t));
            if (t < 4 && blocks > kGemmMaxBlocks / s) continue;
            const double tiles = (double)blocks;
            const double load = tiles * s / 256;  // blocks of a CU
            double us;
            if (t == 1) us = load <= 1.2 ? gemm_alone(t, stages) : gemm_among(t, stages) * std::ceil(load * 4) / 4;
            else if (t == 2) us = load <= 1 ? gemm_alone(t, stages) : gemm_among(t, stages) * std::max(1.85, std::ceil(load));
            else us = load <= 0.75 ? gemm_alone(t, stages) : gemm_among(t, stages) * std::ceil(load);
            if (s > 1) us += 3.2 + 0.21 * s + 1.58e-6 * (double)m * (double)n * s;
            if (us < least) {
                least = us;
                best = GemmShape{t, s};
            }
        }
    }
    return best;
}

}  // namespace ags
