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

constexpr int64_t gemm_up(int64_t x, int64_t unit) { return (x + unit - 1) / unit * unit; }

// The tile and the split with the least estimated time in us.
inline GemmShape gemm_plan(int64_t m, int64_t n, int64_t k) {
    GemmShape best{1, 1};
    double least = 1e30;
    const double stages = (double)gemm_up(k, 64) / 64;
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
        if (s > 1 && (stages < 4 * s || m * n >= (int64_t)1 << 31)) break;
        for (int t = 1; t <= 4; t *= 2) {
            const double tiles = (double)((m + 64 * t - 1) / (64 * t)) * (double)((n + 64 * t - 1) / (64 * t));
            const double load = tiles * s / 256;  // blocks of a CU
            double us = stages / s;
            if (t == 1) us = (us * 0.26 + 1.4) * std::max(1.0, load);
            else if (t == 2) us = us * (load > 1 ? 0.5 * load : 0.34) + 4 * std::max(1.0, load / 10);
            else us = (us * (load > 0.75 ? 1.5 : 1.3) + 5) * std::max(1.0, std::ceil(load));
            if (s > 1) us += 3.2 + 1.3e-6 * (double)m * (double)n * s;
            if (us < least) {
                least = us;
                best = GemmShape{t, s};
            }
        }
    }
    return best;
}

}  // namespace ags
