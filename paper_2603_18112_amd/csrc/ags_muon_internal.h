// Internal declarations of the orthogonalised updates (include/ags_muon.h),
// shared by their host code and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <functional>
#include <vector>

#include "ags_gemm_internal.h"
#include "ags_muon.h"

namespace ags {

// Matrices with a side of up to this many are orthogonalised in 64 bits: X = Q U, Q a
// polynomial in the small matrix U U' alone, so that two passes over U are all.  With so few
// singular values the roundings of 16-bit operands do not average out: up to 0.9 % of the
// result with 1 to 4 of them, 0.3 % from 8 on.
constexpr int32_t kMuonThin = 16;
// Elements of the longer side that a block takes at once, of at most 256 blocks.
constexpr int32_t kMuonThinCols = 128;
// How their Q is made: by steps on U U' or by its eigenvalues; by how much the steps may multiply a
// singular value in all for the first (ags_muon.hip).
enum MuonThinWay : int32_t { kThinSteps = 0, kThinEigen = 1 };
constexpr double kThinStepsGain = 262144.0;
inline MuonThinWay muon_thin_way(double gain) {
    return gain <= kThinStepsGain ? kThinSteps : kThinEigen;
}

// What stands in a matrix's part of the workspace: X in fp32 (before the first
// step: what is to be orthogonalised), X as operands (two, read and written in
// turn), A and b A + c A A as operands, partial sums of squares.  Operands' rows
// are padded with zeros to whole stages of a product.  Of a thin one only sums of products over
// parts of the longer side, and for a handle's, before them, U as the flat buffers hold it.
struct MuonMatrix {
    int64_t offset;         // elements, in w, m and the gradients; or 0
    int64_t ws;             // bytes, in the workspace
    int32_t rows, cols;
    int32_t chunks, chunk;  // for passes over the elements: blocks, and pieces of 8 elements of each
    float scale;
    int32_t parts, part;    // thin ones: blocks along the longer side, and elements of it for each
    int32_t kept;           // a handle's

    __host__ __device__ int64_t side() const { return rows < cols ? rows : cols; }
    __host__ __device__ bool tall() const { return rows > cols; }
    __host__ __device__ int64_t pitch() const { return (cols + 63) / 64 * 64; }       // of X, elements
    __host__ __device__ int64_t a_pitch() const { return (side() + 63) / 64 * 64; }   // of A
    __host__ __device__ int64_t x_at() const { return ws; }
    __host__ __device__ int64_t operand_at(int i) const { return ws + rows * pitch() * (4 + 2 * i); }
    __host__ __device__ int64_t a_at() const { return ws + rows * pitch() * 8; }
    __host__ __device__ int64_t b_at() const { return a_at() + side() * a_pitch() * 2; }
    __host__ __device__ int64_t sums_at() const { return b_at() + side() * a_pitch() * 2; }
    __host__ __device__ int64_t padded_bytes() const { return sums_at() - ws + (chunks * 8 + 63) / 64 * 64; }
    // Thin ones (kMuonThin).
    __host__ __device__ bool thin() const { return side() <= kMuonThin; }
    __host__ __device__ int64_t length() const { return rows < cols ? cols : rows; }
    __host__ __device__ int64_t elements() const { return (int64_t)rows * cols; }
    __host__ __device__ int64_t parts_at() const { return ws + (kept ? (elements() * 4 + 63) / 64 * 64 : 0); }
    __host__ __device__ int64_t bytes() const {
        if (!thin()) return padded_bytes();
        const int64_t sums = (int64_t)parts * kMuonThin * kMuonThin * 8;
        if (kept) return parts_at() - ws + sums;
        // (a small one's workspace is as large as if it were padded, which callers may count on)
        const int64_t padded = padded_bytes() + sums, least = sums > 65536 ? sums : 65536;
        return padded < least ? padded : least;
    }
};

inline MuonMatrix muon_matrix(int64_t offset, int64_t rows, int64_t cols, double scale, bool kept) {
    MuonMatrix m{};
    m.offset = offset;
    m.kept = kept;
    m.rows = (int32_t)rows;
    m.cols = (int32_t)cols;
    m.scale = (float)scale;
    const int64_t pieces = m.thin() && kept ? (m.elements() + 7) / 8 : rows * (m.pitch() / 8);
    m.chunk = (int32_t)std::max<int64_t>(512, gemm_up((pieces + 1023) / 1024, 256));
    m.chunks = (int32_t)((pieces + m.chunk - 1) / m.chunk);
    m.part = (int32_t)(gemm_up((m.length() + 255) / 256, kMuonThinCols));
    m.parts = (int32_t)((m.length() + m.part - 1) / m.part);
    return m;
}

struct MuonTile {
    int32_t matrix, i, j, reserved;
};

// Which blocks do what: tables on the device (a handle's matrices), or one
// matrix and `batch` like it, one after the other in the workspace.
struct MuonWork {
    const MuonMatrix* matrices;  // NULL: `one`
    const MuonTile* tiles;       // of the launch: tiles of an output, or (matrix, chunk)
    MuonMatrix one;
    int32_t blocks;      // in all
    int32_t each;        // without a table: of a matrix
    int32_t tiles_n;     // without a table: tiles to a row; 0: those not above the diagonal
    int32_t t;           // a tile's side is 64 t
    int32_t stages;      // the shortest contracted axis, in stages of 64
};

struct MuonRates {
    float lr, decay;     // decay: 1 - lr weight_decay
};

struct MuonStepArgs {
    MuonWork work;
    char* ws;
    // Where U comes from: replicas and momentum, or a tensor.
    const void* grads;
    int64_t stride, batch_stride, row_stride;
    int32_t K, bf16, nesterov, from_x;
    float momentum;
    float* m;
    double eps;
};

enum MuonResult : int32_t { kMuonMiddle = 0, kMuonWeights = 1, kMuonOut = 2 };

struct MuonProductArgs {
    MuonWork work;
    char* ws;
    float a, b, c;
    int32_t turn;        // which operand form of X is read
    int32_t result;      // what a step's X becomes
    float* w;
    const MuonRates* rates;
    void* out;
    int64_t out_batch_stride, out_stride;
    int32_t out_bf16;
};

struct MuonThinArgs {
    MuonStepArgs in;     // (its work: a block for each part)
    MuonProductArgs out;
    int32_t steps;
    int32_t way;         // a MuonThinWay
    double abc[3 * AGS_MUON_MAX_STEPS];
};

struct MuonProduct {
    int64_t m, n, k, count;
    bool symmetric;
};

inline int64_t muon_tiles(const MuonProduct& p, int t) {
    const int64_t tm = (p.m + 64 * t - 1) / (64 * t), tn = (p.n + 64 * t - 1) / (64 * t);
    return p.symmetric ? tm * (tm + 1) / 2 : tm * tn;
}

// The tile side for a launch of products: the least estimated time, the tiles going to
// the CUs the longest first.  Cold operands and the longer ends of these kernels
// cost 2.5, 6 and 12 us a launch more than gemm_alone says, and long launches with
// tiles of 128 squared half as much again: the power limit leaves them less of the clock.
// Within 2 % of the fastest of the choices for each launch of ResNet-50's matrices,
// VGG-16's classifier, eight 512 x 2048 and 1000 x 512; the launches by themselves, tiles of
// 64 / 128 / 256 squared (us): VGG-16's A - / 718 / 524, its A A - / 163 / 208, its X - /
// 1115 / 1007, eight A of 512 x 2048 16.7 / 20.7 / -.  Tiles of 128 x 64 gained nothing: those
// eight 16.6, ResNet-50's A 43 against 39.
inline int muon_tile_side(const std::vector<MuonProduct>& v) {
    int best = 1;
    double least = 1e30;
    for (int t : {1, 2, 4}) {
        double sum = 0, longest = 0;
        int64_t tiles = 0;
        for (const MuonProduct& p : v) {
            const double stages = (double)((p.k + 63) / 64);
            const int64_t n = muon_tiles(p, t) * p.count;
            tiles += n;
            sum += (double)n * gemm_among(t, stages);
            longest = std::max(longest, gemm_alone(t, stages));
        }
        double us = sum / 256 + longest;
        if (v.size() == 1) {
            us = tiles <= 256 ? longest
                              : std::max(longest, (double)((tiles + 255) / 256) * gemm_among(t, (double)((v[0].k + 63) / 64)));
        } else if (tiles <= 16384) {
            std::vector<double> each, cu(256, 0.0);
            for (const MuonProduct& p : v)
                each.insert(each.end(), (size_t)(muon_tiles(p, t) * p.count), gemm_among(t, (double)((p.k + 63) / 64)));
            std::sort(each.begin(), each.end(), std::greater<double>());
            us = longest;
            for (double d : each) {
                std::pop_heap(cu.begin(), cu.end(), std::greater<double>());
                cu.back() += d;
                if (cu.back() > d) us = std::max(us, cu.back());
                std::push_heap(cu.begin(), cu.end(), std::greater<double>());
            }
        }
        if (sum > 256 * 150 && t < 4) us *= 1.5;
        us += t == 4 ? 12 : t == 2 ? 6 : 2.5;
        if (us < least) {
            least = us;
            best = t;
        }
    }
    return best;
}

// Weak for the same reason as the clipping launchers.
__attribute__((weak)) hipError_t launch_muon_sum(const MuonStepArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_muon_start(const MuonStepArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_muon_thin(const MuonThinArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_muon_gram(const MuonProductArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_muon_square(const MuonProductArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_muon_apply(const MuonProductArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_muon_rates(MuonRates*, MuonRates, hipStream_t);

}  // namespace ags
