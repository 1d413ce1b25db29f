// gfx950 kernels of the orthogonalised updates (include/ags_muon.h).
//
// muon_sum_kernel     the replicas' mean, the momentum, U; sums of its squares
// muon_start_kernel   X = U / (|U| + eps), as fp32 and as operands
// muon_gram_kernel    A = X X' (or X' X)
// muon_square_kernel  b A + c A A
// muon_apply_kernel   X <- a X + (b A + c A A) X; the last one updates the weights
// muon_thin_gram_kernel, muon_thin_apply_kernel   both for thin matrices, all steps in one;
//                     muon_thin_eigen_kernel   between them for long schedules
//
// Every launch covers all matrices: a block finds its tile in a table, or from
// its number where all matrices are alike.
//
// Measured (us): sum and start, bound by memory, for ResNet-50's 25.5 M elements from 16 bf16
// replicas 230 and 46 (4.9 and 5.5 TB/s), for the 123.6 M of VGG-16's classifier from 4 fp32
// replicas 733 and 249 (4.7 and 5.0).  A step of the latter: A 525 to 550 (the 136 tiles of
// 4096 x 25088 leave CUs idle; matrix pipes busy 76 %), A A 165, X 1010 to 1050 (1.0 PFLOP/s;
// X in fp32, read and written as a tile ends, stands beside the products).  A step of
// ResNet-50's 54 matrices: 33 (one operand's reads by XCD, and its longest tiles), 17, 72
// (380 MB: 5.3 TB/s).  1000 x 512: 8, 6 and 6, each a launch and its waits for memory.
#include "ags_gemm_device.h"
#include "ags_muon_internal.h"

namespace ags {
namespace {

using gemm::Side;
using gemm::store8;
using mx::load8;
using mx::Unaligned;
typedef unsigned short u16;
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// Powers of two that bring the operands into fp16's range, whose largest number is 2^16 - 2^5: X and A
// have singular values up to 1.41 and 1.988, b A + c A A up to 3.99, roundings included (the
// schedule is checked for these); elements down to 2^-14 of the scale keep 11 bits.  (The usual
// coefficients: 1.25, 1.56, 2.84.)
constexpr float kScaleX = 32768.0f, kScaleA = 32768.0f, kScaleB = 16384.0f;

__device__ __forceinline__ unsigned pack_half(float x, float y) {
    const v2h v = __builtin_convertvector((mx::v2f{x, y}), v2h);
    unsigned u;
    __builtin_memcpy(&u, &v, 4);
    return u;
}

// 8 elements as fp16 to an aligned place, zeros from `left` on.
__device__ __forceinline__ void store_half8(u16* p, int64_t left, const float* x) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = i < left ? x[i] : 0.0f;
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack_half(y[0], y[1]), pack_half(y[2], y[3]), pack_half(y[4], y[5]), pack_half(y[6], y[7]));
}

// The matrix of this block and its number in it (i, j: its tile; i: its chunk).
// Blocks of one matrix go to one XCD as far as that balances: blocks b, b + 8,
// ... share one.
struct Found {
    MuonMatrix m;
    int64_t index;  // in a batch
    int32_t i, j;
};

template <bool TILES>
__device__ __forceinline__ Found find(const MuonWork& w) {
    Found f;
    if (w.tiles) {
        const MuonTile t = w.tiles[blockIdx.x];
        f.m = w.matrices[t.matrix];
        f.index = 0;
        f.i = t.i;
        f.j = t.j;
        return f;
    }
    const unsigned total = (unsigned)w.blocks, xcd = blockIdx.x % tile::kXcds, at = blockIdx.x / tile::kXcds;
    const unsigned base = total / tile::kXcds, rest = total % tile::kXcds;
    const unsigned b = xcd * base + min(xcd, rest) + at;
    f.m = w.one;
    f.index = b / (unsigned)w.each;
    const unsigned t = b % (unsigned)w.each;
    f.m.ws += f.index * f.m.bytes();
    if (!TILES) {
        f.i = (int)t;
        f.j = 0;
    } else if (w.tiles_n) {
        f.i = (int)(t / (unsigned)w.tiles_n);
        f.j = (int)(t % (unsigned)w.tiles_n);
    } else {  // t = i (i + 1) / 2 + j, j <= i
        int i = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1) / 2 > (int)t) --i;
        while ((i + 1) * (i + 2) / 2 <= (int)t) ++i;
        f.i = i;
        f.j = (int)t - i * (i + 1) / 2;
    }
    return f;
}

// ------------------------------------------------------------- elements --

constexpr int kThreads = 256;

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Eight elements of the tensor that is orthogonalised.
__device__ __forceinline__ void load_x(const MuonStepArgs& a, const Found& f, int64_t row, int64_t c, float* x) {
    const int64_t at = f.index * a.batch_stride + row * a.row_stride + c, left = f.m.cols - c;
    if (a.bf16) load8(static_cast<const u16*>(a.grads) + at, left, x);
    else load8(static_cast<const float*>(a.grads) + at, left, x);
}

template <typename T>
__device__ __forceinline__ void mean8(const MuonStepArgs& a, int64_t at, int64_t left, float* g) {
    const T* p = static_cast<const T*>(a.grads) + at;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 0.0f;
    int k = 0;
    for (; k + 4 <= a.K; k += 4) {
        float y[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) load8(p + (k + u) * a.stride, left, y[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] += y[u][i];
    }
    for (; k < a.K; ++k) {
        float y[8];
        load8(p + k * a.stride, left, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] += y[i];
    }
    const float n = (float)a.K;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] /= n;
}

// A chunk's pieces of 8 elements, thread after thread.  A thin matrix (a handle's) is one row of
// all its elements (room for the last eight included), and its squares are summed with its products.
__global__ __launch_bounds__(kThreads) void muon_sum_kernel(MuonStepArgs a) {
    __shared__ double red[4];
    const Found f = find<false>(a.work);
    const bool thin = f.m.thin();
    const int cols = thin ? f.m.rows * f.m.cols : f.m.cols;
    const unsigned per_row = thin ? (unsigned)(cols + 7) / 8 : (unsigned)(f.m.pitch() / 8);
    const unsigned total = thin ? per_row : (unsigned)f.m.rows * per_row;
    const unsigned end = min(total, (unsigned)(f.i + 1) * (unsigned)f.m.chunk);
    double sum = 0.0;
    for (unsigned p = (unsigned)f.i * (unsigned)f.m.chunk + threadIdx.x; p < end; p += kThreads) {
        const int64_t row = p / per_row, c = (int64_t)(p - (unsigned)row * per_row) * 8, left = cols - c;
        if (left <= 0) continue;
        float u[8];
        if (a.from_x) {
            load_x(a, f, row, c, u);
        } else {
            const int64_t at = f.m.offset + row * cols + c;
            float m[8];
            load8(a.m + at, left, m);
            if (a.bf16) mean8<u16>(a, at, left, u);
            else mean8<float>(a, at, left, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m[i] = fmaf(a.momentum, m[i], u[i]);
                u[i] = a.nesterov ? fmaf(a.momentum, m[i], u[i]) : m[i];
            }
            store8(a.m + at, left, m);
            // (past the row's end u is 0)
            store8(reinterpret_cast<float*>(a.ws + f.m.x_at()) + row * f.m.pitch() + c, 8, u);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fma((double)u[i], (double)u[i], sum);
    }
    if (thin) return;
    sum = block_sum(sum, red);
    if (threadIdx.x == 0) reinterpret_cast<double*>(a.ws + f.m.sums_at())[f.i] = sum;
}

__global__ __launch_bounds__(kThreads) void muon_start_kernel(MuonStepArgs a) {
    __shared__ double red[4];
    const Found f = find<false>(a.work);
    const double* sums = reinterpret_cast<const double*>(a.ws + f.m.sums_at());
    double sum = 0.0;
    for (int i = threadIdx.x; i < f.m.chunks; i += kThreads) sum += sums[i];
    const double inv = 1.0 / (sqrt(block_sum(sum, red)) + a.eps);
    const int64_t pitch = f.m.pitch();
    const unsigned per_row = (unsigned)(pitch / 8), total = (unsigned)f.m.rows * per_row;
    const unsigned end = min(total, (unsigned)(f.i + 1) * (unsigned)f.m.chunk);
    float* x = reinterpret_cast<float*>(a.ws + f.m.x_at());
    u16 *h = reinterpret_cast<u16*>(a.ws + f.m.operand_at(0)), *h1 = reinterpret_cast<u16*>(a.ws + f.m.operand_at(1));
    for (unsigned p = (unsigned)f.i * (unsigned)f.m.chunk + threadIdx.x; p < end; p += kThreads) {
        const int64_t row = p / per_row, c = (int64_t)(p - (unsigned)row * per_row) * 8, at = row * pitch + c;
        float u[8] = {};
        if (c < f.m.cols) {
            if (a.from_x) load_x(a, f, row, c, u);
            else load8(x + at, 8, u);
            // a zero matrix stays zero with eps = 0 too
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = u[i] == 0.0f ? 0.0f : (float)((double)u[i] * inv);
        }
        store8(x + at, 8, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] *= kScaleX;
        store_half8(h + at, 8, u);
        // the second form's padding, which the products never write
        if (c + 8 > f.m.cols) {
            const float zero[8] = {};
            store_half8(h1 + at, 8, zero);
        }
    }
    // that of A and b A + c A A
    const int64_t s = f.m.side(), ap = f.m.a_pitch(), from = s / 8 * 8, pads = (ap - from) / 8;
    if (s == ap) return;
    for (int64_t p = (int64_t)f.i * kThreads + threadIdx.x; p < s * pads; p += (int64_t)f.m.chunks * kThreads) {
        const int64_t at = p / pads * ap + from + p % pads * 8;
        const float zero[8] = {};
        store_half8(reinterpret_cast<u16*>(a.ws + f.m.a_at()) + at, 8, zero);
        store_half8(reinterpret_cast<u16*>(a.ws + f.m.b_at()) + at, 8, zero);
    }
}

// ------------------------------------------------------------- products --

// How a wave goes through 32 rows of fp32 results in LDS: eight of a row to a lane, from
// column `c` on, of the rows row(i).
template <int FN>
struct Walk {
    static constexpr int kLanes = FN * 4, kRows = 64 / kLanes, kSteps = 32 / kRows;
    int c, first, end;  // no rows where the lane's columns lie outside

    __device__ __forceinline__ Walk(int lane, int64_t rows, int64_t cols)
        : c(lane % kLanes * 8), first(lane / kLanes), end(c < cols ? (int)min(rows, (int64_t)32) : 0) {}
    __device__ __forceinline__ int row(int i) const { return first + i * kRows; }
    __device__ __forceinline__ bool has(int i) const { return row(i) < end; }
    __device__ __forceinline__ char* at(char* strip, int i) const { return strip + row(i) * gemm::kPitch<FN> + c * 4; }
};

// Tiles below the diagonal are stored above it too: four lanes take the strip's
// 32 rows of a column, 64 bytes of a row.
struct SymmetricOut {
    u16* to;             // A, or b A + c A A
    const u16* from;     // A, where the latter is made
    int64_t pitch;
    float add, times;    // x times + A add
    bool mirror;

    template <int FN>
    struct Old {
        uint4 v[Walk<FN>::kSteps];
    };
    template <int FN>
    __device__ __forceinline__ Old<FN> begin(int lane, int64_t row0, int64_t col0, int64_t rows, int64_t cols) const {
        const Walk<FN> walk(lane, rows, cols);
        Old<FN> old;
#pragma unroll
        for (int i = 0; i < walk.kSteps; ++i) {
            old.v[i] = make_uint4(0, 0, 0, 0);
            if (from && walk.has(i))
                old.v[i] = *reinterpret_cast<const uint4*>(from + (row0 + walk.row(i)) * pitch + col0 + walk.c);
        }
        return old;
    }

    template <int FN>
    __device__ __forceinline__ void band(const gemm::v16f (&acc)[FN], char* sm, int lane, int64_t row0, int64_t col0,
                                         int64_t rows, int64_t cols, const Old<FN>& old) const {
        const Walk<FN> walk(lane, rows, cols);
        gemm::to_strip<FN>(acc, sm, lane);
#pragma unroll
        for (int i = 0; i < walk.kSteps; ++i) {
            if (!walk.has(i)) continue;
            float x[8];
            gemm::read8(walk.at(sm, i), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= times;
            if (from) {
                const gemm::v8h y = __builtin_bit_cast(gemm::v8h, old.v[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fmaf((float)y[e], add, x[e]);
            }
            store_half8(to + (row0 + walk.row(i)) * pitch + col0 + walk.c, cols - walk.c, x);
            if (mirror) {
                float* p = reinterpret_cast<float*>(walk.at(sm, i));
                *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
            }
        }
        if (!mirror) return;
        gemm::lds_wait();
        const int t = (lane & 3) * 8;
        if (t >= rows) return;
#pragma unroll 2
        for (int c = lane >> 2; c < FN * 32; c += 16) {
            if (c >= cols) break;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = *reinterpret_cast<const float*>(sm + (t + i) * gemm::kPitch<FN> + c * 4);
            store_half8(to + (col0 + c) * pitch + row0 + t, rows - t, x);
        }
    }
};

struct ApplyOut {
    const MuonProductArgs& a;
    const Found& f;

    template <int FN>
    struct Old {
        float4 v[Walk<FN>::kSteps][2];
    };
    // (zero past the row's end)
    template <int FN>
    __device__ __forceinline__ Old<FN> begin(int lane, int64_t row0, int64_t col0, int64_t rows, int64_t cols) const {
        const Walk<FN> walk(lane, rows, cols);
        const int64_t pitch = f.m.pitch();
        const float* xs = reinterpret_cast<const float*>(a.ws + f.m.x_at()) + row0 * pitch + col0 + walk.c;
        Old<FN> old;
#pragma unroll
        for (int i = 0; i < walk.kSteps; ++i)
            if (walk.has(i)) {
                old.v[i][0] = *reinterpret_cast<const float4*>(xs + walk.row(i) * pitch);
                old.v[i][1] = *reinterpret_cast<const float4*>(xs + walk.row(i) * pitch + 4);
            }
        return old;
    }

    template <int FN>
    __device__ __forceinline__ void band(const gemm::v16f (&acc)[FN], char* sm, int lane, int64_t row0, int64_t col0,
                                         int64_t rows, int64_t cols, const Old<FN>& ahead) const {
        const Walk<FN> walk(lane, rows, cols);
        const int64_t pitch = f.m.pitch(), left = cols - walk.c, col = col0 + walk.c;
        float* xs = reinterpret_cast<float*>(a.ws + f.m.x_at()) + row0 * pitch + col;
        u16* h = reinterpret_cast<u16*>(a.ws + f.m.operand_at(a.turn ^ 1)) + row0 * pitch + col;
        float* w = a.w + f.m.offset + row0 * f.m.cols + col;
        const bool weights = a.result == kMuonWeights;
        gemm::to_strip<FN>(acc, sm, lane);
        const float rate = weights ? -a.rates->lr * f.m.scale : 0.0f, decay = weights ? a.rates->decay : 0.0f;
#pragma unroll
        for (int i = 0; i < walk.kSteps; ++i) {
            if (!walk.has(i)) continue;
            const int t = walk.row(i);
            const float old[8] = {ahead.v[i][0].x, ahead.v[i][0].y, ahead.v[i][0].z, ahead.v[i][0].w,
                                  ahead.v[i][1].x, ahead.v[i][1].y, ahead.v[i][1].z, ahead.v[i][1].w};
            float x[8];
            gemm::read8(walk.at(sm, i), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fmaf(a.a, old[e], x[e] * (1.0f / (kScaleB * kScaleX)));
            if (a.result == kMuonMiddle) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = e < left ? x[e] : 0.0f;
                float4* p = reinterpret_cast<float4*>(xs + t * pitch);
                p[0] = make_float4(x[0], x[1], x[2], x[3]);
                p[1] = make_float4(x[4], x[5], x[6], x[7]);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= kScaleX;
                store_half8(h + t * pitch, 8, x);
            } else if (weights) {
                float v[8];
                load8(w + (int64_t)t * f.m.cols, left, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(rate, x[e], v[e] * decay);
                store8(w + (int64_t)t * f.m.cols, left, v);
            } else {
                const int64_t o = f.index * a.out_batch_stride + (row0 + t) * a.out_stride + col;
                if (a.out_bf16) store8(static_cast<u16*>(a.out) + o, left, x);
                else store8(static_cast<float*>(a.out) + o, left, x);
            }
        }
    }
};

template <int T, int NA, int NB>
__global__ __launch_bounds__(256, 1) void muon_gram_kernel(MuonProductArgs a) {
    extern __shared__ __attribute__((aligned(16))) char sm[];
    const Found f = find<true>(a.work);
    const int64_t s = f.m.side(), pitch = f.m.pitch();
    const SymmetricOut out{reinterpret_cast<u16*>(a.ws + f.m.a_at()), nullptr, f.m.a_pitch(), 0.0f,
                           kScaleA / (kScaleX * kScaleX), f.i != f.j};
    const Side x{a.ws + f.m.operand_at(a.turn), pitch * 2, f.m.rows, pitch};
    const int64_t i0 = (int64_t)f.i * 64 * T, j0 = (int64_t)f.j * 64 * T;
    if (f.m.tall())
        gemm::product_tile<gemm::Fp16, T, T, NA, NB, gemm::kAlong, gemm::kAlong>(x, x, 0, (f.m.rows + 63) / 64, i0, j0, s, s, sm, out);
    else
        gemm::product_tile<gemm::Fp16, T, T, NA, NB, gemm::kAcross, gemm::kAcross>(x, x, 0, (int)(pitch / 64), i0, j0, s, s, sm, out);
}

template <int T, int NA, int NB>
__global__ __launch_bounds__(256, 1) void muon_square_kernel(MuonProductArgs a) {
    extern __shared__ __attribute__((aligned(16))) char sm[];
    const Found f = find<true>(a.work);
    const int64_t s = f.m.side(), pitch = f.m.a_pitch();
    const u16* gram = reinterpret_cast<const u16*>(a.ws + f.m.a_at());
    const SymmetricOut out{reinterpret_cast<u16*>(a.ws + f.m.b_at()), gram, pitch, a.b * (kScaleB / kScaleA),
                           a.c * (kScaleB / (kScaleA * kScaleA)), f.i != f.j};
    const Side x{gram, pitch * 2, s, 0};
    gemm::product_tile<gemm::Fp16, T, T, NA, NB, gemm::kAcross, gemm::kAcross>(x, x, 0, (int)(pitch / 64), (int64_t)f.i * 64 * T,
                                                           (int64_t)f.j * 64 * T, s, s, sm, out);
}

template <int T, int NA, int NB>
__global__ __launch_bounds__(256, 1) void muon_apply_kernel(MuonProductArgs a) {
    extern __shared__ __attribute__((aligned(16))) char sm[];
    const Found f = find<true>(a.work);
    const int64_t s = f.m.side(), pitch = f.m.pitch(), ap = f.m.a_pitch();
    const Side x{a.ws + f.m.operand_at(a.turn), pitch * 2, f.m.rows, pitch}, b{a.ws + f.m.b_at(), ap * 2, s, 0};
    const int64_t i0 = (int64_t)f.i * 64 * T, j0 = (int64_t)f.j * 64 * T;
    const ApplyOut out{a, f};
    if (f.m.tall())
        gemm::product_tile<gemm::Fp16, T, T, NA, NB, gemm::kAcross, gemm::kAcross>(x, b, 0, (int)(ap / 64), i0, j0, f.m.rows, f.m.cols, sm,
                                                               out);
    else
        gemm::product_tile<gemm::Fp16, T, T, NA, NB, gemm::kAcross, gemm::kAlong>(b, x, 0, (int)(ap / 64), i0, j0, f.m.rows, f.m.cols, sm,
                                                              out);
}

// ------------------------------------------------------------------ thin --

// A thin matrix as `n` columns of its shorter side, from c0 of the longer on, in LDS.
constexpr int kThin = kMuonThin, kThinCols = kMuonThinCols;
struct ThinTile {
    float v[kThin][kThinCols + 1];
};

// Calls f(i, c) for every element i of the shorter side and c of n of the longer,
// neighbours in memory by neighbouring threads.
template <typename F>
__device__ __forceinline__ void thin_each(bool tall, int s, int n, F&& f) {
    for (int t = threadIdx.x; t < s * n; t += kThreads) {
        if (tall) f(t % s, t / s);
        else f(t / n, t % n);
    }
}

__device__ __forceinline__ void thin_load(const MuonStepArgs& a, const Found& f, int64_t c0, int n, ThinTile& x) {
    const bool tall = f.m.tall();
    thin_each(tall, (int)f.m.side(), n, [&](int i, int c) {
        const int64_t row = tall ? c0 + c : i, col = tall ? i : c0 + c;
        float v;
        if (!a.from_x) {
            v = reinterpret_cast<const float*>(a.ws + f.m.x_at())[row * f.m.cols + col];
        } else {
            const int64_t at = f.index * a.batch_stride + row * a.row_stride + col;
            v = a.bf16 ? gemm::bf16_value(static_cast<const u16*>(a.grads)[at]) : static_cast<const float*>(a.grads)[at];
        }
        x.v[i][c] = v;
    });
}

// U U' (U' U) over a part of the longer side: a thread has one sum, whose products are
// exact in fp64.
__global__ __launch_bounds__(kThreads) void muon_thin_gram_kernel(MuonThinArgs a) {
    __shared__ ThinTile x;
    const Found f = find<false>(a.in.work);
    const int s = (int)f.m.side(), i = threadIdx.x / kThin, j = threadIdx.x % kThin;
    const int64_t from = (int64_t)f.i * f.m.part, end = min(f.m.length(), from + f.m.part);
    double sum = 0.0;
    for (int64_t c0 = from; c0 < end; c0 += kThinCols) {
        const int n = (int)min(end - c0, (int64_t)kThinCols);
        __syncthreads();
        thin_load(a.in, f, c0, n, x);
        __syncthreads();
        if (i < s && j < s)
#pragma unroll 4
            for (int c = 0; c < n; ++c) sum = fma((double)x.v[i][c], (double)x.v[j][c], sum);
    }
    reinterpret_cast<double*>(a.in.ws + f.m.parts_at())[(int64_t)f.i * kThreads + threadIdx.x] = sum;
}

struct ThinSquare {
    double v[kThin][kThin + 1];
};

__device__ __forceinline__ double thin_product(const ThinSquare& a, const ThinSquare& b, int i, int j) {
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < kThin; ++k) sum = fma(a.v[i][k], b.v[k][j], sum);
    return sum;
}

// Index i's partner in a round among m (even): every pair meets once in m - 1 rounds; an
// index past m is by itself.
__device__ __forceinline__ int thin_partner(int i, int round, int m) {
    const int n = m - 1;
    int p = 2 * round - i;
    p = p < 0 ? p + n : p >= n ? p - n : p;
    p = i == round ? n : p;
    p = i == n ? round : p;
    return i >= m ? i : p;
}
// Row i of the rotation that takes A's element (i, p) away: *self for i, the result for p.
// The angle is within 2^-22, the rotation's rows of length 1 in fp64.
__device__ __forceinline__ double thin_rotation(const ThinSquare& A, int i, int p, double* self) {
    const int lo = min(i, p), hi = max(i, p);
    const float off = (float)A.v[lo][hi];
    const bool none = i == p || fabsf(off) < 0x1p-100f;  // (no branch: two of these go on at once)
    const float d = (float)(A.v[hi][hi] - A.v[lo][lo]) * 0.5f * __builtin_amdgcn_rcpf(off), l = fabsf(d);
    const float root = l > 1e9f ? l : __builtin_amdgcn_sqrtf(fmaf(d, d, 1.0f));
    const double t = (double)copysignf(__builtin_amdgcn_rcpf(l + root), d);
    const double r = fma(t, t, 1.0);
    double c = (double)__builtin_amdgcn_rsqf((float)r);
#pragma unroll
    for (int k = 0; k < 2; ++k) c *= fma(-0.5 * r, c * c, 1.5);
    *self = none ? 1.0 : c;
    return none ? 0.0 : i == lo ? -t * c : t * c;
}

// Eigenvalues (the diagonal of A) and eigenvectors (columns of V) of A[0], of trace 1, by
// Jacobi's rotations, eight pairs at a time; returns which of the two buffers holds them.
// Off-diagonal elements vanish quadratically, in 4 to 8 sweeps in simulations of
// full, graded and repeated spectra; those below 2^-30 are cleared outright, what is left of them
// would be below 2^-52.  Elements between indices of no weight (below) do not matter.
__device__ __forceinline__ int thin_eigen(ThinSquare (&A)[2], ThinSquare (&V)[2], int s, int i, int j) {
    constexpr int kSweeps = 16;
    const int m = (s + 1) & ~1;
    int at = 0;
    V[0].v[i][j] = i == j ? 1.0 : 0.0;
    __syncthreads();
    for (int sweep = 0; sweep < kSweeps; ++sweep) {
        const bool left = i != j && fabs(A[at].v[i][j]) > 0x1p-80 && fmax(A[at].v[i][i], A[at].v[j][j]) > 0x1p-50;
        if (!__syncthreads_or(left)) break;
        for (int round = 0; round < m - 1; ++round, at ^= 1) {
            const ThinSquare &X = A[at], &W = V[at];
            const int p = thin_partner(i, round, m), q = thin_partner(j, round, m);
            double ci, cj;
            const double si = thin_rotation(X, i, p, &ci), sj = thin_rotation(X, j, q, &cj);
            const double u = fma(sj, X.v[i][q], cj * X.v[i][j]), v = fma(sj, X.v[p][q], cj * X.v[p][j]);
            const bool clear = i != j && p == j && fabs(X.v[min(i, j)][max(i, j)]) < 0x1p-30;
            const double a = fma(si, v, ci * u), w = fma(sj, W.v[i][q], cj * W.v[i][j]);
            A[at ^ 1].v[i][j] = clear ? 0.0 : a;
            V[at ^ 1].v[i][j] = w;
            __syncthreads();
        }
    }
    return at;
}

// A of a matrix, summed over its parts, its trace, and one over the norm.
__device__ __forceinline__ double thin_gram(const MuonStepArgs& a, const Found& f, ThinSquare& A, double* trace,
                                            double* inv) {
    const double* parts = reinterpret_cast<const double*>(a.ws + f.m.parts_at());
    double sum = 0.0;
#pragma unroll 8
    for (int k = 0; k < f.m.parts; ++k) sum += parts[(int64_t)k * kThreads + threadIdx.x];
    A.v[threadIdx.x / kThin][threadIdx.x % kThin] = sum;
    __syncthreads();
    *trace = 0.0;
    for (int k = 0; k < (int)f.m.side(); ++k) *trace += A.v[k][k];
    // a zero matrix stays zero with eps = 0 too
    *inv = *trace == 0.0 ? 0.0 : 1.0 / (sqrt(*trace) + a.eps);
    __syncthreads();
    return sum;
}

// X = Q U, Q U in fp64, in one of two ways, by how much the steps multiply a singular value near zero
// in all (kThinStepsGain): that is what they do to roundings in directions that U does not have.
//
// kThinSteps: by steps on A alone (p = a + b A + c A A: A <- p A p, Q <- p Q; the matrices are
// polynomials of one symmetric one and commute).  A's own roundings, 2^-53 of its trace, grow by p^2
// a step, and where they reach 1 the steps break off: by up to 2^36 here (ten usual steps).
// kThinEigen: by eigenvalues of A (muon_thin_eigen_kernel, a block to a matrix), each put through the
// steps by itself: Q has f(s) / s for the singular value s.  Those below 2^-46 of their sum,
// which A's own roundings reach (sums of up to 2^20 products), count as none: singular values
// under 2^-23 of |U|.
//
// In graphs (us), 5 / 10 / 11 / 32 usual steps, the last two by eigenvalues: 1 x 4096 17 / 23 / 14 /
// 15, 16 x 4096 26 / 32 / 93 / 95, 16 x 100 000 77 / 83 / 143 / 144, 24 of 16 x 8192 65 / 86 / 139 / 141
// (as the products above, five steps take 123, 124, 1914 and 286).  Bound by the waits of each
// launch and by fp64 in order; memory takes 3 us of the longest.  A round of rotations takes
// 0.65 us, a chain of LDS reads and some forty operations.
__global__ __launch_bounds__(kThreads) void muon_thin_eigen_kernel(MuonThinArgs a) {
    __shared__ ThinSquare A[2], V[2];
    const Found f = find<false>(a.in.work);
    if (f.i != 0) return;
    const int i = threadIdx.x / kThin, j = threadIdx.x % kThin;
    double trace, inv;
    const double sum = thin_gram(a.in, f, A[0], &trace, &inv);
    A[0].v[i][j] = trace > 0.0 ? sum / trace : 0.0;
    const int at = thin_eigen(A, V, (int)f.m.side(), i, j);
    // (a NaN or an infinity of U makes the trace one, and is not compared away)
    double q = trace < HUGE_VAL ? 0.0 : __builtin_nan("");
    if (A[at].v[j][j] > 0x1p-46) {
        double y = A[at].v[j][j] * trace * inv * inv;
        q = inv;
        for (int t = 0; t < a.steps; ++t) {
            const double p = fma(fma(a.abc[3 * t + 2], y, a.abc[3 * t + 1]), y, a.abc[3 * t]);
            q *= p;
            y *= p * p;
        }
    }
    A[at ^ 1].v[j][i] = V[at].v[i][j] * q;
    __syncthreads();
    // (in place of the first part, which no block reads any more)
    reinterpret_cast<double*>(a.in.ws + f.m.parts_at())[threadIdx.x] = thin_product(V[at], A[at ^ 1], i, j);
}

// The steps by every block anew, or what the eigenvalues' kernel left, then its part of Q U.
template <int WAY>
__global__ __launch_bounds__(kThreads) void muon_thin_apply_kernel(MuonThinArgs a) {
    __shared__ ThinTile x;
    __shared__ ThinSquare A, Q, P;
    const Found f = find<false>(a.in.work);
    const int s = (int)f.m.side(), i = threadIdx.x / kThin, j = threadIdx.x % kThin;
    if constexpr (WAY == kThinSteps) {
        double trace, inv;
        const double sum = thin_gram(a.in, f, A, &trace, &inv);
        A.v[i][j] = sum * inv * inv;
        Q.v[i][j] = i == j ? inv : 0.0;
        __syncthreads();
        for (int t = 0; t < a.steps; ++t) {
            const double p = fma(a.abc[3 * t + 2], thin_product(A, A, i, j),
                                 fma(a.abc[3 * t + 1], A.v[i][j], i == j ? a.abc[3 * t] : 0.0));
            P.v[i][j] = p;
            __syncthreads();
            const double pq = thin_product(P, Q, i, j), pa = thin_product(P, A, i, j);
            __syncthreads();
            Q.v[i][j] = pq;
            A.v[i][j] = pa;
            __syncthreads();
            const double pap = thin_product(A, P, i, j);
            __syncthreads();
            A.v[i][j] = pap;
            __syncthreads();
        }
    } else {
        Q.v[i][j] = reinterpret_cast<const double*>(a.in.ws + f.m.parts_at())[threadIdx.x];
    }
    const MuonProductArgs& o = a.out;
    const bool tall = f.m.tall(), weights = o.result == kMuonWeights;
    const float rate = weights ? -o.rates->lr * f.m.scale : 0.0f, decay = weights ? o.rates->decay : 0.0f;
    const int64_t from = (int64_t)f.i * f.m.part, end = min(f.m.length(), from + f.m.part);
    for (int64_t c0 = from; c0 < end; c0 += kThinCols) {
        const int n = (int)min(end - c0, (int64_t)kThinCols);
        __syncthreads();
        thin_load(a.in, f, c0, n, x);
        __syncthreads();
        thin_each(tall, s, n, [&](int r, int c) {
            double v = 0.0;
            for (int k = 0; k < s; ++k) v = fma(Q.v[r][k], (double)x.v[k][c], v);
            const float y = (float)v;
            const int64_t row = tall ? c0 + c : r, col = tall ? r : c0 + c;
            if (weights) {
                float* w = o.w + f.m.offset + row * f.m.cols + col;
                *w = fmaf(rate, y, *w * decay);
            } else {
                const int64_t at = f.index * o.out_batch_stride + row * o.out_stride + col;
                if (o.out_bf16) static_cast<u16*>(o.out)[at] = (u16)gemm::pack_bf16(y, 0.0f);
                else static_cast<float*>(o.out)[at] = y;
            }
        });
    }
}

// The learning rate in force, written by one lane, as that of the AGS step.
__global__ __launch_bounds__(64) void muon_rates_kernel(MuonRates* p, MuonRates r) {
    if (threadIdx.x == 0) *p = r;
}

// ------------------------------------------------------------- launches --

template <typename Kernel>
hipError_t launch_tiles(Kernel kernel, int t, int na, int nb, const MuonProductArgs& a, hipStream_t s) {
    const int lds = gemm::lds_bytes(t, t, na, nb);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.work.blocks), dim3(256), lds, s, a);
    return hipGetLastError();
}

}  // namespace

// Tiles of 128 squared: four buffers where all blocks fit the CUs at once even so; else two
// of each operand, and a third of b, which still leaves a CU two blocks, where every tile
// has stages enough to use it: X of eight 2048 x 512 23.6 -> 22.7 us, VGG-16's A A 182 -> 163;
// ResNet-50's X, most of whose tiles have one to four, would go from 75 to 77.
#define MUON_LAUNCH(KERNEL)                                                                       \
    (a.work.t == 4          ? launch_tiles(KERNEL<4, 2, 3>, 4, 2, 3, a, s)                        \
     : a.work.t == 1        ? launch_tiles(KERNEL<1, 4, 4>, 1, 4, 4, a, s)                        \
     : a.work.blocks <= 256 ? launch_tiles(KERNEL<2, 4, 4>, 2, 4, 4, a, s)                        \
     : a.work.stages >= 8   ? launch_tiles(KERNEL<2, 2, 3>, 2, 2, 3, a, s)                        \
                            : launch_tiles(KERNEL<2, 2, 2>, 2, 2, 2, a, s))

hipError_t launch_muon_sum(const MuonStepArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(muon_sum_kernel, dim3((unsigned)a.work.blocks), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_muon_start(const MuonStepArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(muon_start_kernel, dim3((unsigned)a.work.blocks), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_muon_thin(const MuonThinArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)a.in.work.blocks), block(kThreads);
    hipLaunchKernelGGL(muon_thin_gram_kernel, grid, block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.way == kThinEigen) {
        hipLaunchKernelGGL(muon_thin_eigen_kernel, grid, block, 0, s, a);
        e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    if (a.way == kThinSteps) hipLaunchKernelGGL(muon_thin_apply_kernel<kThinSteps>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(muon_thin_apply_kernel<kThinEigen>, grid, block, 0, s, a);
    return hipGetLastError();
}
hipError_t launch_muon_gram(const MuonProductArgs& a, hipStream_t s) { return MUON_LAUNCH(muon_gram_kernel); }
hipError_t launch_muon_square(const MuonProductArgs& a, hipStream_t s) { return MUON_LAUNCH(muon_square_kernel); }
hipError_t launch_muon_apply(const MuonProductArgs& a, hipStream_t s) { return MUON_LAUNCH(muon_apply_kernel); }
hipError_t launch_muon_rates(MuonRates* p, MuonRates r, hipStream_t s) {
    hipLaunchKernelGGL(muon_rates_kernel, dim3(1), dim3(64), 0, s, p, r);
    return hipGetLastError();
}

}  // namespace ags
