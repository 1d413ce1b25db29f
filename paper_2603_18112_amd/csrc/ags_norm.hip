// gfx950 kernels of the layer norm (include/ags_norm.h).
//
// norm_kernel           a wave or a block keeps a row in registers: read once,
//                       written once.
// norm_long_kernel      rows that do not fit: read three times, mostly from the
//                       caches.
// norm_backward_kernel  the same for dx; every lane also sums the weight's and the
//                       bias's gradients of its columns over the block's rows.
// norm_dx_long_kernel, norm_columns_kernel   the two separately, for long rows.
// norm_join_kernel      adds the blocks' sums.
//
// All are bound by memory: x (and dy) read once and y (dx) written once, with a few
// operations a byte.  Measured (us, bytes that have to move over the time): forward 8192 x
// 4096 bf16 25.5 (5.3 TB/s; a copy's rate is 4.7), 5001 x 1000 fp32 11.6 (3.5), one row of
// 4096 3.1; backward with both gradients 16384 x 8192 bf16 151 + 5 (5.2), 5001 x 1000 fp32
// 15.1 + 4.1 (3.1).  Small ones are bound by a launch and two or three waits for memory, long
// rows by their three reads: 2048 x 65536 bf16 forward 215 (2.5), backward 246 + 108 + 8 (2.2).
#include <type_traits>

#include "ags_mx_device.h"
#include "ags_norm_internal.h"

namespace ags {
namespace {

using mx::load8;
using mx::Unaligned;
typedef mx::v2f v2f;
typedef mx::v2bf v2bf;

__device__ __forceinline__ unsigned pack2(float x, float y) {
    const v2bf v = __builtin_convertvector((v2f{x, y}), v2bf);
    unsigned u;
    __builtin_memcpy(&u, &v, 4);
    return u;
}

// 8 elements to p, as many as lie in the row.
__device__ __forceinline__ void store8(unsigned short* p, int64_t left, const float* x) {
    Unaligned<unsigned, 4, 2> w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.v[i] = pack2(x[2 * i], x[2 * i + 1]);
    if (left >= 8) {
        *reinterpret_cast<Unaligned<unsigned, 4, 2>*>(p) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = (unsigned short)(w.v[i >> 1] >> (16 * (i & 1)));
}
__device__ __forceinline__ void store8(float* p, int64_t left, const float* x) {
    if (left >= 8) {
        Unaligned<float, 8, 4> w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.v[i] = x[i];
        *reinterpret_cast<Unaligned<float, 8, 4>*>(p) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = x[i];
}

// A tensor of either type, element `at` on.
__device__ __forceinline__ void load8_any(const void* p, bool bf16, int64_t at, int64_t left, float* x) {
    if (bf16) load8(static_cast<const unsigned short*>(p) + at, left, x);
    else load8(static_cast<const float*>(p) + at, left, x);
}
__device__ __forceinline__ void store8_any(void* p, bool bf16, int64_t at, int64_t left, const float* x) {
    if (bf16) store8(static_cast<unsigned short*>(p) + at, left, x);
    else store8(static_cast<float*>(p) + at, left, x);
}

// v plus what the lane that CTRL names holds, zero where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ float plus(float v) {
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, ROWS, 0xf, false));
}

// The sum over a wave, in every lane: within rows of 16 lanes by shifts of 1, 2, 4, 8,
// then the rows' last lanes to the next row and the next half.  (Six shuffles through
// LDS took a third of a row's time.)
__device__ __forceinline__ float wave_sum(float v) {
    v = plus<0x111, 0xf>(v);
    v = plus<0x112, 0xf>(v);
    v = plus<0x114, 0xf>(v);
    v = plus<0x118, 0xf>(v);
    v = plus<0x142, 0xa>(v);
    v = plus<0x143, 0xc>(v);
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// The same in fp64, by halves.
template <int CTRL, int ROWS>
__device__ __forceinline__ double plus(double v) {
    const int2 u = __builtin_bit_cast(int2, v);
    return v + __builtin_bit_cast(double, make_int2(__builtin_amdgcn_update_dpp(0, u.x, CTRL, ROWS, 0xf, false),
                                                    __builtin_amdgcn_update_dpp(0, u.y, CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ double wave_sum(double v) {
    v = plus<0x111, 0xf>(v);
    v = plus<0x112, 0xf>(v);
    v = plus<0x114, 0xf>(v);
    v = plus<0x118, 0xf>(v);
    v = plus<0x142, 0xa>(v);
    v = plus<0x143, 0xc>(v);
    const int2 u = __builtin_bit_cast(int2, v);
    return __builtin_bit_cast(double, make_int2(__builtin_amdgcn_readlane(u.x, 63), __builtin_amdgcn_readlane(u.y, 63)));
}

// Sums of N values over the G lanes of a row, in every lane.  Over a block they
// meet in LDS, in two slots (or arrays) in turn: one barrier a sum, since the next
// sum's barrier lies between two uses of a slot.
template <int G, typename S, int N>
__device__ __forceinline__ void row_sum(S (&v)[N], S (*red)[N][16], int slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (G > 64) {
        constexpr int kWaves = G / 64;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) red[slot][i][threadIdx.x >> 6] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            S s = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s += red[slot][i][w];
            v[i] = s;
        }
    }
}

// 16 bytes of a row: 8 or 4 elements, as they lie in memory, and as fp32.
template <typename T>
struct Piece {
    static constexpr int kN = 16 / sizeof(T);

    // What lies before the row's end (`left` elements); the rest zeros.
    static __device__ __forceinline__ uint4 load(const T* p, int64_t left) {
        if (left >= kN) {
            const auto w = *reinterpret_cast<const Unaligned<unsigned, 4, sizeof(T)>*>(p);
            return make_uint4(w.v[0], w.v[1], w.v[2], w.v[3]);
        }
        unsigned v[4] = {};
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (i < left) {
                if constexpr (kN == 8) v[i >> 1] |= (unsigned)p[i] << (16 * (i & 1));
                else v[i] = __float_as_uint(p[i]);
            }
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    static __device__ __forceinline__ void unpack(uint4 w, float* x) {
        const unsigned v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < kN; ++i)
            x[i] = __uint_as_float(kN == 4 ? v[i] : i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
    }
};

// N elements of a tensor of either type from element `at` on, as many as lie in it.
template <int N>
__device__ __forceinline__ void load_any(const void* p, bool bf16, int64_t at, int64_t left, float* x) {
    if constexpr (N == 8) {
        load8_any(p, bf16, at, left, x);
    } else if (bf16) {
        const unsigned short* q = static_cast<const unsigned short*>(p) + at;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < left ? __uint_as_float((unsigned)q[i] << 16) : 0.0f;
    } else {
        Piece<float>::unpack(Piece<float>::load(static_cast<const float*>(p) + at, left), x);
    }
}
template <int N>
__device__ __forceinline__ void store_any(void* p, bool bf16, int64_t at, int64_t left, const float* x) {
    if constexpr (N == 8) {
        store8_any(p, bf16, at, left, x);
    } else if (bf16) {
        unsigned short* q = static_cast<unsigned short*>(p) + at;
        const unsigned v[2] = {pack2(x[0], x[1]), pack2(x[2], x[3])};
        if (left >= 4) {
            Unaligned<unsigned, 2, 2> w;
            w.v[0] = v[0], w.v[1] = v[1];
            *reinterpret_cast<Unaligned<unsigned, 2, 2>*>(q) = w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) q[i] = (unsigned short)(v[i >> 1] >> (16 * (i & 1)));
    } else {
        float* q = static_cast<float*>(p) + at;
        if (left >= 4) {
            Unaligned<float, 4, 4> w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w.v[i] = x[i];
            *reinterpret_cast<Unaligned<float, 4, 4>*>(q) = w;
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) q[i] = x[i];
    }
}

// ---------------------------------------------------------------- forward --

// The mean as two fp32 numbers (hi alone would put its rounding into every difference and,
// squared, into the variance: a constant fp32 row of 10000.1 had z = -0.3).  The sum
// of a row is exact where its elements are near one another, and its rounding small beside
// the spread where they are not: fp32 is added in fp64; bf16, of 8 bits, in fp32, times
// 2^-16, which keeps the largest of 2^16 columns in range and denormals whole.  A
// constant row's hi is its value, and all differences are zeros.
//
// Differences from fp32 take hi away first, exact for an element near the mean, then lo.
// Those from bf16 leave lo out: it is no more than 2^-25 of the mean, elements of one row are
// equal or 2^-8 apart, so z takes it in one operation and the variance as its square (8192 x
// 4096 bf16 in a graph 24.9 us; with lo in each difference 25.3, with sums in fp64 too 26.0;
// since the variance is a product, not a quotient, 24.3).
constexpr float kSumScale = 0x1p-16f;

struct Mean {
    float hi, lo;

    __device__ __forceinline__ Mean(double sum, int64_t cols, double inv)
        : hi((float)(sum * inv)), lo((float)(fma(-(double)hi, (double)cols, sum) * inv)) {}
    __device__ __forceinline__ Mean(float sum, int64_t cols, double inv) {
        const float m = sum / (float)cols;
        hi = m * (1.0f / kSumScale);
        lo = fmaf(-m, (float)cols, sum) * (float)inv * (1.0f / kSumScale);
    }
    __device__ __forceinline__ float off(float x) const { return (x - hi) - lo; }
};
// Squares whose sum is not between 2^-90 and fp32's largest number (one comparison of the bits of a
// sum that is not negative).  The power of two that brings such a row's differences into
// fp32's range; NaN stays.
__device__ __forceinline__ bool row_unusual(float squares) {
    return __float_as_uint(squares) - 0x12800000u > 0x7f7fffffu - 0x12800000u;
}
__device__ __forceinline__ float row_scale(float squares, float eps) {
    if (!(squares < 0x1p-90f)) return 0x1p-96f;
    return eps < 0x1p-90f ? 0x1p90f : 1.0f;
}

template <typename T>
using RowSum = typename std::conditional<sizeof(T) == 2, float, double>::type;

template <int N>
__device__ __forceinline__ void add_to(double& sum, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum += (double)x[i];
}
template <int N>
__device__ __forceinline__ void add_to(float& sum, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum = fmaf(x[i], kSumScale, sum);
}

// G lanes to a row, NV pieces of 16 bytes each; a block of B threads has B / G
// rows at a time, and asks for the next ones while it reduces these.  KEEP: weight and
// bias stay in registers, for all the block's rows.  T: x's type.
template <typename T, int G, int NV, int B, bool KEEP>
__global__ __launch_bounds__(B) void norm_kernel(NormArgs a) {
    constexpr int N = Piece<T>::kN;
    constexpr bool kLater = sizeof(T) == 2;  // what the mean's lo is taken into
    __shared__ RowSum<T> red_sum[1][1][16];
    __shared__ float red[2][1][16];
    const int lane = threadIdx.x % G;
    const int64_t cols = a.cols, step = (int64_t)gridDim.x * (B / G);
    int64_t row = (int64_t)blockIdx.x * (B / G) + threadIdx.x / G;
    uint4 raw[NV];
    auto fetch = [&](int64_t r) {
        const T* p = static_cast<const T*>(a.x) + r * a.x_stride;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
            raw[j] = Piece<T>::load(p + c, r < a.rows ? cols - c : 0);
        }
    };
    fetch(row);
    auto affine = [&](int j, float (&w)[N], float (&b)[N]) {
        const int64_t c = ((int64_t)j * G + lane) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = 1.0f, b[i] = 0.0f;
        if (c < cols) {
            if (a.weight) load_any<N>(a.weight, a.w_bf16, c, cols - c, w);
            if (a.bias) load_any<N>(a.bias, a.w_bf16, c, cols - c, b);
        }
    };
    float w[KEEP ? NV : 1][N], b[KEEP ? NV : 1][N];
    if constexpr (KEEP) {
#pragma unroll
        for (int j = 0; j < NV; ++j) affine(j, w[j], b[j]);
    }
    for (; row < a.rows; row += step) {
        float x[NV][N], s[1] = {0.0f};
        RowSum<T> sum[1] = {0};
#pragma unroll
        for (int j = 0; j < NV; ++j) Piece<T>::unpack(raw[j], x[j]);
        if (row + step < a.rows) fetch(row + step);
#pragma unroll
        for (int j = 0; j < NV; ++j) add_to(sum[0], x[j]);
        row_sum<G>(sum, red_sum, 0);
        const Mean mean(sum[0], cols, a.inv_cols);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[j][i] = kLater ? x[j][i] - mean.hi : mean.off(x[j][i]);
                if (c + i < cols) s[0] = fmaf(x[j][i], x[j][i], s[0]);
            }
        }
        row_sum<G>(s, red, 0);
        auto reciprocal = [&](float squares, float scale) {
            float var = squares * (float)a.inv_cols;
            if constexpr (kLater) {
                const float lo = mean.lo * scale;
                var = fmaf(-lo, lo, var);
                var = var < 0.0f ? 0.0f : var;  // (NaN stays)
            }
            return scale / sqrtf(var + a.eps * scale * scale);
        };
        float rstd = reciprocal(s[0], 1.0f);
        const float scale = row_unusual(s[0]) ? row_scale(s[0], a.eps) : 1.0f;
        if (scale != 1.0f) {  // (all the row's lanes, or none)
            s[0] = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int64_t c = ((int64_t)j * G + lane) * N;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float d = x[j][i] * scale;
                    if (c + i < cols) s[0] = fmaf(d, d, s[0]);
                }
            }
            row_sum<G>(s, red, 1);
            rstd = reciprocal(s[0], scale);
        }
        const float shift = -mean.lo * rstd;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
            if (c >= cols) continue;
            const int k = KEEP ? j : 0;
            if constexpr (!KEEP) affine(j, w[0], b[0]);
#pragma unroll
            for (int i = 0; i < N; ++i)
                x[j][i] = fmaf(kLater ? fmaf(x[j][i], rstd, shift) : x[j][i] * rstd, w[k][i], b[k][i]);
            store_any<N>(a.y, a.y_bf16, row * a.y_stride + c, cols - c, x[j]);
        }
        if (a.saved && lane == 0) {
            a.saved[row] = mean.hi;
            a.saved[a.rows + row] = rstd;
        }
    }
}

constexpr int kLong = 1024;  // threads to a long row

template <typename T>
__global__ __launch_bounds__(kLong) void norm_long_kernel(NormArgs a) {
    __shared__ double red_sum[1][1][16];
    __shared__ float red[2][1][16];
    const int64_t cols = a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* p = static_cast<const T*>(a.x) + row * a.x_stride;
        float s[1] = {0.0f}, x[8];
        double sum[1] = {0.0};
        for (int64_t c = threadIdx.x * 8; c < cols; c += kLong * 8) {
            load8(p + c, cols - c, x);
            if constexpr (sizeof(T) == 2) {
                float part = 0.0f;
                add_to(part, x);
                sum[0] += (double)part * (1.0 / kSumScale);
            } else {
                add_to(sum[0], x);
            }
        }
        row_sum<kLong>(sum, red_sum, 0);
        const Mean mean(sum[0], cols, a.inv_cols);
        float scale = 1.0f;
        for (int pass = 0; pass < 2; ++pass) {  // (a second one where row_scale asks for it)
            s[0] = 0.0f;
            for (int64_t c = threadIdx.x * 8; c < cols; c += kLong * 8) {
                load8(p + c, cols - c, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = mean.off(x[i]) * scale;
                    if (c + i < cols) s[0] = fmaf(d, d, s[0]);
                }
            }
            row_sum<kLong>(s, red, pass);
            if (pass || !row_unusual(s[0])) break;
            scale = row_scale(s[0], a.eps);
            if (scale == 1.0f) break;
        }
        const float rstd = scale / sqrtf(s[0] / (float)cols + a.eps * scale * scale);
        for (int64_t c = threadIdx.x * 8; c < cols; c += kLong * 8) {
            float w[8] = {1, 1, 1, 1, 1, 1, 1, 1}, b[8] = {};
            if (a.weight) load8_any(a.weight, a.w_bf16, c, cols - c, w);
            if (a.bias) load8_any(a.bias, a.w_bf16, c, cols - c, b);
            load8(p + c, cols - c, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = fmaf(mean.off(x[i]) * rstd, w[i], b[i]);
            store8_any(a.y, a.y_bf16, row * a.y_stride + c, cols - c, x);
        }
        if (a.saved && threadIdx.x == 0) {
            a.saved[row] = mean.hi;
            a.saved[a.rows + row] = rstd;
        }
    }
}

// --------------------------------------------------------------- backward --

// As norm_kernel; DW: the sums over the block's rows are wanted too.  A part is
// a block's rows.
template <typename T, int G, int NV, int B, bool DW>
__global__ __launch_bounds__(B) void norm_backward_kernel(NormBackwardArgs a) {
    constexpr int N = Piece<T>::kN;
    // 1024 threads have 128 registers each: no row ahead, the weight read anew
    constexpr bool kRoom = B < 1024 || !DW;
    __shared__ float red[2][2][16];
    const int lane = threadIdx.x % G;
    const int64_t cols = a.cols, step = (int64_t)gridDim.x * (B / G);
    int64_t row = (int64_t)blockIdx.x * (B / G) + threadIdx.x / G;
    uint4 raw_x[NV], raw_d[NV];
    float mean = 0.0f, rstd = 0.0f;
    auto fetch = [&](int64_t r) {
        const T *px = static_cast<const T*>(a.x) + r * a.x_stride, *pd = static_cast<const T*>(a.dy) + r * a.dy_stride;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
            raw_x[j] = Piece<T>::load(px + c, cols - c);
            raw_d[j] = Piece<T>::load(pd + c, cols - c);
        }
        mean = a.saved[r];
        rstd = a.saved[a.rows + r];
    };
    if (kRoom && row < a.rows) fetch(row);
    auto weight = [&](int j, float (&w)[N]) {
        const int64_t c = ((int64_t)j * G + lane) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = 1.0f;
        if (c < cols && a.weight) load_any<N>(a.weight, a.w_bf16, c, cols - c, w);
    };
    float w[kRoom ? NV : 1][N], dw[NV][N], db[NV][N];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < N; ++i) dw[j][i] = 0.0f, db[j][i] = 0.0f;
        if constexpr (kRoom) weight(j, w[j]);
    }
    int slot = 0;
    for (; row < a.rows; row += step, slot ^= 1) {
        if constexpr (!kRoom) fetch(row);
        float z[NV][N], g[NV][N], s[2] = {0.0f, 0.0f};
        const float mu = mean, rs = rstd;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            Piece<T>::unpack(raw_x[j], z[j]);
            Piece<T>::unpack(raw_d[j], g[j]);
        }
        if (kRoom && row + step < a.rows) fetch(row + step);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int k = kRoom ? j : 0;
            if constexpr (!kRoom) weight(j, w[0]);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                z[j][i] = (z[j][i] - mu) * rs;
                if constexpr (DW) {
                    dw[j][i] = fmaf(g[j][i], z[j][i], dw[j][i]);
                    db[j][i] += g[j][i];
                }
                g[j][i] *= w[k][i];
                s[0] += g[j][i];
                s[1] = fmaf(g[j][i], z[j][i], s[1]);  // (past the row's end g is zero)
            }
        }
        if (!a.dx) continue;
        row_sum<G>(s, red, slot);
        const float m0 = s[0] / (float)cols, m1 = s[1] / (float)cols;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = ((int64_t)j * G + lane) * N;
            if (c >= cols) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) z[j][i] = rs * (g[j][i] - m0 - z[j][i] * m1);
            store_any<N>(a.dx, a.bf16, row * a.dx_stride + c, cols - c, z[j]);
        }
    }
    if constexpr (DW) {
        float* out = a.partials + (int64_t)blockIdx.x * 2 * cols;
        if constexpr (G == B) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int64_t c = ((int64_t)j * G + lane) * N;
                if (c >= cols) continue;
                store_any<N>(out, false, c, cols - c, dw[j]);
                store_any<N>(out, false, cols + c, cols - c, db[j]);
            }
        } else {
            // the block's waves, each with rows of its own, one after the other
            __shared__ float sum[2][G * NV * N];
            for (int k = 0; k < B / G; ++k) {
                if ((int)threadIdx.x / G == k) {
#pragma unroll
                    for (int j = 0; j < NV; ++j)
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const int at = (j * N + i) * G + lane;
                            sum[0][at] = k ? sum[0][at] + dw[j][i] : dw[j][i];
                            sum[1][at] = k ? sum[1][at] + db[j][i] : db[j][i];
                        }
                }
                __syncthreads();
            }
            for (int t = threadIdx.x; t < 2 * G * NV; t += B) {
                const int which = t / (G * NV), j = t / G % NV, l = t % G;
                const int64_t c = ((int64_t)j * G + l) * N;
                if (c >= cols) continue;
                float v[N];
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = sum[which][(j * N + i) * G + l];
                store_any<N>(out, false, which * cols + c, cols - c, v);
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kLong) void norm_dx_long_kernel(NormBackwardArgs a) {
    __shared__ float red[2][2][16];
    const int64_t cols = a.cols;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, slot ^= 1) {
        const T *px = static_cast<const T*>(a.x) + row * a.x_stride, *pd = static_cast<const T*>(a.dy) + row * a.dy_stride;
        const float mean = a.saved[row], rstd = a.saved[a.rows + row];
        float s[2] = {0.0f, 0.0f};
        for (int pass = 0; pass < 2; ++pass) {
            const float m0 = s[0] / (float)cols, m1 = s[1] / (float)cols;
            for (int64_t c = threadIdx.x * 8; c < cols; c += kLong * 8) {
                float z[8], g[8], w[8] = {1, 1, 1, 1, 1, 1, 1, 1};
                load8(px + c, cols - c, z);
                load8(pd + c, cols - c, g);
                if (a.weight) load8_any(a.weight, a.w_bf16, c, cols - c, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    z[i] = (z[i] - mean) * rstd;
                    g[i] *= w[i];
                    if (pass == 0) {
                        s[0] += g[i];
                        s[1] = fmaf(g[i], z[i], s[1]);
                    } else {
                        z[i] = rstd * (g[i] - m0 - z[i] * m1);
                    }
                }
                if (pass == 1) store8(static_cast<T*>(a.dx) + row * a.dx_stride + c, cols - c, z);
            }
            if (pass == 0) row_sum<kLong>(s, red, slot);
        }
    }
}

// A block takes 512 columns of a part's rows, each wave every fourth row.
template <typename T>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormBackwardArgs a) {
    __shared__ float sum[2][4][512];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t cols = a.cols, c = ((int64_t)blockIdx.x * 64 + lane) * 8;
    const int64_t r0 = a.rows * blockIdx.y / a.parts, r1 = a.rows * (blockIdx.y + 1) / a.parts;
    float dw[8] = {}, db[8] = {};
    if (c < cols) {
        for (int64_t row = r0 + wave; row < r1; row += 4) {
            float z[8], g[8];
            load8(static_cast<const T*>(a.x) + row * a.x_stride + c, cols - c, z);
            load8(static_cast<const T*>(a.dy) + row * a.dy_stride + c, cols - c, g);
            const float mean = a.saved[row], rstd = a.saved[a.rows + row];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[i] = fmaf(g[i], (z[i] - mean) * rstd, dw[i]);
                db[i] += g[i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        sum[0][wave][i * 64 + lane] = dw[i];
        sum[1][wave][i * 64 + lane] = db[i];
    }
    __syncthreads();
    if (wave >= 2 || c >= cols) return;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = i * 64 + lane;
        v[i] = sum[wave][0][at] + sum[wave][1][at] + (sum[wave][2][at] + sum[wave][3][at]);
    }
    store8(a.partials + ((int64_t)blockIdx.y * 2 + wave) * cols + c, cols - c, v);
}

// 64 columns of one of the two gradients to a block; its waves share the parts.
constexpr int kJoinWaves = 16;

__global__ __launch_bounds__(kJoinWaves * 64) void norm_join_kernel(NormBackwardArgs a) {
    __shared__ float sum[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles = (a.cols + 63) / 64, cols = a.cols;
    const int which = blockIdx.x >= tiles;
    void* out = which ? a.dbias : a.dweight;
    if (!out) return;
    const int64_t c = (blockIdx.x - which * tiles) * 64 + lane;
    float v = 0.0f;
    if (c < cols) {
        const float* p = a.partials + which * cols + c;
#pragma unroll 16
        for (int k = wave; k < a.parts; k += kJoinWaves) v += p[(int64_t)k * 2 * cols];
    }
    sum[wave][lane] = v;
    __syncthreads();
    if (wave || c >= cols) return;
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < kJoinWaves; ++k) v += sum[k][lane];
    if (a.dw_bf16) {
        unsigned short* o = static_cast<unsigned short*>(out) + c;
        if (a.accumulate) v += __uint_as_float((unsigned)*o << 16);
        *o = (unsigned short)pack2(v, 0.0f);
    } else {
        float* o = static_cast<float*>(out) + c;
        *o = a.accumulate ? v + *o : v;
    }
}

// Blocks that the card holds at once are enough: they go through the rows.
unsigned norm_blocks(int64_t rows, int64_t at_once, int64_t most) {
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>((rows + at_once - 1) / at_once, most));
}

// NV below is in pieces of bf16; rows of fp32 have twice as many.  More lanes to a row
// have fewer registers each and more rows in all under way: 8192 x 4096 bf16 with 512, 256
// and 128 lanes 27.4, 32 and 39 us (4.9 TB/s; a copy 4.7); for 16384 x 8192 with 1024,
// 512 and 256 lanes 117, 112 and 112.
template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t s) {
    const int64_t n = a.cols;
    constexpr int F = sizeof(T) / 2;
#define NORM_FORWARD(G, NV, B, MOST, KEEP)                                                                 \
    hipLaunchKernelGGL((norm_kernel<T, G, NV * F, B, KEEP>), dim3(norm_blocks(a.rows, B / G, MOST)), dim3(B), 0, s, a)
    // one row to a wave: more waves are worth more than weights in registers (5001 x
    // 1000 fp32 11.5 us against 15.2; 16384 x 1024 bf16 19.5 and 16.2)
    if (n <= 512) NORM_FORWARD(64, 1, 256, 2048, true);
    else if (n <= 1024 && a.rows <= 6144) NORM_FORWARD(64, 2, 256, 1536, false);
    else if (n <= 1024) NORM_FORWARD(64, 2, 256, 1536, true);
    else if (n <= 2048) NORM_FORWARD(256, 1, 256, 2048, true);
    else if (n <= 4096) NORM_FORWARD(512, 1, 512, 1024, true);
    else if (n <= 8192) NORM_FORWARD(512, 2, 512, 768, true);
    else if (n <= 16384) NORM_FORWARD(1024, 2, 1024, 512, true);
    else if (F == 1 && n <= kNormForwardCols) NORM_FORWARD(1024, 4 / F, 1024, 256, false);
    else
        hipLaunchKernelGGL((norm_long_kernel<T>), dim3(norm_blocks(a.rows, 1, 512)), dim3(kLong), 0, s, a);
#undef NORM_FORWARD
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const NormBackwardArgs& a, hipStream_t s) {
    const int64_t n = a.cols;
    const bool dw = a.dweight || a.dbias;
    constexpr int F = sizeof(T) / 2;
#define NORM_BACKWARD(G, NV, B)                                                                                       \
    do {                                                                                                              \
        if (dw) hipLaunchKernelGGL((norm_backward_kernel<T, G, NV * F, B, true>), dim3(a.parts), dim3(B), 0, s, a);   \
        else hipLaunchKernelGGL((norm_backward_kernel<T, G, NV * F, B, false>),                                       \
                                dim3(norm_blocks(a.rows, B / G, 1024)), dim3(B), 0, s, a);                            \
    } while (0)
    if (a.rows == 0) {}  // empty sums
    else if (n <= 512) NORM_BACKWARD(64, 1, 512);
    else if (n <= 1024) NORM_BACKWARD(64, 2, 256);
    else if (n <= 2048) NORM_BACKWARD(256, 1, 256);
    else if (n <= 4096) NORM_BACKWARD(256, 2, 256);
    else if (n <= 8192) NORM_BACKWARD(512, 2, 512);
    else if (n <= kNormBackwardCols) NORM_BACKWARD(1024, 2, 1024);
    else {
        if (a.dx)
            hipLaunchKernelGGL((norm_dx_long_kernel<T>), dim3(norm_blocks(a.rows, 1, 512)), dim3(kLong), 0, s, a);
        if (dw)
            hipLaunchKernelGGL((norm_columns_kernel<T>), dim3((unsigned)((n + 511) / 512), a.parts), dim3(256), 0, s, a);
    }
#undef NORM_BACKWARD
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !dw) return e;
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(2 * ((n + 63) / 64))), dim3(kJoinWaves * 64), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
    return a.bf16 ? forward<unsigned short>(a, s) : forward<float>(a, s);
}

hipError_t launch_norm_backward(const NormBackwardArgs& a, hipStream_t s) {
    return a.bf16 ? backward<unsigned short>(a, s) : backward<float>(a, s);
}

}  // namespace ags
