// gfx950 kernels of the gated products (include/ags_glu.h).
//
// glu_store_kernel, glu_pack_kernel   operands laid out for the products
// glu_product_kernel   both products of a tile; the activation and its product with
//                      the other (or their gradients) as the sums are stored
// glu_few_kernel       few rows of x: every weight read once, straight into registers
// glu_act_kernel       dg and du from what the forward pass saved
// glu_dx_kernel, glu_dw_kernel   the products of the backward pass
// glu_join_kernel, glu_join_plain_kernel   sum the parts of a contracted axis
#include <type_traits>

#include "ags_gemm_device.h"
#include "ags_glu_internal.h"

namespace ags {
namespace {

using gemm::bf16_value;
using gemm::pack_bf16;
using gemm::Side;
using gemm::store8;
using mx::load8;
using mx::Unaligned;
typedef unsigned short u16;

// ----------------------------------------------------------------- layout --

// A thread takes 8 elements of a row of the laid-out weight.
__global__ __launch_bounds__(256) void glu_store_kernel(GluStoreArgs a) {
    const int64_t padded = glu_padded(a.k), pieces = padded / 8, total = glu_lines(a.n) * pieces;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t line = t / pieces, c = (t - line * pieces) * 8, row = line / 32 * 16 + line % 16;
        const bool up = line & 16;
        float x[8] = {};
        if (row < a.n && c < a.k) {
            const int64_t at = row * (up ? a.up_stride : a.gate_stride) + c;
            const void* p = up ? a.up : a.gate;
            if (a.bf16) load8(static_cast<const u16*>(p) + at, a.k - c, x);
            else load8(static_cast<const float*>(p) + at, a.k - c, x);
        }
        store8(static_cast<u16*>(a.data) + line * padded + c, 8, x);
    }
}

__global__ __launch_bounds__(256) void glu_pack_kernel(GluPackArgs a) {
    const int64_t pieces = a.padded / 8, total = a.rows * pieces;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t row = t / pieces, c = (t - row * pieces) * 8;
        float x[8];
        load8(static_cast<const u16*>(a.x) + row * a.stride + c, a.k - c, x);
        store8(static_cast<u16*>(a.out) + row * a.padded + c, 8, x);
    }
}

// ------------------------------------------------------------- activation --

// act(g), and its derivative.
__device__ __forceinline__ float act_of(int act, float g) {
    if (act == AGS_GLU_SILU) return g / (1.0f + expf(-g));
    return 0.5f * g * (1.0f + erff(g * 0.70710678f));
}
__device__ __forceinline__ void act_both(int act, float g, float* f, float* d) {
    if (act == AGS_GLU_SILU) {
        const float s = 1.0f / (1.0f + expf(-g));
        *f = g * s;
        *d = s * fmaf(g, 1.0f - s, 1.0f);
    } else {
        const float c = 0.5f * (1.0f + erff(g * 0.70710678f));
        *f = g * c;
        *d = fmaf(g * 0.39894228f, expf(-0.5f * g * g), c);
    }
}

// Eight sums of gate and the same eight of up, hidden units from `unit` on.
__device__ __forceinline__ void put_pair(const GluArgs& a, int64_t row, int64_t unit, float* g, float* u) {
    const int64_t line = unit / 16 * 32 + unit % 16, left = a.n - unit;
    if (a.mode == kGluForward) {
        if (a.saved) {
            u16* s = static_cast<u16*>(a.saved) + row * glu_lines(a.n) + line;
            store8(s, 8, g);
            store8(s + 16, 8, u);
        }
        if (left <= 0) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = act_of(a.act, g[i]) * u[i];
        const int64_t at = row * a.h_stride + unit;
        if (a.h_bf16) store8(static_cast<u16*>(a.h) + at, left, g);
        else store8(static_cast<float*>(a.h) + at, left, g);
    } else {
        float dh[8];
        load8(static_cast<const u16*>(a.dh) + row * a.dh_stride + unit, left, dh);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f, d;
            act_both(a.act, g[i], &f, &d);
            // (a padding unit has g = u = dh = 0)
            g[i] = dh[i] * u[i] * d;
            u[i] = dh[i] * f;
        }
        u16* p = static_cast<u16*>(a.grads) + row * glu_grads(a.n) + line;
        store8(p, 8, g);
        store8(p + 16, 8, u);
        const int64_t lines = glu_lines(a.n);
        if (line / 32 * 32 + 32 == lines && lines < glu_grads(a.n)) {
            const float zero[8] = {};
            store8(p + 32, 8, zero);
            store8(p + 48, 8, zero);
        }
    }
}

// What a product tile's sums become.  (Not unrolled: four copies of these loops stand in
// the tile of 256 squared.)
struct PairOut {
    const GluArgs& a;

    template <int WIDE>
    __device__ __forceinline__ void strip(const char* sm, int pitch, int lane, int64_t row0, int64_t col0, int64_t rows,
                                          int64_t cols) const {
        constexpr int kLanes = WIDE / 16, kRows = 64 / kLanes;
        const int q = lane % kLanes, c = q / 2 * 32 + (q & 1) * 8;
        if (c >= cols) return;
        const int end = (int)min(rows, (int64_t)32);
#pragma unroll 1
        for (int t = lane / kLanes; t < end; t += kRows) {
            float g[8], u[8];
            gemm::read8(sm + t * pitch + c * 4, g);
            gemm::read8(sm + t * pitch + c * 4 + 64, u);
            put_pair(a, row0 + t, (col0 + c) / 32 * 16 + c % 16, g, u);
        }
    }
};

// One part's sums where there is one, to rows of n.
template <typename Out>
struct OrPart {
    const Out& out;
    float* p;
    int64_t n;

    template <int WIDE>
    __device__ __forceinline__ void strip(const char* sm, int pitch, int lane, int64_t row0, int64_t col0, int64_t rows,
                                          int64_t cols) const {
        if (!p) {
            out.template strip<WIDE>(sm, pitch, lane, row0, col0, rows, cols);
            return;
        }
        constexpr int kLanes = WIDE / 8, kRows = 64 / kLanes;
        const int c = lane % kLanes * 8;
        if (c >= cols) return;
        const int end = (int)min(rows, (int64_t)32);
#pragma unroll 2
        for (int t = lane / kLanes; t < end; t += kRows) {
            float x[8];
            gemm::read8(sm + t * pitch + c * 4, x);
            store8(p + (row0 + t) * n + col0 + c, cols - c, x);
        }
    }
};

// Eight results of a row from column c on: added to what is there, or not.
__device__ __forceinline__ void put_row(const GluBackArgs& a, bool dw, int64_t row, int64_t c, float* x) {
    void* p = a.out;
    if (dw) {
        if (row & 16) p = a.out_up;
        row = row / 32 * 16 + row % 16;
        if (row >= a.n) return;
    }
    const int64_t at = row * a.stride + c, left = a.k - c;
    if (a.accumulate) {
        float y[8];
        if (a.bf16) load8(static_cast<const u16*>(p) + at, left, y);
        else load8(static_cast<const float*>(p) + at, left, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += y[i];
    }
    if (a.bf16) store8(static_cast<u16*>(p) + at, left, x);
    else store8(static_cast<float*>(p) + at, left, x);
}

struct RowOut {
    const GluBackArgs& a;
    bool dw;

    template <int WIDE>
    __device__ __forceinline__ void strip(const char* sm, int pitch, int lane, int64_t row0, int64_t col0, int64_t rows,
                                          int64_t cols) const {
        constexpr int kLanes = WIDE / 8, kRows = 64 / kLanes;
        const int c = lane % kLanes * 8;
        if (c >= cols) return;
        const int end = (int)min(rows, (int64_t)32);
#pragma unroll 2
        for (int t = lane / kLanes; t < end; t += kRows) {
            float x[8];
            gemm::read8(sm + t * pitch + c * 4, x);
            put_row(a, dw, row0 + t, col0 + c, x);
        }
    }
};

// --------------------------------------------------------------- products --

constexpr unsigned kBand = 6;

template <int T, int NB, bool ALONG_A, bool ALONG_B, typename Out>
__device__ __forceinline__ void product(const Side& a, const Side& b, int64_t m, int64_t n, int64_t k, int splits,
                                        float* partials, unsigned tm, unsigned tn, const Out& out) {
    extern __shared__ __attribute__((aligned(16))) char sm[];
    const unsigned tiles = tm * tn, split = blockIdx.x / tiles;
    unsigned ti, tj;
    tile::tile_of_block<kBand>(blockIdx.x % tiles, tm, tn, ti, tj);
    const int64_t i0 = (int64_t)ti * 64 * T, j0 = (int64_t)tj * 64 * T;
    const int stages = (int)((k + gemm::kDepth - 1) / gemm::kDepth);
    const int s0 = (int)((int64_t)stages * split / splits), s1 = (int)((int64_t)stages * (split + 1) / splits);
    float* part = splits > 1 ? partials + (int64_t)split * m * n : nullptr;
    gemm::product_tile<gemm::Bf16, T, T, NB, ALONG_A, ALONG_B>(a, b, s0, s1, i0, j0, m, n, sm, OrPart<Out>{out, part, n});
}

template <int T, int NB>
__global__ __launch_bounds__(256, 1) void glu_product_kernel(GluArgs a, unsigned tm, unsigned tn) {
    const int64_t lines = glu_lines(a.n), padded = glu_padded(a.k);
    product<T, NB, false, false>(Side{a.x, a.x_stride * 2, a.rows, 0}, Side{a.w, padded * 2, lines, 0}, a.rows, lines,
                                 padded, a.splits, a.partials, tm, tn, PairOut{a});
}

template <int T, int NB>
__global__ __launch_bounds__(256, 1) void glu_dx_kernel(GluBackArgs a, unsigned tm, unsigned tn) {
    const int64_t lines = glu_lines(a.n), padded = glu_padded(a.k), grads = glu_grads(a.n);
    product<T, NB, false, true>(Side{a.grads, grads * 2, a.rows, 0}, Side{a.w, padded * 2, lines, padded}, a.rows, a.k,
                                grads, a.splits, a.partials, tm, tn, RowOut{a, false});
}

template <int T, int NB>
__global__ __launch_bounds__(256, 1) void glu_dw_kernel(GluBackArgs a, unsigned tm, unsigned tn) {
    const int64_t lines = glu_lines(a.n), grads = glu_grads(a.n);
    product<T, NB, true, true>(Side{a.grads, grads * 2, a.rows, grads}, Side{a.x, a.x_stride * 2, a.rows, a.x_width},
                               lines, a.k, a.rows, a.splits, a.partials, tm, tn, RowOut{a, true});
}

// Sums of parts: a thread takes eight units (or columns) of a row, and has the
// loads of four parts under way.
__device__ __forceinline__ void join8(const float* p, int64_t part, int splits, int64_t left, float* x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.0f;
    for (int s = 0; s < splits; s += 4) {
        float y[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) load8(p + min(s + u, splits - 1) * part, left, y[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] += s + u < splits ? y[u][i] : 0.0f;
    }
}

__global__ __launch_bounds__(256) void glu_join_kernel(GluArgs a) {
    const int64_t lines = glu_lines(a.n), pieces = lines / 16, total = a.rows * pieces, part = a.rows * lines;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t row = t / pieces, unit = (t - row * pieces) * 8;
        const float* p = a.partials + row * lines + unit / 16 * 32 + unit % 16;
        float g[8], u[8];
        join8(p, part, a.splits, 8, g);
        join8(p + 16, part, a.splits, 8, u);
        put_pair(a, row, unit, g, u);
    }
}

__global__ __launch_bounds__(256) void glu_join_plain_kernel(GluBackArgs a, int64_t m, int32_t dw) {
    const int64_t pieces = (a.k + 7) / 8, total = m * pieces, part = m * a.k;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t row = t / pieces, c = (t - row * pieces) * 8;
        float x[8];
        join8(a.partials + row * a.k + c, part, a.splits, a.k - c, x);
        put_row(a, dw, row, c, x);
    }
}

__global__ __launch_bounds__(256) void glu_act_kernel(GluActArgs a) {
    const int64_t lines = glu_lines(a.n), pieces = lines / 16, total = a.rows * pieces;
    GluArgs g{};
    g.n = a.n;
    g.act = a.act;
    g.mode = kGluGrads;
    g.dh = a.dh;
    g.dh_stride = a.dh_stride;
    g.grads = a.grads;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t row = t / pieces, unit = (t - row * pieces) * 8;
        const u16* p = static_cast<const u16*>(a.saved) + row * lines + unit / 16 * 32 + unit % 16;
        float x[8], u[8];
        load8(p, 8, x);
        load8(p + 16, 8, u);
        put_pair(g, row, unit, x, u);
    }
}

// --------------------------------------------------------------- few rows --

// Up to 16 MT rows of x against all of w: every weight is read once, straight
// into registers, so the kernel is bound by the weights' bytes.  A block takes 32
// lines of w, 16 units of gate and of up; its waves share the contracted axis,
// 32 elements (64 bytes of a line) at a time, and their sums meet in LDS, in a
// fixed order.
constexpr int kFewWaves = 8;

template <int MT>
__global__ __launch_bounds__(kFewWaves * 64) void glu_few_kernel(GluArgs a) {
    __shared__ float red[kFewWaves][2][MT][4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int64_t padded = glu_padded(a.k), line = (int64_t)blockIdx.x * 32;
    const u16* pw = static_cast<const u16*>(a.w) + (line + r) * padded + q * 8;
    const u16* px[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
        px[t] = static_cast<const u16*>(a.x) + min((int64_t)(t * 16 + r), a.rows - 1) * a.x_stride + q * 8;
    gemm::v4f acc[2][MT];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[s][t] = gemm::v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t chunks = padded / 32;
    for (int64_t c = w; c < chunks; c += kFewWaves) {
        const uint4 g = *reinterpret_cast<const uint4*>(pw + c * 32);
        const uint4 u = *reinterpret_cast<const uint4*>(pw + 16 * padded + c * 32);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const uint4 x = *reinterpret_cast<const uint4*>(px[t] + c * 32);
            acc[0][t] = gemm::Bf16::mfma16(g, x, acc[0][t]);
            acc[1][t] = gemm::Bf16::mfma16(u, x, acc[1][t]);
        }
    }
    // Lane l holds row l % 16 of x, and of the 16 units the four from 4 (l / 16).
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[w][s][t][i][lane] = acc[s][t][i];
    __syncthreads();
    for (int e = threadIdx.x; e < MT * 32; e += kFewWaves * 64) {
        const int t = e >> 5, row = e >> 1 & 15, half = e & 1;
        if (t * 16 + row >= a.rows) continue;
        float g[8], u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int l = (half * 2 + i / 4) * 16 + row;
            g[i] = u[i] = 0.0f;
#pragma unroll
            for (int v = 0; v < kFewWaves; ++v) {
                g[i] += red[v][0][t][i % 4][l];
                u[i] += red[v][1][t][i % 4][l];
            }
        }
        put_pair(a, t * 16 + row, line / 2 + half * 8, g, u);
    }
}

// --------------------------------------------------------------- launches --

unsigned blocks_for(int64_t items) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 8192)); }

template <typename Kernel, typename Args>
hipError_t launch_tiles(Kernel kernel, const Args& a, int t, int nb, int64_t m, int64_t n, hipStream_t s) {
    const unsigned tm = (unsigned)((m + 64 * t - 1) / (64 * t)), tn = (unsigned)((n + 64 * t - 1) / (64 * t));
    const int lds = gemm::lds_bytes(t, t, nb);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3(tm * tn * (unsigned)a.splits), dim3(256), lds, s, a, tm, tn);
    return hipGetLastError();
}

// Four buffers where all blocks fit the CUs at once even so.
#define GLU_LAUNCH(KERNEL, M, N)                                                                          \
    [&] {                                                                                                 \
        const int64_t tiles = (((M) + 64 * p.t - 1) / (64 * p.t)) * (((N) + 64 * p.t - 1) / (64 * p.t)) * p.splits; \
        if (p.t == 4) return launch_tiles(KERNEL<4, 2>, a, 4, 2, M, N, s);                                \
        if (p.t == 2) return tiles <= 256 ? launch_tiles(KERNEL<2, 4>, a, 2, 4, M, N, s)                  \
                                          : launch_tiles(KERNEL<2, 2>, a, 2, 2, M, N, s);                 \
        return launch_tiles(KERNEL<1, 4>, a, 1, 4, M, N, s);                                              \
    }()

}  // namespace

hipError_t launch_glu_store(const GluStoreArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(glu_store_kernel, dim3(blocks_for(glu_lines(a.n) * glu_padded(a.k) / 8)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_glu_pack(const GluPackArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(glu_pack_kernel, dim3(blocks_for(a.rows * a.padded / 8)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_glu_product(const GluArgs& args, hipStream_t s) {
    GluArgs a = args;
    const int64_t lines = glu_lines(a.n);
    if (glu_few(a.rows)) {
        const dim3 grid((unsigned)(lines / 32)), block(kFewWaves * 64);
        if (a.rows <= 16) hipLaunchKernelGGL((glu_few_kernel<1>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((glu_few_kernel<2>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    const GemmShape p = gemm_plan(a.rows, lines, glu_padded(a.k));
    a.splits = p.splits;
    hipError_t e = GLU_LAUNCH(glu_product_kernel, a.rows, lines);
    if (e == hipSuccess && a.splits > 1) {
        hipLaunchKernelGGL(glu_join_kernel, dim3(blocks_for(a.rows * lines / 16)), dim3(256), 0, s, a);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_glu_act(const GluActArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(glu_act_kernel, dim3(blocks_for(a.rows * glu_lines(a.n) / 16)), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_glu_dx(const GluBackArgs& args, hipStream_t s) {
    GluBackArgs a = args;
    const GemmShape p = gemm_plan(a.rows, a.k, glu_grads(a.n));
    a.splits = p.splits;
    hipError_t e = GLU_LAUNCH(glu_dx_kernel, a.rows, a.k);
    if (e == hipSuccess && a.splits > 1) {
        hipLaunchKernelGGL(glu_join_plain_kernel, dim3(blocks_for(a.rows * ((a.k + 7) / 8))), dim3(256), 0, s, a, a.rows, 0);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_glu_dw(const GluBackArgs& args, hipStream_t s) {
    GluBackArgs a = args;
    const int64_t lines = glu_lines(a.n);
    const GemmShape p = gemm_plan(lines, a.k, a.rows);
    a.splits = p.splits;
    hipError_t e = GLU_LAUNCH(glu_dw_kernel, lines, a.k);
    if (e == hipSuccess && a.splits > 1) {
        hipLaunchKernelGGL(glu_join_plain_kernel, dim3(blocks_for(lines * ((a.k + 7) / 8))), dim3(256), 0, s, a, lines, 1);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace ags
