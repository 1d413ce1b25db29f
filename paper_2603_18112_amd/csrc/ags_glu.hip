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

// A thread takes 8 elements of a row of the laid-out weight.  Memory-bound: gate and up of
// 16384 x 4096 bf16 97 us, 5.5 TB/s read and written.
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
        store8(static_cast<u16*>(a.data) + line / 32 * 32 * padded + c / 64 * 2048 + line % 32 * 64 + c % 64, 8, x);
    }
}

// Rows that the products cannot read where they lie, copied: 1000 x 2047 4.6 us, a launch.
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

// act(g), and its derivative, in fp32.  The hardware's 2^x and 1 / x are within an
// ulp; the argument's rounding costs e^-g |g| ulps, of which little is left in
// g / (1 + e^-g).  (expf and a division take four times the instructions, 2 ms
// against 1.85 for 8192 x 4096 -> 16384.)
__device__ __forceinline__ float sigmoid(float g) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
}
// (1 + erf(g / sqrt 2)) / 2, and e^(-g g / 2): erfc(x) = p(t) e^(-x x), t = 1 / (1 + 0.43 x), for
// x >= 0, so that results far below zero keep their bits.  p, of degree 8, has the least largest
// relative error for 0 <= x <= 9.5 (linear programming over 3500 points): 1.5 x 2^-24; the
// whole is within (8 + 1.3 g g) 2^-24 in emulated fp32, the second part the exponent's rounding.
// (Formula 7.1.26 of Abramowitz and Stegun, of degree 5, is within 1.5e-7 absolutely: 1 % off
// at g = -8.  With it 8192 x 4096 -> 16384 forward takes 1.70 ms, so 1.71.)
__device__ __forceinline__ float normal_below(float g, float* e) {
    const float x = fabsf(g), t = __builtin_amdgcn_rcpf(fmaf(0.304055930f, x, 1.0f));
    *e = __builtin_amdgcn_exp2f(g * g * -0.72134752f);
    float p = fmaf(0.073707901f, t, -0.310373306f);
    p = fmaf(p, t, 0.383705586f);
    p = fmaf(p, t, -0.085725665f);
    p = fmaf(p, t, 0.246844411f);
    p = fmaf(p, t, 0.204951108f);
    p = fmaf(p, t, 0.244375437f);
    p = fmaf(p, t, 0.242514610f);
    const float q = 0.5f * p * t * *e;
    return g < 0.0f ? q : 1.0f - q;
}
__device__ __forceinline__ float act_of(int act, float g) {
    if (act == AGS_GLU_SILU) return g * sigmoid(g);
    float e;
    return g * normal_below(g, &e);
}
__device__ __forceinline__ void act_both(int act, float g, float* f, float* d) {
    if (act == AGS_GLU_SILU) {
        const float s = sigmoid(g);
        *f = g * s;
        *d = s * fmaf(g, 1.0f - s, 1.0f);
    } else {
        float e;
        const float c = normal_below(g, &e);
        *f = g * c;
        *d = fmaf(g * 0.39894228f, e, c);
    }
}

// g and u are saved with 24 bits each, fp32 without the last 8 of its mantissa: the
// upper 16 bits of a row's, then the next 8.  (In bf16 they would cost the gradients
// as much as their own rounding does: dgate off by 0.31 % of its norm, not 0.24.)
__device__ __forceinline__ unsigned bits24(float x) {
    const unsigned b = __float_as_uint(x);
    return (b & 0x7fffffffu) > 0x7f800000u ? b : b + 0x80u;  // (in bits 8 .. 31)
}
// Four elements' upper halves, and their next bytes.
__device__ __forceinline__ void split24(float a, float b, float c, float d, uint2* hi, unsigned* lo) {
    const unsigned x = bits24(a), y = bits24(b), z = bits24(c), w = bits24(d);
    *hi = make_uint2(__builtin_amdgcn_perm(y, x, 0x07060302u), __builtin_amdgcn_perm(w, z, 0x07060302u));
    const unsigned p = __builtin_amdgcn_perm(y, x, 0x0c0c0501u), q = __builtin_amdgcn_perm(w, z, 0x0c0c0501u);
    *lo = p | (q << 16);
}
__device__ __forceinline__ void join24(uint4 hi, uint2 lo, float* x) {
    const unsigned h[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned l = (i < 4 ? lo.x : lo.y) >> (8 * (i & 3)) & 0xffu;
        x[i] = __uint_as_float((i & 1 ? h[i >> 1] & 0xffff0000u : h[i >> 1] << 16) | l << 8);
    }
}

// Where a row of dg and du ends in a stage of their products: zeros up to there.
__device__ __forceinline__ void pad_grads(u16* row, int64_t n, int half) {
    const int64_t lines = glu_lines(n);
    if (lines < glu_grads(n)) {
        *reinterpret_cast<uint4*>(row + lines + half * 16) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(row + lines + half * 16 + 8) = make_uint4(0, 0, 0, 0);
    }
}

// Eight sums of gate and the same eight of up, hidden units from `unit` on.
__device__ __forceinline__ void put_pair(const GluArgs& a, int64_t row, int64_t unit, float* g, float* u) {
    const int64_t lines = glu_lines(a.n), line = unit / 16 * 32 + unit % 16, left = a.n - unit;
    if (a.mode == kGluForward) {
        if (a.saved) {
            char* s = static_cast<char*>(a.saved) + row * 3 * lines;
#pragma unroll
            for (int up = 0; up < 2; ++up) {
                const float* x = up ? u : g;
                uint2 hi[2];
                unsigned lo[2];
                split24(x[0], x[1], x[2], x[3], &hi[0], &lo[0]);
                split24(x[4], x[5], x[6], x[7], &hi[1], &lo[1]);
                *reinterpret_cast<uint4*>(s + (line + 16 * up) * 2) = make_uint4(hi[0].x, hi[0].y, hi[1].x, hi[1].y);
                *reinterpret_cast<uint2*>(s + 2 * lines + line + 16 * up) = make_uint2(lo[0], lo[1]);
            }
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
        u16* p = static_cast<u16*>(a.grads) + row * glu_grads(a.n);
        store8(p + line, 8, g);
        store8(p + line + 16, 8, u);
        if (line / 32 * 32 + 32 == lines) pad_grads(p, a.n, unit % 16 / 8);
    }
}

// 32 rows of BYTES bytes from LDS, PITCH apart, to memory: those of the first
// `rows` rows and `bytes` bytes.  T: the elements, whose alignment is all that the
// 16-byte stores need.
template <typename T, int BYTES, int PITCH, bool NT = false>
__device__ __forceinline__ void store_rows(const char* strip, int lane, char* to, int64_t stride, int64_t rows,
                                           int64_t bytes) {
    constexpr int kLanes = BYTES / 16, kRows = 64 / kLanes, kN = 16 / sizeof(T);
    typedef Unaligned<T, kN, sizeof(T)> Piece;
    const int c = lane % kLanes * 16, t0 = lane / kLanes;
    if (c >= bytes) return;
#pragma unroll
    for (int t = 0; t < 32; t += kRows) {
        if (t0 + t >= rows) continue;
        const uint4 raw = *reinterpret_cast<const uint4*>(strip + (t0 + t) * PITCH + c);
        const Piece v = __builtin_bit_cast(Piece, raw);
        char* p = to + (t0 + t) * stride + c;
        if constexpr (NT) {
            typedef unsigned u4 __attribute__((ext_vector_type(4)));
            __builtin_nontemporal_store(__builtin_bit_cast(u4, raw), reinterpret_cast<u4*>(p));
        } else if (c + 16 <= bytes) {
            *reinterpret_cast<Piece*>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (c + (i + 1) * (int)sizeof(T) <= bytes) reinterpret_cast<T*>(p)[i] = v.v[i];
        }
    }
}

// Rows of fp32 results in LDS, eight at a time: f(t, c, x) for row t and column c.
template <int FN, typename F>
__device__ __forceinline__ void each8(const char* strip, int lane, int64_t rows, int64_t cols, const F& f) {
    constexpr int kLanes = FN * 4, kRows = 64 / kLanes;
    const int c = lane % kLanes * 8;
    if (c >= cols) return;
    const int end = (int)min(rows, (int64_t)32);
#pragma unroll 2
    for (int t = lane / kLanes; t < end; t += kRows) {
        float x[8];
        gemm::read8(strip + t * gemm::kPitch<FN> + c * 4, x);
        f(t, c, x);
    }
}

// One part's sums to rows of n.
template <int FN>
__device__ __forceinline__ void put_part(const gemm::v16f (&acc)[FN], float* part, int64_t n, char* strip, int lane,
                                         int64_t row0, int64_t col0, int64_t rows, int64_t cols) {
    gemm::to_strip<FN>(acc, strip, lane);
    each8<FN>(strip, lane, rows, cols,
              [&](int t, int c, float* x) { store8(part + (row0 + t) * n + col0 + c, cols - c, x); });
}

// What a tile's sums of gate and up become.  A fragment's registers 0 .. 7 are of gate, 8 .. 15
// of up, for the same units of the block of 16: 4 h .. 4 h + 3 and 8 + 4 h .. (h:
// the lane's half).  So the activation is taken in registers, and what goes through
// LDS, for stores of whole rows, is rounded already.
template <int MODE, int ACT>
struct PairOut {
    const GluArgs& a;
    float* part;

    template <int FN>
    __device__ __forceinline__ gemm::Nothing begin(int, int64_t, int64_t, int64_t, int64_t) const {
        return {};
    }

    template <int FN>
    __device__ __forceinline__ void band(const gemm::v16f (&acc)[FN], char* strip, int lane, int64_t row0, int64_t col0,
                                         int64_t rows, int64_t cols, gemm::Nothing) const {
        if constexpr (MODE == kGluPart) put_part<FN>(acc, part, glu_lines(a.n), strip, lane, row0, col0, rows, cols);
        else if constexpr (MODE == kGluForward) forward<FN>(acc, strip, lane, row0, col0, rows, cols);
        else grads<FN>(acc, strip, lane, row0, col0, rows, cols);
    }

    template <int FN>
    __device__ __forceinline__ void forward(const gemm::v16f (&acc)[FN], char* strip, int lane, int64_t row0,
                                            int64_t col0, int64_t rows, int64_t cols) const {
        const int r = lane & 31, h = lane >> 5;
        const int64_t unit = col0 / 2, left = a.n - unit, lines = glu_lines(a.n);
        constexpr int kHalf = FN * 32 + 16, kFull = FN * 64 + 16;  // bytes of a row in LDS
#pragma unroll
        for (int y = 0; y < FN; ++y)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                float x[4];
                __builtin_amdgcn_sched_barrier(0);  // (a few registers at a time)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = act_of(ACT, acc[y][4 * g + i]) * acc[y][8 + 4 * g + i];
                if (a.h_bf16)
                    *reinterpret_cast<uint2*>(strip + r * kHalf + y * 32 + g * 16 + h * 8) =
                        make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
                else
                    *reinterpret_cast<float4*>(strip + r * kFull + y * 64 + g * 32 + h * 16) =
                        make_float4(x[0], x[1], x[2], x[3]);
            }
        gemm::lds_wait();
        const int64_t at = row0 * a.h_stride + unit;
        if (a.h_bf16)
            store_rows<u16, FN * 32, kHalf>(strip, lane, static_cast<char*>(a.h) + at * 2, a.h_stride * 2, rows, left * 2);
        else
            store_rows<float, FN * 64, kFull>(strip, lane, static_cast<char*>(a.h) + at * 4, a.h_stride * 4, rows,
                                              left * 4);
        if (!a.saved) return;
        gemm::lds_wait();
        char* low = strip + 32 * kFull;
#pragma unroll
        for (int y = 0; y < FN; ++y)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint2 hi;
                unsigned lo;
                split24(acc[y][4 * g], acc[y][4 * g + 1], acc[y][4 * g + 2], acc[y][4 * g + 3], &hi, &lo);
                *reinterpret_cast<uint2*>(strip + r * kFull + y * 64 + g * 16 + h * 8) = hi;
                *reinterpret_cast<unsigned*>(low + r * kHalf + y * 32 + g * 8 + h * 4) = lo;
            }
        gemm::lds_wait();
        char* s = static_cast<char*>(a.saved) + row0 * 3 * lines;
        store_rows<unsigned, FN * 64, kFull, true>(strip, lane, s + col0 * 2, 3 * lines, rows, cols * 2);
        store_rows<unsigned, FN * 32, kHalf, true>(low, lane, s + 2 * lines + col0, 3 * lines, rows, cols);
    }

    template <int FN>
    __device__ __forceinline__ void grads(const gemm::v16f (&acc)[FN], char* strip, int lane, int64_t row0,
                                          int64_t col0, int64_t rows, int64_t cols) const {
        const int r = lane & 31, h = lane >> 5;
        constexpr int kHalf = FN * 32 + 16, kFull = FN * 64 + 16, kLanes = FN * 2, kRows = 64 / kLanes;
        {   // dh: whole rows, zeros past their ends
            const int64_t c = lane % kLanes * 8, unit = col0 / 2 + c;
#pragma unroll
            for (int t = lane / kLanes; t < 32; t += kRows) {
                float x[8];
                load8(static_cast<const u16*>(a.dh) + (row0 + t) * a.dh_stride + unit, t < rows ? a.n - unit : 0, x);
                store8(reinterpret_cast<u16*>(strip + t * kHalf) + c, 8, x);
            }
        }
        gemm::lds_wait();
        uint2 d[FN][2];
#pragma unroll
        for (int y = 0; y < FN; ++y)
#pragma unroll
            for (int g = 0; g < 2; ++g)
                d[y][g] = *reinterpret_cast<const uint2*>(strip + r * kHalf + y * 32 + g * 16 + h * 8);
        gemm::lds_wait();
#pragma unroll
        for (int y = 0; y < FN; ++y)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const float dh[4] = {bf16_value((u16)d[y][g].x), bf16_value((u16)(d[y][g].x >> 16)),
                                     bf16_value((u16)d[y][g].y), bf16_value((u16)(d[y][g].y >> 16))};
                float dg[4], du[4];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float f, e;
                    act_both(ACT, acc[y][4 * g + i], &f, &e);
                    dg[i] = dh[i] * acc[y][8 + 4 * g + i] * e;
                    du[i] = dh[i] * f;
                }
                char* p = strip + r * kFull + y * 64 + g * 16 + h * 8;
                *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(dg[0], dg[1]), pack_bf16(dg[2], dg[3]));
                *reinterpret_cast<uint2*>(p + 32) = make_uint2(pack_bf16(du[0], du[1]), pack_bf16(du[2], du[3]));
            }
        gemm::lds_wait();
        const int64_t pitch = glu_grads(a.n);
        u16* to = static_cast<u16*>(a.grads) + row0 * pitch;
        store_rows<unsigned, FN * 64, kFull>(strip, lane, reinterpret_cast<char*>(to + col0), pitch * 2, rows, cols * 2);
        if (cols > 0 && cols <= FN * 32 && r < rows) pad_grads(to + r * pitch, a.n, h);
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

// dx, or (DW) rows of dgate and dup, sixteen of each in turn.
template <bool DW>
struct RowOut {
    const GluBackArgs& a;
    float* part;

    template <int FN>
    __device__ __forceinline__ gemm::Nothing begin(int, int64_t, int64_t, int64_t, int64_t) const {
        return {};
    }

    template <int FN>
    __device__ __forceinline__ void band(const gemm::v16f (&acc)[FN], char* strip, int lane, int64_t row0, int64_t col0,
                                         int64_t rows, int64_t cols, gemm::Nothing) const {
        if (part) {
            put_part<FN>(acc, part, a.k, strip, lane, row0, col0, rows, cols);
        } else if (a.bf16 && !a.accumulate) {
            const int r = lane & 31, h = lane >> 5;
            constexpr int kFull = FN * 64 + 16;
#pragma unroll
            for (int y = 0; y < FN; ++y)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<uint2*>(strip + r * kFull + y * 64 + g * 16 + h * 8) =
                        make_uint2(pack_bf16(acc[y][4 * g], acc[y][4 * g + 1]),
                                   pack_bf16(acc[y][4 * g + 2], acc[y][4 * g + 3]));
            gemm::lds_wait();
            const int64_t row = DW ? row0 / 2 : row0, left = DW ? min((int64_t)16, a.n - row) : rows;
            const int64_t at = (row * a.stride + col0) * 2;
            if constexpr (DW) {
                store_rows<u16, FN * 64, kFull>(strip, lane, static_cast<char*>(a.out) + at, a.stride * 2, left, cols * 2);
                store_rows<u16, FN * 64, kFull>(strip + 16 * kFull, lane, static_cast<char*>(a.out_up) + at, a.stride * 2,
                                                left, cols * 2);
            } else {
                store_rows<u16, FN * 64, kFull>(strip, lane, static_cast<char*>(a.out) + at, a.stride * 2, left, cols * 2);
            }
        } else {
            gemm::to_strip<FN>(acc, strip, lane);
            each8<FN>(strip, lane, rows, cols, [&](int t, int c, float* x) { put_row(a, DW, row0 + t, col0 + c, x); });
        }
    }
};

// --------------------------------------------------------------- products --

constexpr unsigned kBand = 4;

// The tile of this block, and its part of the contracted axis.
struct Place {
    int64_t i0, j0;
    int s0, s1;
    unsigned split;
};

template <int TM, int TN>
__device__ __forceinline__ Place place(int64_t k, int splits, unsigned tm, unsigned tn) {
    const unsigned tiles = tm * tn;
    Place p;
    p.split = blockIdx.x / tiles;
    unsigned ti, tj;
    tile::tile_of_block<kBand>(blockIdx.x % tiles, tm, tn, ti, tj);
    p.i0 = (int64_t)ti * 64 * TM;
    p.j0 = (int64_t)tj * 64 * TN;
    const int stages = (int)((k + gemm::kDepth - 1) / gemm::kDepth);
    p.s0 = (int)((int64_t)stages * p.split / splits);
    p.s1 = (int)((int64_t)stages * (p.split + 1) / splits);
    return p;
}

// Its sums' place where the axis is cut.
__device__ __forceinline__ float* part_of(float* partials, int splits, const Place& p, int64_t m, int64_t n) {
    return splits > 1 ? partials + (int64_t)p.split * m * n : nullptr;
}

// The three products are bound by the matrix instructions and, with them, by the card's power:
// 8192 x 4096 -> 16384 (2.2 TFLOP each) forward 1.64 ms (1.34 PFLOP/s; with g and u saved
// 1.80), dx 1.68, dw 1.65, matrix pipes busy 66, 70 and 74 % of the cycles, the clock at
// 1.6 to 1.7 GHz (the library's bf16 products of those sizes: 1.60, 1.60, 1.88).  Small ones,
// in tiles of less than 256 squared, by LDS reads: 1000 x 2047 -> 1001 17 us each.
template <int TM, int TN, int NA, int NB, int MODE, int ACT>
__global__ __launch_bounds__(256, 1) void glu_product_kernel(GluArgs a, unsigned tm, unsigned tn) {
    extern __shared__ __attribute__((aligned(16))) char sm[];
    const int64_t lines = glu_lines(a.n), padded = glu_padded(a.k);
    const Place p = place<TM, TN>(padded, a.splits, tm, tn);
    gemm::product_tile<gemm::Bf16, TM, TN, NA, NB, gemm::kAcross, gemm::kAcrossPanels>(
        Side{a.x, a.x_stride * 2, a.rows, 0}, Side{a.w, padded * 2, lines, 0}, p.s0, p.s1, p.i0, p.j0, a.rows, lines, sm,
        PairOut<MODE, ACT>{a, part_of(a.partials, a.splits, p, a.rows, lines)});
}

template <int TM, int TN, int NA, int NB>
__global__ __launch_bounds__(256, 1) void glu_dx_kernel(GluBackArgs a, unsigned tm, unsigned tn) {
    extern __shared__ __attribute__((aligned(16))) char sm[];
    const int64_t lines = glu_lines(a.n), padded = glu_padded(a.k), grads = glu_grads(a.n);
    const Place p = place<TM, TN>(grads, a.splits, tm, tn);
    gemm::product_tile<gemm::Bf16, TM, TN, NA, NB, gemm::kAcross, gemm::kAlongPanels>(
        Side{a.grads, grads * 2, a.rows, 0}, Side{a.w, padded * 2, lines, padded}, p.s0, p.s1, p.i0, p.j0, a.rows, a.k, sm,
        RowOut<false>{a, part_of(a.partials, a.splits, p, a.rows, a.k)});
}

template <int TM, int TN, int NA, int NB>
__global__ __launch_bounds__(256, 1) void glu_dw_kernel(GluBackArgs a, unsigned tm, unsigned tn) {
    extern __shared__ __attribute__((aligned(16))) char sm[];
    const int64_t lines = glu_lines(a.n), grads = glu_grads(a.n);
    const Place p = place<TM, TN>(a.rows, a.splits, tm, tn);
    gemm::product_tile<gemm::Bf16, TM, TN, NA, NB, gemm::kAlong, gemm::kAlong>(
        Side{a.grads, grads * 2, a.rows, grads}, Side{a.x, a.x_stride * 2, a.rows, a.x_width}, p.s0, p.s1, p.i0, p.j0,
        lines, a.k, sm, RowOut<true>{a, part_of(a.partials, a.splits, p, lines, a.k)});
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

// dg and du: 6 bytes of g and u, 2 of dh and 4 written for each unit and row.  Memory-bound:
// 8192 x 16384 292 us, 5.5 TB/s.
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
        const char* p = static_cast<const char*>(a.saved) + row * 3 * lines;
        const int64_t line = unit / 16 * 32 + unit % 16;
        float x[8], u[8];
        join24(*reinterpret_cast<const uint4*>(p + line * 2), *reinterpret_cast<const uint2*>(p + 2 * lines + line), x);
        join24(*reinterpret_cast<const uint4*>(p + line * 2 + 32),
               *reinterpret_cast<const uint2*>(p + 2 * lines + line + 16), u);
        put_pair(g, row, unit, x, u);
    }
}

// --------------------------------------------------------------- few rows --

// Up to 16 MT rows of x against all of w: every weight is read once, straight
// into registers, so the kernel is bound by the weights' bytes.  A block takes 32
// lines of w, 16 units of gate and of up; its waves share the contracted axis and
// their sums meet in LDS, in a fixed order.  A wave's loads are of whole cache lines, 8
// lines of w and 128 bytes each, one after the other in memory: as an operand the 16
// lanes r then hold line r / 2, the even ones the first 32 of 64 elements, the odd
// ones the second.  Products with both halves of x are taken, and of their results those
// that met their own half: twice the matrix instructions, which wait for memory anyway.
// One row through two weights of 4096 x 4096 12.9 us, 5.2 TB/s of weights.
constexpr int kFewWaves = 8;

template <int MT>
struct FewOperands {
    static constexpr int kBatch = MT == 1 ? 2 : 1;  // chunks of 64 elements; two such sets are under way
    uint4 w[kBatch][4], x[kBatch][MT][2];
};

template <int MT>
__global__ __launch_bounds__(kFewWaves * 64) void glu_few_kernel(GluArgs a) {
    __shared__ float red[kFewWaves][2][2][2][MT][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int64_t padded = glu_padded(a.k), line = (int64_t)blockIdx.x * 32;
    const int chunks = (int)(padded / 64);
    // a chunk is a panel of w: gate's lines 0 .. 7 and 8 .. 15, up's
    const u16* pw = static_cast<const u16*>(a.w) + line * padded + (r >> 1) * 64 + (r & 1) * 32 + q * 8;
    const u16* px[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
        px[t] = static_cast<const u16*>(a.x) + min((int64_t)(t * 16 + r), a.rows - 1) * a.x_stride + q * 8;
    gemm::v4f acc[4][MT][2];
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[s][t][j] = gemm::v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // Chunks past the end read the last one again, and multiply zeros.
    auto load = [&](FewOperands<MT>& o, int c) {
#pragma unroll
        for (int b = 0; b < FewOperands<MT>::kBatch; ++b) {
            const int at = c + b * kFewWaves, from = min(at, chunks - 1);
#pragma unroll
            for (int s = 0; s < 4; ++s) o.w[b][s] = *reinterpret_cast<const uint4*>(pw + from * 2048 + s * 512);
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    o.x[b][t][j] = *reinterpret_cast<const uint4*>(px[t] + from * 64 + j * 32);
                    if (at >= chunks) o.x[b][t][j] = make_uint4(0, 0, 0, 0);
                }
            if (at >= chunks) o.w[b][0] = o.w[b][1] = o.w[b][2] = o.w[b][3] = make_uint4(0, 0, 0, 0);
        }
    };
    auto multiply = [&](const FewOperands<MT>& o) {
#pragma unroll
        for (int b = 0; b < FewOperands<MT>::kBatch; ++b)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[s][t][j] = gemm::Bf16::mfma16(o.w[b][s], o.x[b][t][j], acc[s][t][j]);
    };
    constexpr int kRound = kFewWaves * FewOperands<MT>::kBatch;
    if (w < chunks) {
        FewOperands<MT> one, two;
        load(one, w);
        for (int c = w; c < chunks; c += 2 * kRound) {
            if (c + kRound < chunks) load(two, c + kRound);
            multiply(one);
            if (c + kRound >= chunks) break;
            if (c + 2 * kRound < chunks) load(one, c + 2 * kRound);
            multiply(two);
        }
    }
    // A lane's four results are of operand lines 4 q .. 4 q + 3: lines 2 q and 2 q + 1 of w,
    // by halves.
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            red[w][s >> 1][s & 1][0][t][lane] = acc[s][t][0][0] + acc[s][t][1][1];
            red[w][s >> 1][s & 1][1][t][lane] = acc[s][t][0][2] + acc[s][t][1][3];
        }
    __syncthreads();
    // Eight units of a row to a thread.
    for (int e = threadIdx.x; e < MT * 32; e += kFewWaves * 64) {
        const int t = e >> 5, row = e >> 1 & 15, half = e & 1;
        if (t * 16 + row >= a.rows) continue;
        float x[2][8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int up = 0; up < 2; ++up) {
                x[up][i] = 0.0f;
#pragma unroll
                for (int v = 0; v < kFewWaves; ++v) x[up][i] += red[v][up][half][i & 1][t][(i >> 1) * 16 + row];
            }
        put_pair(a, t * 16 + row, line / 2 + half * 8, x[0], x[1]);
    }
}

// --------------------------------------------------------------- launches --

unsigned blocks_for(int64_t items) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + 255) / 256, 8192)); }

template <typename Kernel, typename Args>
hipError_t launch_tiles(Kernel kernel, const Args& a, const GemmShape& p, int na, int nb, int64_t m, int64_t n, hipStream_t s) {
    const int64_t tiles_m = gemm_tiles(m, p.tm), tiles_n = gemm_tiles(n, p.tn);
    if (tiles_m * tiles_n > kGemmMaxBlocks / a.splits) return hipErrorInvalidConfiguration;
    const unsigned tm = (unsigned)tiles_m, tn = (unsigned)tiles_n;
    const int lds = gemm::lds_bytes(p.tm, p.tn, na, nb);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3(tm * tn * (unsigned)a.splits), dim3(256), lds, s, a, tm, tn);
    return hipGetLastError();
}

// Four buffers where all blocks fit the CUs at once even so.
#define GLU_LAUNCH(KERNEL, M, N, ...)                                                                     \
    [&] {                                                                                                 \
        const bool one = gemm_tiles(M, p.tm) * gemm_tiles(N, p.tn) * p.splits <= 256;                     \
        if (p.tm == 4) return launch_tiles(KERNEL<4, 4, 2, 3 __VA_ARGS__>, a, p, 2, 3, M, N, s);          \
        if (p.tn == 2) return one ? launch_tiles(KERNEL<2, 2, 4, 4 __VA_ARGS__>, a, p, 4, 4, M, N, s)     \
                                  : launch_tiles(KERNEL<2, 2, 2, 2 __VA_ARGS__>, a, p, 2, 2, M, N, s);    \
        if (p.tm == 2) return one ? launch_tiles(KERNEL<2, 1, 4, 4 __VA_ARGS__>, a, p, 4, 4, M, N, s)     \
                                  : launch_tiles(KERNEL<2, 1, 3, 3 __VA_ARGS__>, a, p, 3, 3, M, N, s);    \
        return launch_tiles(KERNEL<1, 1, 4, 4 __VA_ARGS__>, a, p, 4, 4, M, N, s);                         \
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
    if (glu_few(a.rows, a.n, a.k)) {
        const dim3 grid((unsigned)(lines / 32)), block(kFewWaves * 64);
        if (a.rows <= 16) hipLaunchKernelGGL((glu_few_kernel<1>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((glu_few_kernel<2>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    const GemmShape p = gemm_plan(a.rows, lines, glu_padded(a.k));
    a.splits = p.splits;
    hipError_t e;
    if (a.splits > 1) e = GLU_LAUNCH(glu_product_kernel, a.rows, lines, , kGluPart, AGS_GLU_SILU);
    else if (a.mode == kGluForward && a.act == AGS_GLU_SILU)
        e = GLU_LAUNCH(glu_product_kernel, a.rows, lines, , kGluForward, AGS_GLU_SILU);
    else if (a.mode == kGluForward) e = GLU_LAUNCH(glu_product_kernel, a.rows, lines, , kGluForward, AGS_GLU_GELU);
    else if (a.act == AGS_GLU_SILU) e = GLU_LAUNCH(glu_product_kernel, a.rows, lines, , kGluGrads, AGS_GLU_SILU);
    else e = GLU_LAUNCH(glu_product_kernel, a.rows, lines, , kGluGrads, AGS_GLU_GELU);
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
