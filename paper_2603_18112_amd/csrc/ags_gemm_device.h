// Device functions of the products of 16-bit operands: a block of four waves
// computes a tile of
//
//   c[i][j] = sum_k a(i, k) b(j, k)
//
// with fp32 sums on the matrix instructions.  Either operand lies with its
// contracted axis along its rows ("across": row i holds its k) or along its
// columns ("along": row k holds its i); what becomes of the sums is the caller's
// functor.
#pragma once

#include "ags_mx_device.h"
#include "ags_tile_device.h"

#ifndef __gfx950__
#ifdef __HIP_DEVICE_COMPILE__
#error "gfx950 only: transposing LDS reads and 16-byte loads into LDS"
#endif
#endif

namespace ags {
namespace gemm {

using tile::block_barrier;
using tile::load_lds16;
using tile::wait_loads;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct Bf16 {
    static __device__ __forceinline__ v16f mfma(uint4 a, uint4 b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0,
                                                       0, 0);
    }
    static __device__ __forceinline__ v4f mfma16(uint4 a, uint4 b, v4f c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0,
                                                       0, 0);
    }
};
struct Fp16 {
    static __device__ __forceinline__ v16f mfma(uint4 a, uint4 b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0,
                                                      0);
    }
};

// An operand of `rows` rows, `pitch` bytes apart (a multiple of 16, as is p).
// Across: `rows` is its side of the output, and a row's elements from the end of
// the contracted axis to the next multiple of 64 are zeros (or meet zeros).
// Along: `rows` is the contracted axis, of any length, and a row holds `width`
// elements of its side (a multiple of 8).
struct Side {
    const void* p;
    int64_t pitch, rows, width;
};

// Elements of the contracted axis in a stage.
constexpr int kDepth = 64;

// Bytes of LDS of NB stages of a tile of 64 TM x 64 TN.
constexpr int lds_bytes(int tm, int tn, int nb) { return nb * 64 * (tm + tn) * 2 * kDepth; }

// One operand's part in a tile of W (64, 128 or 256) of its side.
//
// Across, LDS keeps rows of 128 bytes whose 16-byte pieces c stand at c ^ ((row
// / 2) % 8): the operand reads of any 16 rows that differ modulo 16 then fall on
// the 16 places of the 64 banks.  Along, it keeps rows of 2 W bytes, and the
// reads transpose: of 16 lanes, four read 32 bytes of each of four rows, and
// each lane gets one column of them.  The pieces are permuted by 64 bytes a row,
// so that the four rows (and the neighbouring 16 columns of the next 16 lanes)
// lie on different banks.
template <int W, bool ALONG>
struct Loader {
    static constexpr int kLoads = W / 32;       // of a wave, 1024 bytes each, a stage
    static constexpr int kFragments = W / 64;   // 32 of the side each, of a wave
    static constexpr int kRow = ALONG ? 2 * W : 128, kRows = 1024 / kRow;  // bytes of a row, rows of a load

    const char* base;
    int64_t pitch;
    int64_t rows;     // across: of the tile
    unsigned last;    // across: offset of the last row
    unsigned first, width;
    int off[4];       // across: of step j; along: of fragment f

    __device__ __forceinline__ Loader(const Side& s, int64_t at, int w, int lane, int side) {
        const char* p = static_cast<const char*>(s.p);
        pitch = s.pitch;
        const int row = w * kRows + lane * 16 / kRow, piece = lane * 16 % kRow / 16;
        if constexpr (ALONG) {
            base = p + at * 2;
            rows = s.rows;
            width = (unsigned)min((int64_t)W, s.width - at) * 2;
            const int swizzle = W == 64 ? (row >> 1) & 1 : row & 3;
            first = (unsigned)(row * pitch) + (piece ^ (4 * swizzle)) * 16;
            const int h = lane >> 5, g = (lane >> 4) & 1, t = (lane >> 2) & 3, c = lane & 3;
#pragma unroll
            for (int f = 0; f < kFragments; ++f)
                off[f] = (h * 32 + t) * kRow + ((side * kFragments + f) ^ (W == 64 ? t >> 1 : t)) * 64 + g * 32 + c * 8;
        } else {
            base = p + at * pitch;
            rows = min((int64_t)W, s.rows - at);
            const unsigned to = (unsigned)(piece ^ ((row >> 1) & 7)) * 16;  // row + 32 i: the same
            first = (unsigned)(row * pitch) + to;
            last = (unsigned)((rows - 1) * pitch) + to;
            const int r = lane & 31, h = lane >> 5;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                off[j] = (side * (W / 2) + r) * 128 + (((h * 4 + j) ^ ((r >> 1) & 7)) << 4);
        }
    }

    // Load i of stage s to LDS byte `to` (of the operand's part of a buffer); a
    // stage that is not `live` finds a buffer of no bytes.
    __device__ __forceinline__ void load(int i, int s, bool live, unsigned to, int w) const {
        const unsigned at = to + (i * 4 + w) * 1024;
        if constexpr (ALONG) {
            const int64_t left = rows - (int64_t)s * kDepth;
            const unsigned bytes = live && left > 0 ? (unsigned)((min(left, (int64_t)kDepth) - 1) * pitch) + width : 0u;
            const char* p = base + (live ? (int64_t)s * kDepth * pitch : 0);
            load_lds16(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, bytes, 0x00027000), at,
                       first + i * (4 * kRows) * (unsigned)pitch, 0u);
        } else {
            load_lds16(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0,
                                                         live ? (unsigned)(rows * pitch) : 0u, 0x00027000),
                       at, min(first + i * 32 * (unsigned)pitch, last), live ? s * 128u : 0u);
        }
    }

    // Fragment f of step j (of four) from the operand's part of a buffer.  Lane l
    // holds place l % 32 of the side, and of the stage's contracted elements the
    // eight from 32 (l / 32) + 8 j on.
    __device__ __forceinline__ uint4 read(const char* p, int f, int j) const {
        if constexpr (ALONG) {
            typedef __attribute__((address_space(3))) v4s Lds;
            struct Two {
                v4s lo, hi;
            } v;
            const auto q = (__attribute__((address_space(3))) const char*)p + off[f] + j * 8 * kRow;
            v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)q);
            v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(q + 4 * kRow));
            return __builtin_bit_cast(uint4, v);
        } else {
            return *reinterpret_cast<const uint4*>(p + off[j] + f * 4096);
        }
    }
};

// The tile at (i0, j0) of an output m x n, over stages [s0, s1) of the
// contracted axis.  `out` gets 32 rows of a wave's columns at a time, in LDS:
//
//   out(strip, pitch, lane, row0, col0, rows, cols)
//
// rows x cols of them lie in the output (cols at most WIDE = 32 TN of a wave).
// A wave's 32 x 32 fragments: TM x TN.
//
// Loads run NB - 1 stages ahead, spread between the matrix instructions of the
// steps in which their buffer is free.
template <typename E, int TM, int TN, int NB, bool ALONG_A, bool ALONG_B, typename Out>
__device__ __forceinline__ void product_tile(const Side& a, const Side& b, int s0, int s1, int64_t i0, int64_t j0,
                                             int64_t m, int64_t n, char* sm, const Out& out) {
    constexpr int BM = 64 * TM, BN = 64 * TN, FM = TM, FN = TN;
    constexpr int kBuf = (BM + BN) * 128;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w >> 1, wn = w & 1;
    const Loader<BM, ALONG_A> la(a, i0, w, lane, wm);
    const Loader<BN, ALONG_B> lb(b, j0, w, lane, wn);
    const unsigned lds0 = (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)sm);
    constexpr int kLoads = la.kLoads + lb.kLoads;

    auto load_one = [&](int i, int s, int buf) {
        const unsigned p = lds0 + buf * kBuf;
        if (i < BM / 32) la.load(i, s, s < s1, p, w);
        else lb.load(i - BM / 32, s, s < s1, p + BM * 128, w);
    };
    uint4 fa[2][FM], fb[2][FN];
    // Read i of a step's operands, in the order they are needed: a's first
    // fragment, all of b's, the rest of a's.
    auto read_one = [&](int i, int buf, int j, int to) {
        const char* p = sm + buf * kBuf;
        if (i >= 1 && i <= FN) fb[to][i - 1] = lb.read(p + BM * 128, i - 1, j);
        else fa[to][i ? i - FN : 0] = la.read(p, i ? i - FN : 0, j);
    };

    // b's fragments are the instruction's first operand: four results of a lane
    // are then neighbours in a row of the output.
    v16f acc[FM][FN];
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FN; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[x][y][i] = 0.0f;

    // A stage's loads are spread over three steps: the last of the stage NB
    // before and the first two of the next.  sched_barrier keeps the order.
    constexpr int kSlots = 3 * FM;
    auto loads = [&](int slot, int s, int buf) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            if (i >= slot * kLoads / kSlots && i < (slot + 1) * kLoads / kSlots) load_one(i, s, buf);
        __builtin_amdgcn_sched_barrier(0);
    };
    // Step j: products of one row of fragments after the other, the next step's
    // reads between them, none before the last row.
    constexpr int kReads = FM > 1 ? (FM + FN + FM - 2) / (FM > 1 ? FM - 1 : 1) : FM + FN;
    auto step = [&](int j, int next_buf, int slot, int load_stage, int load_buf) {
#pragma unroll
        for (int x = 0; x < FM; ++x) {
#pragma unroll
            for (int i = x * kReads; i < (x + 1) * kReads && i < FM + FN; ++i)
                read_one(i, next_buf, (j + 1) & 3, (j + 1) & 1);
#pragma unroll
            for (int y = 0; y < FN; ++y) acc[x][y] = E::mfma(fb[j & 1][y], fa[j & 1][x], acc[x][y]);
            __builtin_amdgcn_sched_barrier(0);
            if (slot < 3) loads(slot * FM + x, load_stage, load_buf);
        }
    };
    // One stage, in buffer cur; the operands of its first step are in registers.
    // Before its last step the next stage has arrived (those after it need not
    // have) and the block's reads of this one are done, so one barrier serves
    // both buffers.  Past the last stage the loads find a buffer of no bytes, and
    // operands are read that nothing uses.
    auto stage = [&](int s, int cur) {
        const int next = cur + 1 == NB ? 0 : cur + 1, last = cur ? cur - 1 : NB - 1;
        step(0, cur, 1, s + NB - 1, last);
        step(1, cur, 2, s + NB - 1, last);
        step(2, cur, 3, 0, 0);
        wait_loads<(NB - 2) * kLoads>();
        block_barrier();
        step(3, next, 0, s + NB, cur);
    };
    if (s0 < s1) {
#pragma unroll
        for (int t = 0; t < NB - 1; ++t)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load_one(i, s0 + t, t);
        wait_loads<(NB - 2) * kLoads>();
#pragma unroll
        for (int x = 0; x < FM; ++x) loads(x, s0 + NB - 1, NB - 1);
        block_barrier();
#pragma unroll
        for (int i = 0; i < FM + FN; ++i) read_one(i, 0, 0, 0);
        for (int s = s0, cur = 0; s < s1; ++s, cur = cur + 1 == NB ? 0 : cur + 1) stage(s, cur);
        wait_loads<0>();
    }

    // 32 rows at a time go through the wave's own part of LDS.  Lane l holds row
    // l % 32 of a fragment, and of each 8 columns the four from 4 (l / 32).
    block_barrier();
    constexpr int kWide = BN / 2, kPitch = kWide * 4 + 16;
    char* strip = sm + w * 32 * kPitch;
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int x = 0; x < FM; ++x) {
#pragma unroll
        for (int y = 0; y < FN; ++y)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const v16f v = acc[x][y];
                *reinterpret_cast<float4*>(strip + r * kPitch + y * 128 + g * 32 + h * 16) =
                    make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const int64_t row0 = i0 + wm * (BM / 2) + x * 32, col0 = j0 + wn * kWide;
        out.template strip<kWide>(strip, kPitch, lane, row0, col0, m - row0, n - col0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// To nearest even, by the hardware's converter.
__device__ __forceinline__ unsigned pack_bf16(float x, float y) {
    const mx::v2bf v = __builtin_convertvector((mx::v2f{x, y}), mx::v2bf);
    unsigned u;
    __builtin_memcpy(&u, &v, 4);
    return u;
}

__device__ __forceinline__ float bf16_value(unsigned short u) { return __uint_as_float((unsigned)u << 16); }

// 8 elements of a row from p on (an element's alignment), as many as `left`.
__device__ __forceinline__ void store8(unsigned short* p, int64_t left, const float* x) {
    mx::Unaligned<unsigned, 4, 2> w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    if (left >= 8) {
        *reinterpret_cast<mx::Unaligned<unsigned, 4, 2>*>(p) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = (unsigned short)(w.v[i >> 1] >> (16 * (i & 1)));
}
__device__ __forceinline__ void store8(float* p, int64_t left, const float* x) {
    if (left >= 8) {
        mx::Unaligned<float, 8, 4> w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w.v[i] = x[i];
        *reinterpret_cast<mx::Unaligned<float, 8, 4>*>(p) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = x[i];
}

__device__ __forceinline__ void read8(const char* strip, float* x) {
    const float4 a = *reinterpret_cast<const float4*>(strip), b = *reinterpret_cast<const float4*>(strip + 16);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

}  // namespace gemm
}  // namespace ags
