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
//
// Or in panels: `rows` a multiple of 32 (along: zeros, or meet zeros, where it
// was rounded up to one), `pitch` of 128 (64 elements); panel (i, j), rows from 32 i and
// elements from 64 j on, is 4096 bytes in one piece, row after row, and the
// panels of the same rows follow one another.  What a tile loads in a stage then lies
// in pieces of 4 KiB, not in lines a pitch apart, which fall on few of the memory's
// channels where the pitch is a power of two.
struct Side {
    const void* p;
    int64_t pitch, rows, width;
};

// Elements of the contracted axis in a stage.
constexpr int kDepth = 64;

// Bytes of LDS of a tile of 64 TM x 64 TN: NA stages of a, NB of b.
constexpr int lds_bytes(int tm, int tn, int na, int nb) { return 64 * (tm * na + tn * nb) * 2 * kDepth; }

// One operand's part in a tile of W (64, 128 or 256) of its side.
//
// Across, LDS keeps rows of 128 bytes whose 16-byte pieces c stand at c ^ ((row
// / 2) % 8): the operand reads of any 16 rows that differ modulo 16 then fall on
// the 16 places of the 64 banks.  Along, it keeps rows of 2 W bytes, and the
// reads transpose: of 16 lanes, four read 32 bytes of each of four rows, and
// each lane gets one column of them.  The pieces are permuted by 64 bytes a row,
// so that the four rows (and the neighbouring 16 columns of the next 16 lanes)
// lie on different banks.
enum Form : int { kAcross = 0, kAlong = 1, kAcrossPanels = 2, kAlongPanels = 3 };

template <int W, int FORM>
struct Loader {
    static constexpr bool ALONG = FORM & 1, PANELS = FORM & 2;
    static constexpr int kLoads = W / 32;       // of a wave, 1024 bytes each, a stage
    static constexpr int kFragments = W / 64;   // 32 of the side each, of a wave
    static constexpr int kRow = ALONG ? 2 * W : 128, kRows = 1024 / kRow;  // bytes of a row, rows of a load
    static constexpr unsigned kStage = PANELS ? 4096 : 128;  // across: bytes to the next stage

    const char* base;     // along: of the stage that is loaded next; across: of the tile
    unsigned pitch, records, offset;
    unsigned last;        // across: offset of the last row
    unsigned first, width;
    int left;             // along: of the contracted axis
    int off[4];           // across: of step j; along: of fragment f

    __device__ __forceinline__ Loader(const Side& s, int64_t at, int stage, bool live, int w, int lane, int side) {
        const char* p = static_cast<const char*>(s.p);
        pitch = (unsigned)s.pitch;
        const int row = w * kRows + lane * 16 / kRow, piece = lane * 16 % kRow / 16;
        if constexpr (ALONG) {
            base = p + (PANELS ? at / 64 * 4096 : at * 2) + (int64_t)stage * kDepth * s.pitch;
            left = (int)(s.rows - (int64_t)stage * kDepth);
            // (in panels: the bytes of 32 rows from this column on)
            width = PANELS ? 32 * pitch - (unsigned)(at / 64 * 4096) : (unsigned)min((int64_t)W, s.width - at) * 2;
            last = offset = 0;
            const int swizzle = W == 64 ? (row >> 1) & 1 : row & 3, from = piece ^ (4 * swizzle);
            first = PANELS ? row * 128 + from / 8 * 4096 + from % 8 * 16 : row * pitch + from * 16;
            const int h = lane >> 5, g = (lane >> 4) & 1, t = (lane >> 2) & 3, c = lane & 3;
#pragma unroll
            for (int f = 0; f < kFragments; ++f)
                off[f] = (h * 32 + t) * kRow + ((side * kFragments + f) ^ (W == 64 ? t >> 1 : t)) * 64 + g * 32 + c * 8;
            records = live ? along_records() : 0u;
        } else {
            base = p + at * s.pitch;
            const int rows = (int)min((int64_t)W, s.rows - at);
            offset = stage * kStage;
            records = live ? rows * pitch : 0u;
            left = 0;
            width = 0;
            const unsigned to = (unsigned)(piece ^ ((row >> 1) & 7)) * 16;  // row + 32 i: the same
            first = (PANELS ? row * 128 : row * pitch) + to;
            last = PANELS ? (rows / 32 - 1) * 32 * pitch + first : (rows - 1) * pitch + to;
            const int r = lane & 31, h = lane >> 5;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                off[j] = (side * (W / 2) + r) * 128 + (((h * 4 + j) ^ ((r >> 1) & 7)) << 4);
        }
    }

    __device__ __forceinline__ unsigned along_records() const {
        if constexpr (PANELS) return left > 0 ? (min(left, kDepth) - 32) * pitch + width : 0u;
        return left > 0 ? (min(left, kDepth) - 1) * pitch + width : 0u;
    }

    // The next stage; one that is not `live` finds a buffer of no bytes.
    __device__ __forceinline__ void advance(bool live) {
        if constexpr (ALONG) {
            base += (int64_t)kDepth * pitch;
            left -= kDepth;
            records = live ? along_records() : 0u;
        } else {
            offset = live ? offset + kStage : 0u;  // (it may be taken off the buffer's size)
            records = live ? records : 0u;
        }
    }

    // Load i of the stage to LDS byte `to` (of the operand's part of a buffer).
    __device__ __forceinline__ void load(int i, unsigned to, int w) const {
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, records, 0x00027000);
        const unsigned at = to + (i * 4 + w) * 1024;
        constexpr int kMore = 4 * kRows;  // rows to the next load
        if constexpr (ALONG && PANELS) load_lds16(r, at, first + i * kMore / 32 * 32 * pitch + i * kMore % 32 * 128, 0u);
        else if constexpr (ALONG) load_lds16(r, at, first + i * kMore * pitch, 0u);
        else load_lds16(r, at, min(first + i * 32 * pitch, last), offset);
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

// What LDS operations the wave has under way are done.
__device__ __forceinline__ void lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A wave's 32 rows of 32 FN results as fp32 in its part of LDS, kPitch<FN> bytes
// a row.  Lane l holds row l % 32 of a fragment, and of each 8 columns the four
// from 4 (l / 32): registers 4 g .. 4 g + 3 are of columns 8 g + 4 (l / 32) on.
template <int FN>
constexpr int kPitch = FN * 128 + 16;
template <int FN>
constexpr int kStrip = 32 * kPitch<FN>;

// For outputs that read nothing.
struct Nothing {};

template <int FN>
__device__ __forceinline__ void to_strip(const v16f (&acc)[FN], char* strip, int lane) {
    char* p = strip + (lane & 31) * kPitch<FN> + (lane >> 5) * 16;
#pragma unroll
    for (int y = 0; y < FN; ++y)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<float4*>(p + y * 128 + g * 32) =
                make_float4(acc[y][4 * g], acc[y][4 * g + 1], acc[y][4 * g + 2], acc[y][4 * g + 3]);
    lds_wait();
}

// The tile at (i0, j0) of an output m x n, over stages [s0, s1) of the
// contracted axis.  A wave has TM x TN fragments of 32 x 32 results; `out` gets 32 rows of
// them at a time, and the wave's part of LDS:
//
//   out.band<TN>(fragments, strip, lane, row0, col0, rows, cols, ahead)
//
// from (row0, col0) on rows x cols lie in the output (more than the 32 x 32 TN, or
// none).  `ahead` is what out.begin<TN>(lane, row0, col0, rows, cols) returned: tiles of
// up to 128 squared have the registers to ask, before their first stage, for what their bands
// will read; larger ones ask when a band begins.
//
// LDS holds NA stages of a and NB of b (NB = NA or NA + 1).  A stage is four steps.  Loads of
// a start in the last step of stage s for s + NA, whose buffer the barrier before it
// has freed; those of b in the first step for s + NB - 1.  What a stage loads has
// at least three steps (NA = 2) to arrive.
template <typename E, int TM, int TN, int NA, int NB, int FORM_A, int FORM_B, typename Out>
__device__ __forceinline__ void product_tile(const Side& a, const Side& b, int s0, int s1, int64_t i0, int64_t j0,
                                             int64_t m, int64_t n, char* sm, const Out& out) {
    constexpr int BM = 64 * TM, BN = 64 * TN, FM = TM, FN = TN;
    static_assert(NB == NA || NB == NA + 1, "the count of loads under way below");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = w >> 1, wn = w & 1;
    Loader<BM, FORM_A> la(a, i0, s0, s0 < s1, w, lane, wm);
    Loader<BN, FORM_B> lb(b, j0, s0, s0 < s1, w, lane, wn);
    const unsigned lds0 = (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)sm);
    constexpr int kA = BM / 32, kB = BN / 32;          // a wave's loads of a stage
    constexpr int kBufA = BM * 128, kBufB = BN * 128, kAtB = NA * kBufA;

    uint4 fa[2][FM], fb[2][FN];
    // Read i of a step's operands from buffers ca and cb, in the order they are needed:
    // a's first fragment, all of b's, the rest of a's.
    auto read_one = [&](int i, int ca, int cb, int j, int to) {
        if (i >= 1 && i <= FN) fb[to][i - 1] = lb.read(sm + kAtB + cb * kBufB, i - 1, j);
        else fa[to][i ? i - FN : 0] = la.read(sm + ca * kBufA, i ? i - FN : 0, j);
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

    // A step multiplies all pairs of fragments; the next step's reads stand
    // between the products of its first half, loads between those of its second:
    // an instruction or two to each, which issue while the matrix cores work.
    // sched_barrier keeps the order.
    constexpr int kProducts = FM * FN, kReads = FM + FN, kHalf = kProducts > 8 ? kProducts / 2 : kProducts;
    constexpr int kFirst = kProducts > 8 ? kProducts / 2 : 0;
    auto step = [&](int j, int ca, int cb, auto&& load, int n) {
#pragma unroll
        for (int q = 0; q < kProducts; ++q) {
#pragma unroll
            for (int i = 0; i < kReads; ++i)
                if (i * kHalf / kReads == q) read_one(i, ca, cb, (j + 1) & 3, (j + 1) & 1);
            acc[q / FN][q % FN] = E::mfma(fb[j & 1][q % FN], fa[j & 1][q / FN], acc[q / FN][q % FN]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < n; ++i)
                if (kFirst + i * (kProducts - kFirst) / n == q) load(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto nothing = [](int) {};
    // One stage, in buffers ca and cb; the operands of its first step are in registers.
    // Before its last step the next stage has arrived (those after it need not
    // have) and the block's reads of this one are done, so one barrier serves both.
    // Past the last stage the loads find a buffer of no bytes, and operands are read
    // that nothing uses.
    constexpr int kUnderWay = (NA - 2) * kA + (NB - 2) * kB;
    auto stage = [&](int s, int ca, int cb) {
        const int next_a = ca + 1 == NA ? 0 : ca + 1, next_b = cb + 1 == NB ? 0 : cb + 1, free_b = cb ? cb - 1 : NB - 1;
        step(0, ca, cb, [&](int i) { lb.load(i, lds0 + kAtB + free_b * kBufB, w); }, kB);
        lb.advance(s + NB < s1);
        step(1, ca, cb, nothing, 0);
        step(2, ca, cb, nothing, 0);
        wait_loads<kUnderWay>();
        block_barrier();
        step(3, next_a, next_b, [&](int i) { la.load(i, lds0 + ca * kBufA, w); }, kA);
        la.advance(s + NA + 1 < s1);
    };
    const int64_t row0 = i0 + wm * (BM / 2), col0 = j0 + wn * (BN / 2);
    constexpr bool kAhead = FM <= 2;
    decltype(out.template begin<FN>(lane, row0, col0, m, n)) ahead[kAhead ? FM : 1];
    if constexpr (kAhead) {
#pragma unroll
        for (int x = 0; x < FM; ++x)
            ahead[x] = out.template begin<FN>(lane, row0 + x * 32, col0, m - row0 - x * 32, n - col0);
    }
    if (s0 < s1) {
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            if (t < NA) {
#pragma unroll
                for (int i = 0; i < kA; ++i) la.load(i, lds0 + t * kBufA, w);
                la.advance(s0 + t + 1 < s1);
            }
            if (t < NB - 1) {
#pragma unroll
                for (int i = 0; i < kB; ++i) lb.load(i, lds0 + kAtB + t * kBufB, w);
                lb.advance(s0 + t + 1 < s1);
            }
        }
        wait_loads<(NA - 1) * kA + (NB - 2) * kB>();
        block_barrier();
#pragma unroll
        for (int i = 0; i < FM + FN; ++i) read_one(i, 0, 0, 0, 0);
        for (int s = s0, ca = 0, cb = 0; s < s1; ++s) {
            stage(s, ca, cb);
            ca = ca + 1 == NA ? 0 : ca + 1;
            cb = cb + 1 == NB ? 0 : cb + 1;
        }
        wait_loads<0>();
    }

    // 32 rows at a time, through the wave's own part of LDS.
    block_barrier();
    char* strip = sm + w * kStrip<FN>;
    // (written out: the compiler gives up unrolling the loop where `out` is long, and
    // the sums would go to memory)
    auto band = [&](const v16f (&c)[FN], int x) {
        const int64_t row = row0 + x * 32;
        if constexpr (!kAhead) ahead[0] = out.template begin<FN>(lane, row, col0, m - row, n - col0);
        out.template band<FN>(c, strip, lane, row, col0, m - row, n - col0, ahead[kAhead ? x : 0]);
        lds_wait();
        __builtin_amdgcn_sched_barrier(0);
    };
    band(acc[0], 0);
    if constexpr (FM > 1) band(acc[1], 1);
    if constexpr (FM > 2) {
        band(acc[2], 2);
        band(acc[3], 3);
    }
    static_assert(FM == 1 || FM == 2 || FM == 4, "bands of a tile");
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
