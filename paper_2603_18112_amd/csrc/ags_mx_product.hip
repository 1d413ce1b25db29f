// gfx950 kernels of the products of 4-bit operands (include/ags_mx.h).
//
// mx_tile_kernel    a block of four waves takes a tile of the output; stages of
//                   256 elements of the contracted axis go from memory straight
//                   into LDS while the matrix cores work on those before.
// mx_join_kernel    adds the partial sums of a contracted axis cut in parts.
// mx_few_kernel     few rows (tokens): a block of eight waves takes 16 rows of
//                   the weights, the waves share the contracted axis.
#include <algorithm>
#include <type_traits>

#include "ags_mx_device.h"
#include "ags_mx_internal.h"
#include "ags_tile_device.h"

#ifndef __gfx950__
#ifdef __HIP_DEVICE_COMPILE__
#error "gfx950 only: scaled matrix instructions and 16-byte loads into LDS"
#endif
#endif

namespace ags {
namespace {

using tile::block_barrier;
using tile::load_lds16;
using tile::load_lds4;
using tile::tile_of_block;
using tile::wait_loads;

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kFp4 = 4;  // operand format of the scaled matrix instruction

__device__ __forceinline__ v8i operand(uint4 v) {
    return v8i{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
}

using mx::v2bf;
using mx::v2f;

// To nearest even, by the hardware's converter.
__device__ __forceinline__ unsigned pack_bf16(float x, float y) {
    const v2bf v = __builtin_convertvector((v2f{x, y}), v2bf);
    unsigned u;
    __builtin_memcpy(&u, &v, 4);
    return u;
}
__device__ __forceinline__ unsigned short bf16_round(float x) { return (unsigned short)pack_bf16(x, 0.0f); }

// Where results go: the output, or one part's sums.
struct Out {
    char* p;
    int64_t stride;
    bool bf16, add;
};

__device__ __forceinline__ Out output_of(const MxProductArgs& a, unsigned split) {
    Out o{static_cast<char*>(a.out), a.stride, a.bf16 != 0, a.accumulate != 0};
    if (a.splits > 1) o = Out{reinterpret_cast<char*>(a.partials + (int64_t)split * a.m * a.n), a.n, false, false};
    return o;
}

__device__ __forceinline__ void store1(const Out& o, int64_t at, float v) {
    if (o.bf16) {
        unsigned short* p = reinterpret_cast<unsigned short*>(o.p) + at;
        *p = bf16_round(o.add ? v + __uint_as_float((unsigned)*p << 16) : v);
    } else {
        float* p = reinterpret_cast<float*>(o.p) + at;
        *p = o.add ? v + *p : v;
    }
}

// Four results of a row from column j, as many as lie before column n.
__device__ __forceinline__ void store4(const Out& o, int64_t i, int64_t j, float4 v, int64_t n) {
    const int64_t at = i * o.stride + j;
    const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int t = 0; t < 4; ++t)
        if (j + t < n) store1(o, at + t, e[t]);
}

// ------------------------------------------------------------ tile kernel --

// Tiles in bands of kBand rows (tile_of_block): 8192^3 to bf16 /
// fp32, bands of 1, 4, 6, 8, 16, 64: 265 / 311, 252 / 269, 252 / 268, 252 / 276,
// 258 / 285, 271 / 312 us; a linear layer's step of that size, three products
// after the storing kernels, bands of 3, 4, 5, 6, 7, 8, 10: 920, 951, 924, 926,
// 913, 957, 934 (and 4096 x 4096 x 16384's backward 364, 361, 360, 359, 364, 373,
// 366).  No band is best everywhere: from memory, bands of 3, 4, 5, 6, 8: 8192^3
// 264, 266, 259, 260, 267; 6144^3 157, 144, 143, 152, 144; 5000^3 87, 85, 93, 86, 94;
// 12288 x 4096 x 4096 121, 125, 119, 124, 124; 9216 x 2048 x 4096 64, 64, 64, 61, 61.
// With the operands in the caches all of these are within 2% of each other.
constexpr unsigned kBand = 6;

// 32 rows of BYTES bytes from LDS (PITCH apart) to memory, those of the first
// `rows` rows and `bytes` bytes.  T: the elements, whose alignment is all that
// the 16-byte accesses to memory need.
template <typename T, int BYTES, int PITCH, bool ADD>
__device__ __forceinline__ void store_strip(const char* strip, int lane, char* to, int64_t stride, int64_t rows,
                                            int64_t bytes) {
    constexpr int kLanes = BYTES / 16, kRows = 64 / kLanes, kN = 16 / sizeof(T);  // lanes of a row, rows of a store
    typedef mx::Unaligned<T, kN, sizeof(T)> Piece;
    const int c = (lane % kLanes) * 16, t0 = lane / kLanes;
    if (c >= bytes) return;
    const bool all = c + 16 <= bytes;
    strip += t0 * PITCH + c;
    to += t0 * stride + c;
#pragma unroll
    for (int t = 0; t < 32; t += kRows) {
        if (t0 + t >= rows) continue;
        const uint4 raw = *reinterpret_cast<const uint4*>(strip + t * PITCH);
        Piece v = __builtin_bit_cast(Piece, raw);
        char* p = to + t * stride;
        if (all) {
            if constexpr (ADD) {
                const Piece u = *reinterpret_cast<const Piece*>(p);
#pragma unroll
                for (int i = 0; i < kN; ++i) v.v[i] += u.v[i];
            }
            *reinterpret_cast<Piece*>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                T* e = reinterpret_cast<T*>(p) + i;
                if (c + (i + 1) * (int)sizeof(T) > bytes) continue;
                if constexpr (ADD) v.v[i] += *e;
                *e = v.v[i];
            }
        }
    }
}

// 32 rows of WIDE fp32 results added to bf16.
template <int WIDE, int PITCH>
__device__ __forceinline__ void store_added(const Out& o, const char* strip, int lane, int64_t row0, int64_t col0,
                                           int64_t m, int64_t n) {
    constexpr int kLanes = WIDE / 4, kRows = 64 / kLanes;
    const int c = (lane % kLanes) * 4;
#pragma unroll 2
    for (int t = lane / kLanes; t < 32; t += kRows) {
        const float4 v = *reinterpret_cast<const float4*>(strip + t * PITCH + c * 4);
        if (row0 + t < m && col0 + c < n) store4(o, row0 + t, col0 + c, v, n);
    }
}

// TM x TN: the tile in units of 64; four waves, two by two, each with TM x TN
// fragments of 32 x 32.
//
// With 256 x 256 outputs a block does 512 operations (256 multiply-adds) for each
// byte of codes it loads, so the matrix cores are the bound: pure 32 x 32 x 64 instructions on
// random codes reach 6.36 PFLOP/s here, where the card's power limit holds the
// clock to 1.5 GHz (9.6 on zeros).  MI355X, operands from the caches (from memory):
// 8192^3 to bf16 245 us, 4.5 PFLOP/s (264), to fp32 263 (276); 4096 x 4096 x 16384
// 117, 4.7 PFLOP/s (130); 4096^3 38 (44); 3000^3 25 (31); 2048 x 4096 x 4096 25 (27);
// 2048^3 10.3, 1.7 PFLOP/s (10.7); in 64 squared 64 x 16384 x 16384 24, bound by the
// weights' bytes, 6.0 TB/s (36, 4.0 TB/s).  Of 252 for 8192^3 in a long run the
// loads of codes and scales cost 45 (without those in the loop 204, timed on a
// copy) and the stores 12 (to fp32 44).  Tried: 16 x 16 x 128 instructions (7.2 PFLOP/s alone, but the
// accumulators were moved about: 259), eight waves (276), stages of 128 columns
// four deep (270), stores past the caches (248 against 244), blocks that stay
// for several tiles (268).
template <int TM, int TN, int NB>
__device__ __forceinline__ void tile_product(const MxProductArgs& a, unsigned tiles_m, unsigned tiles_n) {
    constexpr int BM = 64 * TM, BN = 64 * TN;
    constexpr int kStage = (BM + BN) * 128, kBuf = kStage + (BM + BN) * 8;
    extern __shared__ char sm[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned tiles = tiles_m * tiles_n;
    const unsigned split = blockIdx.x / tiles;
    unsigned ti, tj;
    tile_of_block<kBand>(blockIdx.x % tiles, tiles_m, tiles_n, ti, tj);
    const int64_t i0 = (int64_t)ti * BM, j0 = (int64_t)tj * BN;
    const unsigned pitch = (unsigned)(a.kp / 2);
    const int stages = (int)(a.kp / 256);
    const int s0 = (int)((int64_t)stages * split / a.splits), s1 = (int)((int64_t)stages * (split + 1) / a.splits);
    const int ma = (int)min((int64_t)BM, a.m - i0), nb = (int)min((int64_t)BN, a.n - j0);

    // Buffers of the tile's rows; of no bytes for a stage past the last, whose
    // loads have no scalar offset either (it may be taken off the buffer's size).
    auto buffer = [&](const uint8_t* p, unsigned bytes, int s) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, s < s1 ? bytes : 0u, 0x00027000);
    };
    auto scalar_off = [&](int s, unsigned bytes) { return s < s1 ? s * bytes : 0u; };
    const uint8_t *const ca = a.a + i0 * pitch, *const cb = a.b + j0 * pitch;
    const unsigned pa = (unsigned)mx_scale_rows(a.m) * 8, pb = (unsigned)mx_scale_rows(a.n) * 8;
    const unsigned chunks = (unsigned)(a.kp / 256);
    const uint8_t *const sca = a.sa + i0 * 8, *const scb = a.sb + j0 * 8;
    const unsigned sza = chunks * pa - (unsigned)i0 * 8, szb = chunks * pb - (unsigned)j0 * 8;

    // A wave's load takes 8 rows of 128 bytes.  LDS keeps rows of 128 bytes
    // whose 16-byte pieces c stand at c ^ ((row / 2) % 8): the operand reads of
    // any 16 rows that differ modulo 16 then fall on the 16 places of the 64
    // banks (with c ^ (row % 8) rows 8 apart met on the same banks).
    // Rows past the end repeat the last one; their results are not stored.
    // A stage's scales are 8 bytes a row, A's rows then B's.
    constexpr int kScale = (BM + BN) * 8 % 4096 == 0 ? 16 : 4, kScaleLoads = (BM + BN) * 8 / (256 * kScale);
    unsigned vs[kScaleLoads];
    const unsigned piece = (unsigned)((lane & 7) ^ ((4 * w + (lane >> 4)) & 7)) * 16;  // (i * 4 + w) * 8 + lane / 8
    unsigned first = (unsigned)(w * 8 + (lane >> 3)) * pitch + piece;
    const unsigned last_a = (unsigned)(ma - 1) * pitch + piece, last_b = (unsigned)(nb - 1) * pitch + piece;
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const int at = ((i * 4 + w) * 64 + lane) * kScale;  // byte of A's, then of B's
        const bool is_a = (i * 4 + w) * 64 * kScale < BM * 8;
        // (the last pair of rows may hold a padding row)
        vs[i] = is_a ? (unsigned)min(at, (ma - 1) * 8 / 16 * 16 + (at & 15)) : (unsigned)min(at - BM * 8, (nb - 1) * 8 / 16 * 16 + (at & 15));
    }
    const unsigned lds0 = (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)sm);
    constexpr int kLoads = BM / 32 + BN / 32 + kScaleLoads;
    auto load_one = [&](int i, int s, int buf) {  // load i of a stage
        const unsigned p = lds0 + buf * kBuf;
        if (i < BM / 32) {
            load_lds16(buffer(ca, ma * pitch, s), p + (i * 4 + w) * 1024, min(first + i * 32 * pitch, last_a),
                       scalar_off(s, 128));
        } else if (i < BM / 32 + BN / 32) {
            const int t = i - BM / 32;
            load_lds16(buffer(cb, nb * pitch, s), p + BM * 128 + (t * 4 + w) * 1024, min(first + t * 32 * pitch, last_b),
                       scalar_off(s, 128));
        } else {
            const int t = i - BM / 32 - BN / 32;
            const bool is_a = (t * 4 + w) * 64 * kScale < BM * 8;
            const unsigned to = p + kStage + (t * 4 + w) * 64 * kScale, off = scalar_off(s, is_a ? pa : pb);
            const __amdgpu_buffer_rsrc_t rs = buffer(is_a ? sca : scb, is_a ? sza : szb, s);
            if (kScale == 16) load_lds16(rs, to, vs[t], off);
            else load_lds4(rs, to, vs[t], off);
        }
    };

    // Operands: lane l holds row r = l % 32 of a fragment; its half h = l / 32
    // takes the pieces 4 h + j of a stage in step j of four (the order of the
    // contracted elements is free as long as both operands agree), so that a
    // stage's four scales are one dword.
    constexpr int FM = BM / 64, FN = BN / 64;  // 32 x 32 fragments of a wave
    const int r = lane & 31, h = lane >> 5, wm = w >> 1, wn = w & 1;
    int off[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) off[j] = r * 128 + (((h * 4 + j) ^ ((r >> 1) & 7)) << 4);
    const int oa = wm * (BM / 2) * 128, ob = BM * 128 + wn * (BN / 2) * 128;
    const int osa = kStage + (wm * (BM / 2) + r) * 8 + h * 4, osb = kStage + (BM + wn * (BN / 2) + r) * 8 + h * 4;
    uint4 fa[2][FM], fb[2][FN];
    int ea[2][FM], eb[2][FN];
    // Read i of a step's operands, in the order they are needed: A's first
    // fragment, all of B's, the rest of A's.
    auto read_one = [&](int i, int buf, int j, int to) {
        const char* p = sm + buf * kBuf;
        if (i >= 1 && i <= FN) {
            fb[to][i - 1] = *reinterpret_cast<const uint4*>(p + ob + (i - 1) * 4096 + off[j]);
        } else {
            const int f = i ? i - FN : 0;
            fa[to][f] = *reinterpret_cast<const uint4*>(p + oa + f * 4096 + off[j]);
        }
    };
    auto read_scales = [&](int buf, int to) {
        const char* p = sm + buf * kBuf;
#pragma unroll
        for (int f = 0; f < FM; ++f) ea[to][f] = *reinterpret_cast<const int*>(p + osa + f * 256);
#pragma unroll
        for (int f = 0; f < FN; ++f) eb[to][f] = *reinterpret_cast<const int*>(p + osb + f * 256);
    };

    // B's fragments are the instruction's first operand: four results of a
    // lane are then neighbours in a row of the output.
    v16f acc[FM][FN];
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
        for (int y = 0; y < FN; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[x][y][i] = 0.0f;

#define MX_MULTIPLY(X, J)                                                                                     \
    _Pragma("unroll") for (int y = 0; y < FN; ++y) acc[X][y] =                                                \
        __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(fb[(J) & 1][y]), operand(fa[(J) & 1][X]),     \
                                                        acc[X][y], kFp4, kFp4, J, eb[0][y], J, ea[0][X]);     \
    __builtin_amdgcn_sched_barrier(0);

    // A stage's loads are spread over the steps in which its buffer is free
    // and time is left for them to arrive: the last step of the stage NB before
    // and the first two of the next.  sched_barrier keeps the order.
    constexpr int kSlots = 3 * FM;
#define MX_LOADS(SLOT, S, BUF)                                                                       \
    _Pragma("unroll") for (int i = (SLOT) * kLoads / kSlots; i < ((SLOT) + 1) * kLoads / kSlots; ++i) \
        load_one(i, S, BUF);                                                                         \
    __builtin_amdgcn_sched_barrier(0);

    // Step J: products of one row of fragments after the other, the next
    // step's reads between them, none before the last row.
    constexpr int kReads = FM > 1 ? (FM + FN + FM - 2) / (FM > 1 ? FM - 1 : 1) : FM + FN;
#define MX_STEP(J, NEXT_BUF, SLOT, LOAD_STAGE, LOAD_BUF)                                              \
    _Pragma("unroll") for (int x = 0; x < FM; ++x) {                                                  \
        _Pragma("unroll") for (int i = x * kReads; i < (x + 1) * kReads && i < FM + FN; ++i)          \
            read_one(i, NEXT_BUF, ((J) + 1) & 3, ((J) + 1) & 1);                                      \
        MX_MULTIPLY(x, J)                                                                             \
        if ((SLOT) < 3) { MX_LOADS((SLOT) * FM + x, LOAD_STAGE, LOAD_BUF) }                           \
    }

    // One stage, in buffer cur; the operands of its first step are in registers.
    // Before its last step the next stage has arrived (those after it need not
    // have) and the block's reads of this one are done, so one barrier serves
    // both buffers.  The body has no branches, over which the compiler would move
    // the products: past the last stage the loads find a buffer of no bytes, and
    // operands are read that nothing uses.
    auto stage = [&](int s, int cur) {
        const int next = (cur + 1) % NB, last = (cur + NB - 1) % NB;
        MX_STEP(0, cur, 1, s + NB - 1, last)
        MX_STEP(1, cur, 2, s + NB - 1, last)
        MX_STEP(2, cur, 3, 0, 0)
        wait_loads<(NB - 2) * kLoads>();
        block_barrier();
        read_scales(next, 1);
        MX_STEP(3, next, 0, s + NB, cur)
#pragma unroll
        for (int f = 0; f < FM; ++f) ea[0][f] = ea[1][f];
#pragma unroll
        for (int f = 0; f < FN; ++f) eb[0][f] = eb[1][f];
    };

    if (s0 < s1) {
#pragma unroll
        for (int t = 0; t < NB - 1; ++t)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) load_one(i, s0 + t, t);
        wait_loads<(NB - 2) * kLoads>();
#pragma unroll
        for (int x = 0; x < FM; ++x) { MX_LOADS(x, s0 + NB - 1, NB - 1) }
        block_barrier();
#pragma unroll
        for (int i = 0; i < FM + FN; ++i) read_one(i, 0, 0, 0);
        read_scales(0, 0);
        for (int s = s0, cur = 0; s < s1; ++s, cur = (cur + 1) % NB) stage(s, cur);
        wait_loads<0>();
    }
#undef MX_STEP
#undef MX_LOADS
#undef MX_MULTIPLY

    // 32 rows at a time go through the wave's own part of LDS, so that the
    // stores are of whole rows.  Lane l holds row l % 32 of a fragment, and of
    // each 8 columns the four from 4 (l / 32).
    block_barrier();
    constexpr int kWide = BN / 2;
    char* strip = sm + w * 32 * (kWide * 4 + 16);
    const Out o = output_of(a, split);
#pragma unroll
    for (int x = 0; x < FM; ++x) {
        const int64_t row0 = i0 + wm * (BM / 2) + x * 32, col0 = j0 + wn * kWide;
        const int64_t rows = a.m - row0, cols = a.n - col0;
        if (o.bf16 && !o.add) {
            constexpr int kPitch = kWide * 2 + 16;
#pragma unroll
            for (int y = 0; y < FN; ++y)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const v16f v = acc[x][y];
                    *reinterpret_cast<uint2*>(strip + r * kPitch + y * 64 + g * 16 + h * 8) =
                        make_uint2(pack_bf16(v[4 * g], v[4 * g + 1]), pack_bf16(v[4 * g + 2], v[4 * g + 3]));
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            store_strip<unsigned short, kWide * 2, kPitch, false>(
                strip, lane, o.p + (row0 * o.stride + col0) * 2, o.stride * 2, rows, cols * 2);
        } else {
            constexpr int kPitch = kWide * 4 + 16;
#pragma unroll
            for (int y = 0; y < FN; ++y)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const v16f v = acc[x][y];
                    *reinterpret_cast<float4*>(strip + r * kPitch + y * 128 + g * 32 + h * 16) =
                        make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            char* to = o.p + (row0 * o.stride + col0) * 4;
            if (!o.bf16 && o.add)
                store_strip<float, kWide * 4, kPitch, true>(strip, lane, to, o.stride * 4, rows, cols * 4);
            else if (!o.bf16)
                store_strip<float, kWide * 4, kPitch, false>(strip, lane, to, o.stride * 4, rows, cols * 4);
            else store_added<kWide, kPitch>(o, strip, lane, row0, col0, a.m, a.n);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// Bytes of LDS of NB stages.
template <int TM, int TN, int NB>
constexpr int kTileLds = NB * (64 * TM + 64 * TN) * 136;

template <int TM, int TN, int NB>
__global__ __launch_bounds__(256, 1) void mx_tile_kernel(MxProductArgs a, unsigned tiles_m, unsigned tiles_n) {
    tile_product<TM, TN, NB>(a, tiles_m, tiles_n);
}

// A thread takes four elements of the output, one after the other in its rows,
// and has the loads of four parts under way.  The rule for parts keeps m n below
// 2^31, so 32 bits hold an element's number.
__global__ __launch_bounds__(256) void mx_join_kernel(MxProductArgs a) {
    typedef mx::Unaligned<float, 4, 4> Four;
    const unsigned total = (unsigned)(a.m * a.n), n = (unsigned)a.n;
    const Out o{static_cast<char*>(a.out), a.stride, a.bf16 != 0, a.accumulate != 0};
    for (unsigned t = (blockIdx.x * 256 + threadIdx.x) * 4; t < total; t += gridDim.x * 1024) {
        const unsigned i = t / n, j = t - i * n, count = min(total - t, 4u);
        Four v = {};
        for (int s = 0; s < a.splits; s += 4) {
            Four p[4] = {};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float* from = a.partials + (int64_t)min(s + u, a.splits - 1) * total + t;
                if (count == 4) {
                    p[u] = *reinterpret_cast<const Four*>(from);
                } else {
#pragma unroll
                    for (unsigned e = 0; e < 3; ++e)
                        if (e < count) p[u].v[e] = from[e];
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) v.v[e] += s + u < a.splits ? p[u].v[e] : 0.0f;
        }
        if (count == 4 && j + 4 <= n && !o.add) {
            const int64_t at = i * o.stride + j;
            if (o.bf16) {
                mx::Unaligned<unsigned, 2, 2> w;
                w.v[0] = pack_bf16(v.v[0], v.v[1]), w.v[1] = pack_bf16(v.v[2], v.v[3]);
                *reinterpret_cast<mx::Unaligned<unsigned, 2, 2>*>(reinterpret_cast<unsigned short*>(o.p) + at) = w;
            } else {
                *reinterpret_cast<Four*>(reinterpret_cast<float*>(o.p) + at) = v;
            }
            continue;
        }
#pragma unroll
        for (unsigned e = 0; e < 4; ++e) {  // added to what is there, over the end of a row, or the last few
            const unsigned r = (t + e) / n;
            if (e < count) store1(o, r * o.stride + (t + e - r * n), v.v[e]);
        }
    }
}

// ------------------------------------------------------------- few rows --

// Up to 16 * MT rows of x against all of w: every weight is read once, straight
// into registers, so the kernel is bound by the weights' bytes.  A block takes
// 16 rows of w; of each kFewWaves chunks of 256 columns a wave takes one; the
// waves' sums meet in LDS, in a fixed order.  A wave's loads are of whole lines,
// 8 rows of 128 bytes: as an operand the 16 lanes r then hold rows r / 2, the
// even ones the first half of a chunk and the odd ones the second.  Products
// with both halves of x are taken, and of their results the rows that met their
// own half: twice the matrix instructions, which wait for memory anyway.  (With
// 16 rows of 64 bytes a load, each line was asked for twice.)  T: x's type where
// the block takes up to 16 rows of x to 4 bits itself (each block anew: one
// launch instead of two, for few elements of x), or void where x is stored
// already.
//
// MI355X, weights not in the caches: 1 row 4096 x 4096 5.4 us, 16384 x 16384 28.7
// (5.0 TB/s; 31.1 with half lines and 16 waves), 1 row 4096 x 25088 14.5, 16 rows
// 17.7; from the caches 4.4, 26.4, 10.3, 14.5.  Tried: 16 waves a block (5.3,
// 28.8, 14.0, 18.3; from the caches slower), 8 or 32 rows of w a block (15.3 and
// 17.8 for 1 x 4096 x 25088), 2 to 4 chunks of a wave under way, blocks that stay
// for several groups of rows (29 for 16384 x 16384, 16 and 21 for 4096 x 25088),
// loads past the caches (26.8 for 16384 x 16384, but 12.4 against 10.3 for 4096 x
// 25088 once the weights are cached).
constexpr int kFewWaves = 8;

struct FewX {
    const void* x;  // x, or its codes
    const uint8_t* scales;
    int64_t stride;  // of x
    int64_t k;
};

// The codes of 32 elements of x, columns past the end zero; returns the scale.
template <typename T>
__device__ __forceinline__ unsigned store32(const T* p, int64_t left, uint4* codes) {
    float x[4][8];
    unsigned m = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        mx::load8(p + 8 * g, left - 8 * g, x[g]);
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, mx::magnitude(x[g][i]));
    }
    const unsigned b = mx::scale_byte<false>(m);
    *codes = make_uint4(mx::codes_nearest(x[0], b), mx::codes_nearest(x[1], b), mx::codes_nearest(x[2], b),
                        mx::codes_nearest(x[3], b));
    if (b == 255u) *codes = make_uint4(0u, 0u, 0u, 0u);
    return b;
}

template <int MT, typename T>
__device__ __forceinline__ void few_rows(const MxProductArgs& a, const FewX& fx) {
    constexpr bool kStore = !std::is_void<T>::value;
    // x's codes, [chunk][row][128] with pieces permuted as in the tile kernel,
    // and its scales, [chunk][row][8].
    extern __shared__ char sm[];
    __shared__ float red[kFewWaves][MT][4][64];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, r = lane & 15, q = lane >> 4;
    const int m = (int)a.m, chunks = (int)(a.kp / 256);
    uint8_t *const xs = reinterpret_cast<uint8_t*>(sm), *const xe = xs + chunks * m * 128;
    if constexpr (kStore) {
        const int blocks = chunks * 8;  // of a row
        for (int b = tid; b < blocks * m; b += kFewWaves * 64) {
            const int xr = b / blocks, blk = b % blocks, at = (blk >> 3) * m + xr;
            const int64_t col = (int64_t)blk * 32;
            uint4 codes;
            const unsigned e = store32(static_cast<const T*>(fx.x) + xr * fx.stride + col, fx.k - col, &codes);
            *reinterpret_cast<uint4*>(&xs[at * 128 + (((blk & 7) ^ ((xr >> 1) & 7)) << 4)]) = codes;
            xe[at * 8 + (blk & 7)] = (uint8_t)e;
        }
        __syncthreads();
    }
    const int64_t n0 = (int64_t)blockIdx.x * 16, pitch = a.kp / 2;
    const int64_t pb = mx_scale_rows(a.n) * 8, pa = mx_scale_rows(a.m) * 8;
    const uint8_t *pw[2], *pe[2];  // of rows 0 .. 7 and 8 .. 15
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t row = min(n0 + i * 8 + (r >> 1), a.n - 1);
        const int piece = (r & 1) * 4 + q;
        pw[i] = a.b + row * pitch + piece * 16;
        pe[i] = a.sb + row * 8 + piece;
    }
    v4f acc[MT][2][2];  // [rows of w][half of x]
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[t][i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int c = w; c < chunks; c += kFewWaves) {
        uint4 wv[2];
        int we[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            wv[i] = *reinterpret_cast<const uint4*>(pw[i] + (int64_t)c * 128);
            we[i] = pe[i][c * pb];
        }
        uint4 xv[MT][2] = {};
        int xw[MT][2] = {};
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int xr = t * 16 + r;
            if (xr >= m) continue;  // rows past the end multiply zeros
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int piece = j * 4 + q;
                if constexpr (kStore) {
                    const int at = c * m + xr;
                    xv[t][j] = *reinterpret_cast<const uint4*>(&xs[at * 128 + ((piece ^ ((xr >> 1) & 7)) << 4)]);
                    xw[t][j] = xe[at * 8 + piece];
                } else {
                    xv[t][j] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(fx.x) + xr * pitch +
                                                               (int64_t)c * 128 + piece * 16);
                    xw[t][j] = fx.scales[c * pa + xr * 8 + piece];
                }
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[t][i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        operand(wv[i]), operand(xv[t][j]), acc[t][i][j], kFp4, kFp4, 0, we[i], 0, xw[t][j]);
    }
    // A lane's four results are of operand rows 4 q .. 4 q + 3: rows 2 q and
    // 2 q + 1 of w, by halves.
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            red[w][t][2 * i][lane] = acc[t][i][0][0] + acc[t][i][1][1];
            red[w][t][2 * i + 1][lane] = acc[t][i][0][2] + acc[t][i][1][3];
        }
    __syncthreads();
    // Element (t, i, l): row 16 t + l % 16 of x, column 8 (i / 2) + 2 (l / 16) + i % 2.
    const Out o = output_of(a, 0);
    for (int e = tid; e < MT * 256; e += kFewWaves * 64) {
        const int t = e >> 8, l = (e >> 2) & 63, i = e & 3;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) v += red[k][t][i][l];
        const int64_t xr = t * 16 + (l & 15), col = n0 + (i >> 1) * 8 + (l >> 4) * 2 + (i & 1);
        if (xr < a.m && col < a.n) store1(o, xr * o.stride + col, v);
    }
}

template <int MT, typename T>
__global__ __launch_bounds__(kFewWaves * 64) void mx_few_kernel(MxProductArgs a, FewX x) {
    few_rows<MT, T>(a, x);
}

hipError_t launch_few(const MxProductArgs& a, const FewX& x, hipStream_t s) {
    const dim3 grid((unsigned)((a.n + 15) / 16)), block(kFewWaves * 64);
    if (a.m <= 16) hipLaunchKernelGGL((mx_few_kernel<1, void>), grid, block, 0, s, a, x);
    else hipLaunchKernelGGL((mx_few_kernel<2, void>), grid, block, 0, s, a, x);
    return hipGetLastError();
}

template <int TM, int TN, int NB>
hipError_t launch_tile(const MxProductArgs& a, unsigned tm, unsigned tn, hipStream_t s) {
    constexpr int lds = kTileLds<TM, TN, NB>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(mx_tile_kernel<TM, TN, NB>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((mx_tile_kernel<TM, TN, NB>), dim3(tm * tn * (unsigned)a.splits), dim3(256), lds, s, a, tm, tn);
    return hipGetLastError();
}

// Four buffers where all blocks fit the CUs at once even so; more blocks cover
// each other's loads.  Operands from the caches: 1024 x 4096 x 4096 (256 tiles of 128 squared) 14.4 us
// against 17.0 with two, 256 x 4096 x 25088 (in four parts) 28 against 31.6,
// 512 x 4096 x 8192 (512 tiles of 64 squared) 18.2 against 22.7; two: 2048 x 2048 x
// 500 (1024 tiles) 7.1 against 8.6, 2048 x 4096 x 4096 (512 of 128 squared) 24.6
// against 27.7.
template <int T>
hipError_t launch_tiles(const MxProductArgs& a, hipStream_t s) {
    const unsigned tm = (unsigned)((a.m + 64 * T - 1) / (64 * T)), tn = (unsigned)((a.n + 64 * T - 1) / (64 * T));
    if constexpr (T < 4) {
        constexpr unsigned fit = 256u * (163840u / (unsigned)kTileLds<T, T, 4>);
        if (tm * tn * (unsigned)a.splits <= fit) return launch_tile<T, T, 4>(a, tm, tn, s);
    }
    return launch_tile<T, T, 2>(a, tm, tn, s);
}

}  // namespace

hipError_t launch_mx_product(const MxProductArgs& args, hipStream_t s) {
    MxProductArgs a = args;
    const MxShape p = mx_product_plan(a.m, a.n, a.kp);
    a.splits = p.splits;
    if (p.few) return launch_few(a, FewX{a.a, a.sa, 0, 0}, s);
    hipError_t e = p.tm == 4 ? launch_tiles<4>(a, s) : p.tm == 2 ? launch_tiles<2>(a, s) : launch_tiles<1>(a, s);
    if (e == hipSuccess && a.splits > 1) {
        const unsigned blocks = (unsigned)std::min<int64_t>((a.m * a.n + 1023) / 1024, 4096);
        hipLaunchKernelGGL(mx_join_kernel, dim3(blocks), dim3(256), 0, s, a);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_mx_linear(const MxProductArgs& a, const void* x, bool bf16, int64_t stride, int64_t k, hipStream_t s) {
    const FewX f{x, nullptr, stride, k};
    const dim3 grid((unsigned)((a.n + 15) / 16)), block(kFewWaves * 64);
    const unsigned lds = (unsigned)(a.kp / 256 * a.m * 136);
    if (bf16) hipLaunchKernelGGL((mx_few_kernel<1, unsigned short>), grid, block, lds, s, a, f);
    else hipLaunchKernelGGL((mx_few_kernel<1, float>), grid, block, lds, s, a, f);
    return hipGetLastError();
}

}  // namespace ags
