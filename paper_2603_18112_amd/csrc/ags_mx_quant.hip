// gfx950 kernels that store tensors in 4 bits and read them back
// (include/ags_mx.h).
//
// mx_rows_kernel     blocks along the rows: 32 lanes take 256 consecutive
//                    elements, 8 each; 4 lanes share a block's scale.
// mx_transpose_kernel     blocks along the columns (the transposed form), and those
//                    along the rows in the same pass: a tile of 128 x 128 goes
//                    through LDS, a thread takes 32 rows of a column.
// mx_dequant_kernel  8 codes a thread.
//
// A block's scale is an integer maximum of fp32 bit patterns; codes come from the
// converter instructions.  All stream from HBM and use no matrix cores.  Rows may
// start anywhere: the 16-byte accesses below need their element's alignment only.
//
// MI355X, 8192 x 8192, data from memory (from the caches as far as they go): along
// rows bf16 34 us, 5.0 TB/s (29), fp32 53, 5.7 TB/s (49), bf16 with random bytes
// 50 (42); along columns bf16 39 (31); both forms bf16 50 (40), with random bytes
// 78 (66), fp32 68 (63) and 86 (85); reading back to bf16 32 (26).  With random
// bytes both forms are bound by the converter's work as much as by memory: fp32
// moves half as much again and takes 8 us longer.  Tried: loads past the caches
// (bf16 both 46, but 45 against 40 from the caches), the columns read 4 at a time
// from LDS (58.7 against 57.5).
#include "ags_mx_device.h"
#include "ags_mx_internal.h"

namespace ags {
namespace {

constexpr int kQBlock = 256;
constexpr int kXcds = 8;

__device__ __forceinline__ void load_noise8(const uint8_t* p, int64_t left, unsigned* r) {
    if (left >= 8) {
        const auto w = *reinterpret_cast<const mx::Unaligned<unsigned, 2, 1>*>(p);
        r[0] = w.v[0], r[1] = w.v[1];
        return;
    }
    r[0] = r[1] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < left) r[i >> 2] |= (unsigned)p[i] << (8 * (i & 3));
}

// Codes of 8 elements and, stochastic, their random bytes in two dwords.
__device__ __forceinline__ unsigned stochastic8(const float* x, unsigned byte, const unsigned* r) {
    typedef mx::Stochastic S;
    S c(byte);
    c.put(0, x[0], S::seed<0>(r[0])), c.put(1, x[1], S::seed<1>(r[0]));
    c.put(2, x[2], S::seed<2>(r[0])), c.put(3, x[3], S::seed<3>(r[0]));
    c.put(4, x[4], S::seed<0>(r[1])), c.put(5, x[5], S::seed<1>(r[1]));
    c.put(6, x[6], S::seed<2>(r[1])), c.put(7, x[7], S::seed<3>(r[1]));
    return c.codes();
}
template <bool STOCHASTIC>
__device__ __forceinline__ unsigned codes8(const float* x, unsigned byte, const unsigned* r) {
    const unsigned c = STOCHASTIC ? stochastic8(x, byte, r) : mx::codes_nearest(x, byte);
    return byte == 255u ? 0u : c;
}

// The scale byte of 4 neighbouring lanes' 32 elements.
template <bool STOCHASTIC>
__device__ __forceinline__ unsigned scale_of_quad(const float* x) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, mx::magnitude(x[i]));
    m = max(m, (unsigned)__shfl_xor((int)m, 1, 64));
    m = max(m, (unsigned)__shfl_xor((int)m, 2, 64));
    return mx::scale_byte<STOCHASTIC>(m);
}

template <typename T, bool STOCHASTIC>
__global__ __launch_bounds__(kQBlock) void mx_rows_kernel(MxQuantArgs a, unsigned units, unsigned per_row) {
    const unsigned u = blockIdx.x * (kQBlock / 32) + threadIdx.x / 32;
    if (u >= units) return;  // whole half-waves
    const unsigned row = u / per_row, chunk = u % per_row;
    const int lane = threadIdx.x & 31;
    const int64_t c = (int64_t)chunk * 256 + lane * 8;
    float x[8];
    mx::load8(static_cast<const T*>(a.x) + row * a.stride + c, a.cols - c, x);
    unsigned r[2] = {0, 0};
    if (STOCHASTIC) load_noise8(a.noise + row * a.noise_stride + c, a.cols - c, r);
    const unsigned b = scale_of_quad<STOCHASTIC>(x);
    const int64_t kp = (int64_t)per_row * 256;
    *reinterpret_cast<unsigned*>(a.codes + row * (kp / 2) + c / 2) = codes8<STOCHASTIC>(x, b, r);
    if ((lane & 3) == 0) a.scales[mx::scale_at(a.rows, row, c)] = (uint8_t)b;
}

// ------------------------------------------------------------ tile kernel --

constexpr int kTile = 128;
// Eight waves to a tile: with four, two columns to a lane, LDS left fewer waves
// on a CU to cover the loads (8192 x 8192 bf16 both forms 42.6 -> 40.7 us, with
// random bytes 75.6 -> 71.5; 5001 x 2047, rows that start anywhere, 16.9 -> 12.0).
constexpr int kTBlock = 512;
// Bytes between the columns' codes in LDS: 16-byte writes of neighbouring
// columns fall on different banks.
constexpr int kCodePitch = kTile / 2 + 16;

// A column's 32 values from LDS, and their largest magnitude (as fp32 bits).
template <typename T>
struct Column;
template <>
struct Column<unsigned short> {
    unsigned w[32];
    __device__ __forceinline__ void load(const unsigned short* p) {
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = p[i * kTile];
    }
    __device__ __forceinline__ unsigned largest() const {
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) m = max(m, w[i] & 0x7fffu);
        return m << 16;
    }
    __device__ __forceinline__ float value(int i) const { return __uint_as_float(w[i] << 16); }
};
template <>
struct Column<float> {
    float w[32];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = p[i * kTile];
    }
    __device__ __forceinline__ unsigned largest() const {
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) m = max(m, mx::magnitude(w[i]));
        return m;
    }
    __device__ __forceinline__ float value(int i) const { return w[i]; }
};

// One tile.  ROWS: the form along the rows is wanted too.  The grid covers
// the padded rows and columns, since padding is stored as zeros.
template <typename T, bool STOCHASTIC, bool ROWS>
__global__ __launch_bounds__(kTBlock) void mx_transpose_kernel(MxQuantArgs a, unsigned tiles_c, unsigned tiles) {
    __shared__ alignas(16) T tile[kTile * kTile];
    __shared__ alignas(16) uint8_t noise[STOCHASTIC ? kTile * kTile : 8];
    // The codes and scales of the columns take the tile's place once it has
    // been read (with fp32 values and random bytes two blocks just fit a CU).
    uint8_t *const codes = reinterpret_cast<uint8_t*>(tile), *const col_scale = codes + kTile * kCodePitch;
    static_assert(kTile * (kCodePitch + 4) <= (int)sizeof(tile), "codes and scales fit");
    // Consecutive blocks go to the 8 XCDs in turn; each XCD takes a run of
    // squares of four tiles (padded sizes are multiples of two), so that the
    // halves of a line of codes, which neighbouring tiles write in either form,
    // meet in one L2.  Tile after tile along the rows, the halves of the columns'
    // lines went to memory apart: 8192 x 8192 bf16 from memory 57 against 50 us,
    // with random bytes 86 against 78, fp32 93 against 86.
    const unsigned xcd = blockIdx.x % kXcds, base = tiles / kXcds, rest = tiles % kXcds;
    const unsigned t = xcd * base + min(xcd, rest) + blockIdx.x / kXcds;
    const unsigned square = t / 4, squares_c = tiles_c / 2;
    const int64_t r0 = (int64_t)(square / squares_c * 2 + (t >> 1 & 1)) * kTile;
    const int64_t c0 = (int64_t)(square % squares_c * 2 + (t & 1)) * kTile;
    const int tid = threadIdx.x;
    const int64_t kp = (int64_t)tiles_c * kTile;

    // 16 threads take a row, 8 elements each; 32 rows at a time.
    const int c = (tid & 15) * 8;
    const int64_t left = a.cols - c0 - c;
    const T* px = static_cast<const T*>(a.x) + c0 + c;
    const uint8_t* pn = a.noise + c0 + c;
    constexpr int kAhead = 4;  // rows of a thread, all in flight
#pragma unroll
    for (int i0 = 0; i0 < kTile / (kTBlock / 16); i0 += kAhead) {
        float x[kAhead][8];
        unsigned r[kAhead][2];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t row = r0 + (i0 + i) * (kTBlock / 16) + (tid >> 4);
            const int64_t l = row < a.rows ? left : 0;
            mx::load8(px + row * a.stride, l, x[i]);
            if (STOCHASTIC) load_noise8(pn + row * a.noise_stride, l, r[i]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int lr = (i0 + i) * (kTBlock / 16) + (tid >> 4);
            if constexpr (sizeof(T) == 2) {
                unsigned w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = (__float_as_uint(x[i][2 * j]) >> 16) | (__float_as_uint(x[i][2 * j + 1]) & 0xffff0000u);
                *reinterpret_cast<uint4*>(&tile[lr * kTile + c]) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                float4* p = reinterpret_cast<float4*>(&tile[lr * kTile + c]);
                p[0] = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
                p[1] = make_float4(x[i][4], x[i][5], x[i][6], x[i][7]);
            }
            if (STOCHASTIC) *reinterpret_cast<uint2*>(&noise[lr * kTile + c]) = make_uint2(r[i][0], r[i][1]);
            if (ROWS) {
                const unsigned b = scale_of_quad<STOCHASTIC>(x[i]);
                const unsigned v = codes8<STOCHASTIC>(x[i], b, r[i]);
                // the row's four scales as one dword
                unsigned all = b << (2 * (tid & 12));
                all |= (unsigned)__shfl_xor((int)all, 4, 64);
                all |= (unsigned)__shfl_xor((int)all, 8, 64);
                if (r0 + lr < a.rows) {
                    *reinterpret_cast<unsigned*>(a.codes + (r0 + lr) * (kp / 2) + (c0 + c) / 2) = v;
                    if ((tid & 15) == 0) *reinterpret_cast<unsigned*>(&a.scales[mx::scale_at(a.rows, r0 + lr, c0)]) = all;
                }
            }
        }
    }
    __syncthreads();

    // Two waves take 32 rows, a lane one column.
    const int rb = tid >> 7, cc = tid & 127;
    Column<T> v;
    v.load(&tile[rb * 32 * kTile + cc]);
    const unsigned b = mx::scale_byte<STOCHASTIC>(v.largest());
    unsigned cs[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        if constexpr (STOCHASTIC) {
            mx::Stochastic s(b);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s.put(i, v.value(8 * g + i), mx::Stochastic::seed<0>(noise[(rb * 32 + 8 * g + i) * kTile + cc]));
            cs[g] = b == 255u ? 0u : s.codes();
        } else {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = v.value(8 * g + i);
            cs[g] = codes8<false>(x, b, nullptr);
        }
    }
    __syncthreads();
    *reinterpret_cast<uint4*>(codes + cc * kCodePitch + rb * 16) = make_uint4(cs[0], cs[1], cs[2], cs[3]);
    col_scale[cc * 4 + rb] = (uint8_t)b;
    __syncthreads();
    // Whole columns of the tile: 64 bytes each, four threads to a column.
    const int64_t kpt = mx_padded(a.rows);
    const int col = tid >> 2, part = (tid & 3) * 16;
    if (c0 + col < a.cols)
        *reinterpret_cast<uint4*>(a.codes_t + (c0 + col) * (kpt / 2) + r0 / 2 + part) =
            *reinterpret_cast<const uint4*>(codes + col * kCodePitch + part);
    if (tid < kTile && c0 + tid < a.cols)
        *reinterpret_cast<unsigned*>(&a.scales_t[mx::scale_at(a.cols, c0 + tid, r0)]) =
            *reinterpret_cast<const unsigned*>(&col_scale[tid * 4]);
}

// ---------------------------------------------------------------- reading --

template <typename T>
__global__ __launch_bounds__(kQBlock) void mx_dequant_kernel(MxDequantArgs a, unsigned units, unsigned per_row) {
    const unsigned u = blockIdx.x * (kQBlock / 32) + threadIdx.x / 32;
    if (u >= units) return;
    const unsigned row = u / per_row, chunk = u % per_row;
    const int64_t c = (int64_t)chunk * 256 + (threadIdx.x & 31) * 8, kp = (int64_t)per_row * 256;
    const int64_t left = a.cols - c;
    if (left <= 0) return;
    const unsigned codes = *reinterpret_cast<const unsigned*>(a.codes + row * (kp / 2) + c / 2);
    const unsigned b = a.scales[mx::scale_at(a.rows, row, c)];
    const float s = mx::scale_value(b == 255u ? 0u : b);
    float x[8];
#define MX_PAIR(I)                                                                  \
    {                                                                               \
        const mx::v2f v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, I);        \
        x[2 * I] = v[0], x[2 * I + 1] = v[1];                                       \
    }
    MX_PAIR(0) MX_PAIR(1) MX_PAIR(2) MX_PAIR(3)
#undef MX_PAIR
    if (b == 255u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(0x7fc00000u);
    }
    T* p = static_cast<T*>(a.out) + row * a.stride + c;
    if constexpr (sizeof(T) == 2) {  // every value is exact in bf16
        if (left >= 8) {
            mx::Unaligned<unsigned, 4, 2> w;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w.v[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
            *reinterpret_cast<mx::Unaligned<unsigned, 4, 2>*>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = (unsigned short)(__float_as_uint(x[i]) >> 16);
        }
    } else {
        if (left >= 8) {
            mx::Unaligned<float, 8, 4> w;
#pragma unroll
            for (int i = 0; i < 8; ++i) w.v[i] = x[i];
            *reinterpret_cast<mx::Unaligned<float, 8, 4>*>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = x[i];
        }
    }
}

template <typename T, bool STOCHASTIC>
hipError_t launch_quantize(const MxQuantArgs& a, hipStream_t s) {
    if (!a.codes_t) {
        const unsigned per_row = (unsigned)(mx_padded(a.cols) / 256), units = (unsigned)a.rows * per_row;
        hipLaunchKernelGGL((mx_rows_kernel<T, STOCHASTIC>), dim3((units + kQBlock / 32 - 1) / (kQBlock / 32)),
                           dim3(kQBlock), 0, s, a, units, per_row);
        return hipGetLastError();
    }
    const unsigned tiles_c = (unsigned)(mx_padded(a.cols) / kTile);
    const unsigned tiles = tiles_c * (unsigned)(mx_padded(a.rows) / kTile);
    if (a.codes)
        hipLaunchKernelGGL((mx_transpose_kernel<T, STOCHASTIC, true>), dim3(tiles), dim3(kTBlock), 0, s, a, tiles_c, tiles);
    else
        hipLaunchKernelGGL((mx_transpose_kernel<T, STOCHASTIC, false>), dim3(tiles), dim3(kTBlock), 0, s, a, tiles_c, tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t s) {
    if (a.bf16)
        return a.noise ? launch_quantize<unsigned short, true>(a, s) : launch_quantize<unsigned short, false>(a, s);
    return a.noise ? launch_quantize<float, true>(a, s) : launch_quantize<float, false>(a, s);
}

hipError_t launch_mx_dequantize(const MxDequantArgs& a, hipStream_t s) {
    const unsigned per_row = (unsigned)(mx_padded(a.cols) / 256), units = (unsigned)a.rows * per_row;
    const dim3 grid((units + kQBlock / 32 - 1) / (kQBlock / 32));
    if (a.bf16) hipLaunchKernelGGL(mx_dequant_kernel<unsigned short>, grid, dim3(kQBlock), 0, s, a, units, per_row);
    else hipLaunchKernelGGL(mx_dequant_kernel<float>, grid, dim3(kQBlock), 0, s, a, units, per_row);
    return hipGetLastError();
}

}  // namespace ags
