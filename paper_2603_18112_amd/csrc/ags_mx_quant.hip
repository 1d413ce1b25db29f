// gfx950 kernels that store tensors in 4 bits and read them back
// (include/ags_mx.h).
//
// mx_rows_kernel   blocks along the rows: 32 lanes take 256 consecutive
//                  elements, 8 each; 4 lanes share a block's scale.
// mx_cols_kernel   blocks along the columns (the transposed form): a tile
//                  goes through LDS, a thread takes 32 rows of a column.
// mx_dequant_kernel  8 codes a thread.
//
// All stream from HBM and use no matrix cores.
#include "ags_mx_device.h"
#include "ags_mx_internal.h"

namespace ags {
namespace {

constexpr int kQBlock = 256;

__device__ __forceinline__ float load_elem(const void* x, bool bf16, int64_t i) {
    if (bf16) return __uint_as_float((unsigned)static_cast<const unsigned short*>(x)[i] << 16);
    return static_cast<const float*>(x)[i];
}

// 8 elements from column c of a row that starts at element `at`; columns past
// the end read as zero.
__device__ __forceinline__ void load8(const MxQuantArgs& a, int64_t at, int64_t c, float* x) {
    if (a.aligned && c + 8 <= a.cols) {
        if (a.bf16) {
            const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(a.x) + at + c);
            const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.x) + at + c);
            const float4 u = p[0], v = p[1];
            x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = c + i < a.cols ? load_elem(a.x, a.bf16, at + c + i) : 0.0f;
}

template <bool STOCHASTIC>
__global__ __launch_bounds__(kQBlock) void mx_rows_kernel(MxQuantArgs a, int64_t units, unsigned per_row) {
    const int64_t u = (int64_t)blockIdx.x * (kQBlock / 32) + threadIdx.x / 32;
    if (u >= units) return;  // whole half-waves
    const unsigned row = (unsigned)u / per_row, chunk = (unsigned)u % per_row;
    const int lane = threadIdx.x & 31;
    const int64_t c = (int64_t)chunk * 256 + lane * 8;
    float x[8];
    load8(a, (int64_t)row * a.stride, c, x);
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, mx::magnitude(x[i]));
    m = max(m, (unsigned)__shfl_xor((int)m, 1, 64));
    m = max(m, (unsigned)__shfl_xor((int)m, 2, 64));
    const unsigned b = mx::scale_byte<STOCHASTIC>(m);
    unsigned codes = 0;
    if (b != 255u) {
        if (STOCHASTIC) {
            unsigned char r[8];
            const uint8_t* p = a.noise + (int64_t)row * a.noise_stride + c;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = c + i < a.cols ? p[i] : 0;
            codes = mx::codes_stochastic(x, b, r);
        } else {
            codes = mx::codes_nearest(x, b);
        }
    }
    const int64_t kp = (int64_t)per_row * 256;
    *reinterpret_cast<unsigned*>(a.codes + (int64_t)row * (kp / 2) + c / 2) = codes;
    if ((lane & 3) == 0) a.scales[mx::scale_at(a.rows, row, c)] = (uint8_t)b;
}

// One block: 256 rows (the padding unit of the transposed form) of 16
// columns.  Thread t loads row t; then thread t = column * 16 + part takes
// 32 rows of one column, two threads to a block of the format... each of the
// 16 parts is half a block: 16 rows.
constexpr int kTileCols = 16;

template <bool STOCHASTIC>
__global__ __launch_bounds__(kQBlock) void mx_cols_kernel(MxQuantArgs a, unsigned row_tiles) {
    __shared__ float sx[kTileCols][257];
    __shared__ uint8_t sr[kTileCols][260];
    const int tid = threadIdx.x;
    const int64_t r0 = (int64_t)(blockIdx.x % row_tiles) * 256, c0 = (int64_t)(blockIdx.x / row_tiles) * kTileCols;
    const int64_t row = r0 + tid;
#pragma unroll
    for (int j = 0; j < kTileCols; ++j) {
        const bool in = row < a.rows && c0 + j < a.cols;
        sx[j][tid] = in ? load_elem(a.x, a.bf16, row * a.stride + c0 + j) : 0.0f;
        if (STOCHASTIC) sr[j][tid] = in ? a.noise[row * a.noise_stride + c0 + j] : 0;
    }
    __syncthreads();
    const int j = tid >> 4, part = tid & 15;
    const int64_t col = c0 + j;
    float x[16];
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        x[i] = sx[j][part * 16 + i];
        m = max(m, mx::magnitude(x[i]));
    }
    m = max(m, (unsigned)__shfl_xor((int)m, 1, 64));
    if (col >= a.cols) return;
    const unsigned b = mx::scale_byte<STOCHASTIC>(m);
    unsigned codes[2] = {0, 0};
    if (b != 255u) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            codes[h] = STOCHASTIC ? mx::codes_stochastic(x + 8 * h, b, &sr[j][part * 16 + 8 * h])
                                  : mx::codes_nearest(x + 8 * h, b);
    }
    const int64_t kp = (int64_t)row_tiles * 256;
    *reinterpret_cast<uint2*>(a.codes_t + col * (kp / 2) + (r0 + part * 16) / 2) = make_uint2(codes[0], codes[1]);
    if ((part & 1) == 0) a.scales_t[mx::scale_at(a.cols, col, r0 + part * 16)] = (uint8_t)b;
}

__global__ __launch_bounds__(kQBlock) void mx_dequant_kernel(MxDequantArgs a, int64_t units, unsigned per_row) {
    const int64_t u = (int64_t)blockIdx.x * (kQBlock / 32) + threadIdx.x / 32;
    if (u >= units) return;
    const unsigned row = (unsigned)u / per_row, chunk = (unsigned)u % per_row;
    const int64_t c = (int64_t)chunk * 256 + (threadIdx.x & 31) * 8, kp = (int64_t)per_row * 256;
    const unsigned codes = *reinterpret_cast<const unsigned*>(a.codes + (int64_t)row * (kp / 2) + c / 2);
    const unsigned b = a.scales[mx::scale_at(a.rows, row, c)];
    // 2^e in two steps of normal values; the product is exact in both types
    const float s1 = __uint_as_float(b == 255u ? 0x7fc00000u : ((b >> 1) + 64u) << 23);
    const float s2 = __uint_as_float((b - (b >> 1) + 63u) << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (c + i >= a.cols) break;
        const float v = mx::code_value((codes >> (4 * i)) & 15u) * s1 * s2;
        if (a.bf16)
            static_cast<unsigned short*>(a.out)[(int64_t)row * a.stride + c + i] =
                (unsigned short)(__float_as_uint(v) >> 16);
        else
            static_cast<float*>(a.out)[(int64_t)row * a.stride + c + i] = v;
    }
}

}  // namespace

hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t s) {
    if (a.codes) {
        const unsigned per_row = (unsigned)(mx_padded(a.cols) / 256);
        const int64_t units = a.rows * per_row;
        const dim3 grid((unsigned)((units + kQBlock / 32 - 1) / (kQBlock / 32)));
        if (a.noise) hipLaunchKernelGGL(mx_rows_kernel<true>, grid, dim3(kQBlock), 0, s, a, units, per_row);
        else hipLaunchKernelGGL(mx_rows_kernel<false>, grid, dim3(kQBlock), 0, s, a, units, per_row);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.codes_t) {
        const unsigned row_tiles = (unsigned)(mx_padded(a.rows) / 256);
        const dim3 grid(row_tiles * (unsigned)((a.cols + kTileCols - 1) / kTileCols));
        if (a.noise) hipLaunchKernelGGL(mx_cols_kernel<true>, grid, dim3(kQBlock), 0, s, a, row_tiles);
        else hipLaunchKernelGGL(mx_cols_kernel<false>, grid, dim3(kQBlock), 0, s, a, row_tiles);
    }
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(const MxDequantArgs& a, hipStream_t s) {
    const unsigned per_row = (unsigned)(mx_padded(a.cols) / 256);
    const int64_t units = a.rows * per_row;
    const dim3 grid((unsigned)((units + kQBlock / 32 - 1) / (kQBlock / 32)));
    hipLaunchKernelGGL(mx_dequant_kernel, grid, dim3(kQBlock), 0, s, a, units, per_row);
    return hipGetLastError();
}

}  // namespace ags
