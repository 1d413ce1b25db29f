// Internal declarations of the gated products (include/ags_glu.h), shared by
// their host code and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ags_gemm_internal.h"
#include "ags_glu.h"

namespace ags {

// Rows of a laid-out weight, elements of one; elements of a row of dg and du,
// which lie side by side like the weight's rows.
constexpr int64_t glu_lines(int64_t n) { return 2 * gemm_up(n, 16); }
constexpr int64_t glu_padded(int64_t k) { return gemm_up(k, 64); }
constexpr int64_t glu_grads(int64_t n) { return gemm_up(glu_lines(n), 64); }

struct GluStoreArgs {
    const void *gate, *up;
    int64_t gate_stride, up_stride, n, k;
    void* data;
    int32_t bf16;
};

// x [rows, k] to rows of `padded` elements, the rest zero.
struct GluPackArgs {
    const void* x;
    int64_t rows, k, stride, padded;
    void* out;
};

// A product and what becomes of it.
enum GluMode : int32_t {
    kGluForward = 0,  // act(g) u to h, and g and u to saved where that is wanted
    kGluGrads = 1,    // dg and du of dh to grads
    kGluPart = 2,     // (of the tile kernel) the sums of a part of the contracted axis
};

struct GluArgs {
    const void *x, *w;  // x: rows of whole 16 bytes, k a multiple of 64 with the padding
    int64_t rows, n, k, x_stride;
    int32_t act, mode;
    void* h;
    int32_t h_bf16;
    int64_t h_stride;
    void* saved;
    const void* dh;
    int64_t dh_stride;
    void* grads;  // [rows][glu_grads(n)]
    float* partials;
    int32_t splits;
};

// dg and du from what the forward pass saved.
struct GluActArgs {
    const void *saved, *dh;
    int64_t rows, n, dh_stride;
    int32_t act;
    void* grads;
};

// dx = grads w, or dgate and dup = grads' x.
struct GluBackArgs {
    const void *grads, *w, *x;
    int64_t rows, n, k, x_stride, x_width;
    void *out, *out_up;  // dx; or dgate and dup
    int64_t stride;
    int32_t bf16, accumulate;
    float* partials;
    int32_t splits;
};

// The kernel for few rows of x: reads every weight once.  It and tiles, weights from memory,
// in graphs (us): 1 row x 1024 -> 1024 4.8 and 6.8, x 4096 -> 4096 14.3 and 19.8, x 4096 ->
// 16384 50.9 and 50.0; 16 rows 5.4 and 6.9, 15.8 and 18.4, 54.7 and 50.0, x 16384 -> 4096 47.7
// and 54.8; 24 rows 5.9 and 6.9, 18.5 and 18.8, x 4096 -> 8192 34.4 and 27.6.  (It does not cut
// the contracted axis: 1 row x 16384 -> 1024, 64 blocks, 21.3 for 67 MB, 3.2 TB/s.)
inline bool glu_few(int64_t rows, int64_t n, int64_t k) { return rows <= 16 || (rows <= 32 && n * k <= (int64_t)1 << 24); }

// Weak for the same reason as the clipping launchers.
__attribute__((weak)) hipError_t launch_glu_store(const GluStoreArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_glu_pack(const GluPackArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_glu_product(const GluArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_glu_act(const GluActArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_glu_dx(const GluBackArgs&, hipStream_t);
__attribute__((weak)) hipError_t launch_glu_dw(const GluBackArgs&, hipStream_t);

}  // namespace ags
