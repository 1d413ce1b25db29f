/*
 * libags microscaled 4-bit floating point: tensors held in 4.25 bits an
 * element, and the products of a linear layer on them, in the same library
 * as the AGS step.  The step keeps fp32 master weights; the products that
 * make the next gradients (forward, input gradient, weight gradient) run on
 * the matrix cores from 4-bit operands, and the weight gradient can be
 * written where ags_step reads it.
 *
 * Format (the microscaling format MXFP4 of the OCP specification 1.0).  A
 * row is cut into blocks of 32 elements.  A block has one scale 2^e, stored
 * as the byte e + 127 (E8M0; 255 marks a block that holds a NaN or an
 * infinity: every element reads back as NaN), and 32 elements of 4 bits
 * (E2M1): a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale.
 * For a block with largest magnitude A:
 *
 *   to nearest:   e = floor(log2 A) - 2, ties to the even code, magnitudes
 *                 above 6 * 2^e become 6 * 2^e;
 *   stochastic:   e = the least with A <= 6 * 2^e, so that nothing is cut
 *                 off, and |x| = (n + f) s between two neighbours n s and
 *                 (n + 1) s becomes the upper one where
 *                 f + (r + 1/2) / 256 >= 1, r the element's random byte.
 *                 The caller draws the bytes, so a run can be repeated.
 *
 * e is kept in -127 .. 125 (a zero block has -127; values below the least
 * element round to zero as above, and 6 * 2^125 is the largest value).
 *
 * Storage of a [rows, cols] tensor: cols is padded to a multiple of
 * AGS_MX_PAD; codes are [rows][padded / 2] bytes, element 2i in the low half
 * of byte i, padding 0.  Scales are [padded / 256][rows'][8] bytes, rows' the
 * rows rounded up to AGS_MX_ROWS: the 8 scales of 256 columns, row after row
 * (a product reads the scales of many rows and few columns at a time; row by
 * row they would lie one to a cache line).  Scales of padding columns are 0,
 * those of padding rows undefined.
 *
 * Products contract the blocked axis of both operands:
 *
 *   out[i][j] (+)= sum_k a[i][k] b[j][k]
 *
 * with fp32 sums.  A linear layer y = x w', w [n, k], needs x and w blocked
 * along k; its gradients dx = dy w and dw = dy' x need dy and w' blocked
 * along n, dy' and x' along the tokens: the transposed forms.
 *
 * Conventions as in ags.h: C linkage, ags_status results, arguments checked
 * on the host before any HIP call, then device pointers against their
 * allocations; the text of the last failed call on this thread from
 * ags_last_error(NULL); work goes on hip_stream and the call returns without
 * waiting.  There is no handle: the caller owns every buffer, workspaces
 * included, and orders calls that share one.  A dtype argument is an
 * ags_dtype.
 */
#ifndef AGS_MX_H
#define AGS_MX_H

#include <stddef.h>
#include <stdint.h>

#include "ags.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AGS_MX_BLOCK 32
#define AGS_MX_PAD 256
#define AGS_MX_ROWS 16

/* rows >= 0, cols >= 0 are the logical sizes (an empty tensor has no
 * buffers; its product is zero).  codes and scales are device memory of
 * ags_mx_bytes bytes, 16-byte aligned. */
typedef struct {
    uint8_t *codes;
    uint8_t *scales;
    int64_t rows, cols;
} ags_mx_tensor;

/* Bytes of a tensor's codes and scales (host only).  AGS_E_LAYOUT where
 * cols exceeds 2^24 or the elements, padding included, 2^34. */
ags_status ags_mx_bytes(int64_t rows, int64_t cols, size_t *codes, size_t *scales);

/* Store x [rows, cols] (fp32 or bf16, row i at element i * row_stride,
 * row_stride >= cols) as q [rows, cols], as qt [cols, rows] (x transposed,
 * blocked along its columns), or as both in one pass; the other may be NULL.
 * d_noise: NULL for rounding to nearest, or random bytes [rows][noise_stride]
 * (both forms use an element's one byte).  Rows need their element's alignment
 * only. */
ags_status ags_mx_quantize(const void *d_x, int32_t dtype, int64_t rows, int64_t cols,
                           int64_t row_stride, const uint8_t *d_noise, int64_t noise_stride,
                           const ags_mx_tensor *q, const ags_mx_tensor *qt, void *hip_stream);

/* Read q back to out [q.rows][row_stride] (fp32 or bf16: both hold every
 * value exactly). */
ags_status ags_mx_dequantize(const ags_mx_tensor *q, void *d_out, int32_t dtype,
                             int64_t row_stride, void *hip_stream);

/* out [a.rows][row_stride], row_stride >= b.rows, a.cols == b.cols: the
 * product, added to out's values with accumulate = 1 (in fp32, one rounding
 * to out's type).  d_workspace: ags_mx_product_workspace bytes (16-byte
 * aligned), or NULL where that is 0.  out has at most 2^34 elements and 2^26
 * rows or columns (AGS_E_LAYOUT).  The result does not depend on
 * anything but the operands: sums are added in a fixed order. */
ags_status ags_mx_product_workspace(int64_t m, int64_t n, int64_t k, size_t *out_bytes);
ags_status ags_mx_product(const ags_mx_tensor *a, const ags_mx_tensor *b, void *d_out,
                          int32_t dtype, int64_t row_stride, int32_t accumulate,
                          void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* y [rows][y_stride] = x w' for x [rows, w.cols] (as in ags_mx_quantize):
 * x is stored to nearest in the workspace and multiplied; few rows (single
 * tokens) take one kernel that does both.  The values are those of
 * ags_mx_quantize and ags_mx_product up to the order of fp32 sums. */
ags_status ags_mx_linear_workspace(int64_t rows, int64_t n, int64_t k, size_t *out_bytes);
ags_status ags_mx_linear(const void *d_x, int32_t dtype, int64_t rows, int64_t row_stride,
                         const ags_mx_tensor *w, void *d_y, int32_t y_dtype, int64_t y_stride,
                         void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* The same product for a training step: x is stored along its rows in the
 * workspace and, in the same pass, transposed as `saved` [w.cols, rows], what
 * ags_mx_linear_backward takes.  The results are bit for bit those of
 * ags_mx_quantize and ags_mx_product. */
ags_status ags_mx_linear_save_workspace(int64_t rows, int64_t n, int64_t k, size_t *out_bytes);
ags_status ags_mx_linear_save(const void *d_x, int32_t dtype, int64_t rows, int64_t row_stride,
                              const ags_mx_tensor *w, void *d_y, int32_t y_dtype, int64_t y_stride,
                              const ags_mx_tensor *saved, void *d_workspace,
                              size_t workspace_bytes, void *hip_stream);

/* Gradients of y = x w' for dy [rows, n] (with d_noise as in
 * ags_mx_quantize): dx [rows][dx_stride] = dy w of dy's type and
 * dw [n][dw_stride] (+)= dy' x.  saved: x transposed, [k, rows]; wt: w
 * transposed, [k, n], or NULL where dx is not wanted (need_dx = 0 for the
 * workspace).  dy is stored in the workspace in both forms in one pass; the
 * results are bit for bit those of ags_mx_quantize and ags_mx_product. */
ags_status ags_mx_linear_backward_workspace(int64_t rows, int64_t n, int64_t k, int32_t need_dx,
                                            size_t *out_bytes);
ags_status ags_mx_linear_backward(const void *d_dy, int32_t dtype, int64_t rows, int64_t n,
                                  int64_t row_stride, const uint8_t *d_noise, int64_t noise_stride,
                                  const ags_mx_tensor *saved, const ags_mx_tensor *wt, void *d_dx,
                                  int64_t dx_stride, void *d_dw, int32_t dw_dtype,
                                  int64_t dw_stride, int32_t accumulate, void *d_workspace,
                                  size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* AGS_MX_H */
