/*
 * libags layer norm: rows of activations brought to mean 0 and variance 1,
 * forward and backward, in the same library as the AGS step.  The gradients
 * of the weight and the bias are reduced over the rows in fp32 and can be
 * written where ags_step reads them: a replica's row of the gradient stack.
 *
 * For a row x of n elements:
 *
 *   mean = sum x / n,  rstd = (sum (x - mean)^2 / n + eps)^(-1/2)
 *   z = (x - mean) rstd,  y = z weight + bias
 *
 * and for a gradient dy of y, with g = dy weight:
 *
 *   dx = rstd (g - sum g / n - z sum(g z) / n)
 *   dweight = sum over the rows of dy z,  dbias = sum over the rows of dy
 *
 * Everything is computed in fp32 (the variance from the differences, not
 * from the squares) and rounded once, where it is stored; but the mean is held in
 * 48 bits, so that a row far from zero loses nothing of its differences.  It is
 * saved in fp32, and the backward pass takes it as saved: its z is off by up to
 * 2^-24 |mean| rstd.  Differences must stay in fp32's range (a row's spread below
 * 3.4e38); where their squares leave it they are scaled.
 * Sums are added in an order that the sizes alone fix: equal inputs give equal
 * results bit for bit.  A row that holds a NaN or an infinity has NaN in its whole y and dx, and
 * in what dweight sums; other rows' y and dx are untouched.  Constant rows
 * have z = 0 as long as eps > 0 (with eps = 0 they divide by zero).
 *
 * Conventions as in ags.h: C linkage, ags_status results, arguments checked
 * on the host before any HIP call, then device pointers against their
 * allocations; the text of the last failed call on this thread from
 * ags_last_error(NULL); work goes on hip_stream and the call returns without
 * waiting.  There is no handle: the caller owns every buffer, workspaces
 * included, and orders calls that share one.  Outputs must not overlap each
 * other or the inputs (AGS_E_ARG).  A dtype argument is an ags_dtype.
 */
#ifndef AGS_NORM_H
#define AGS_NORM_H

#include <stddef.h>
#include <stdint.h>

#include "ags.h"

#ifdef __cplusplus
extern "C" {
#endif

/* y [rows][y_stride] from x [rows, cols] (row i at element i * x_stride;
 * rows need their element's alignment only).  d_weight, d_bias: [cols] of
 * w_dtype; NULL stands for ones and zeros.  0 <= eps <= 3.4e38; in fp32, where one
 * above zero is at least 1.2e-38.  d_saved: fp32
 * [2][rows], the means, then the rstds, for the backward pass; or NULL.
 * AGS_E_LAYOUT where cols exceeds 2^24 or rows 2^40. */
ags_status ags_layer_norm(const void *d_x, int32_t dtype, int64_t rows, int64_t cols,
                          int64_t x_stride, const void *d_weight, const void *d_bias,
                          int32_t w_dtype, double eps, void *d_y, int32_t y_dtype,
                          int64_t y_stride, float *d_saved, void *hip_stream);

/* Workspace of ags_layer_norm_backward, for calls that want dweight or dbias
 * (others need none). */
ags_status ags_layer_norm_backward_workspace(int64_t rows, int64_t cols, size_t *out_bytes);

/* Gradients for dy [rows][dy_stride], of x's type, and what the forward pass
 * saved.  dx [rows][dx_stride] has x's type; d_dweight and d_dbias [cols] are
 * of dw_dtype, added to what is there with accumulate = 1 (in fp32, one
 * rounding).  Each of the three may be NULL.  With no rows, dweight and dbias
 * are zero (or left, with accumulate). */
ags_status ags_layer_norm_backward(const void *d_dy, int64_t dy_stride, const void *d_x,
                                   int32_t dtype, int64_t rows, int64_t cols, int64_t x_stride,
                                   const float *d_saved, const void *d_weight, int32_t w_dtype,
                                   void *d_dx, int64_t dx_stride, void *d_dweight, void *d_dbias,
                                   int32_t dw_dtype, int32_t accumulate, void *d_workspace,
                                   size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* AGS_NORM_H */
