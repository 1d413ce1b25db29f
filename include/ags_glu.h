/*
 * libags gated feed-forward products: the wide half of a gated feed-forward
 * block,
 *
 *   h = act(g) * u,  g = x gate',  u = x up'
 *
 * for x [rows, k] and two weights [n, k], forward and backward, in the same
 * library as the AGS step.  Both products, the activation and the
 * elementwise product are one kernel; for a gradient dh of h
 *
 *   dg = dh u act'(g),  du = dh act(g)
 *   dx = dg gate + du up,  dgate = dg' x,  dup = du' x
 *
 * act is SiLU, g / (1 + e^-g), or GELU, g (1 + erf(g / sqrt 2)) / 2.
 *
 * Activations, weights and gradients are bf16, sums fp32; act and act' are computed in
 * fp32, act(g) within 2^-24 (20 + 2 g g) of itself.  h is rounded once.
 * The backward pass rounds dg and du to bf16, as operands of its products;
 * where g and u were saved they have 24 bits (16 of mantissa).  Sums are added in an order that
 * the sizes alone fix: equal inputs give equal results bit for bit.  NaN and
 * infinities go where the formulas take them.
 *
 * Conventions as in ags.h: C linkage, ags_status results, arguments checked
 * on the host before any HIP call, then device pointers against their
 * allocations; the text of the last failed call on this thread from
 * ags_last_error(NULL); work goes on hip_stream and the call returns without
 * waiting.  There is no handle: the caller owns every buffer, workspaces
 * included (16-byte aligned), and orders calls that share one.  Outputs must
 * not overlap each other or the inputs (AGS_E_ARG).  A dtype argument is an
 * ags_dtype.
 */
#ifndef AGS_GLU_H
#define AGS_GLU_H

#include <stddef.h>
#include <stdint.h>

#include "ags.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { AGS_GLU_SILU = 0, AGS_GLU_GELU = 1 } ags_glu_act;

/* Both weights, laid out for the products: rows of `padded` = k rounded up to
 * 64 bf16 elements; 16 rows of gate, the same 16 of up, and so on, `lines` = 2
 * (n rounded up to 16) rows in all, padding zero.  They lie in panels of 32 rows
 * and 64 elements, each in one piece, row after row; panel (i, j) is the
 * (i padded / 64 + j)-th.  data: device memory of
 * ags_glu_bytes bytes, 16-byte aligned (NULL where that is 0). */
typedef struct {
    void *data;
    int64_t n, k;
} ags_glu_weight;

/* Bytes of a weight's data (host only).  AGS_E_LAYOUT where n or k exceeds
 * 2^20. */
ags_status ags_glu_bytes(int64_t n, int64_t k, size_t *out_bytes);

/* Lay out gate and up [n, k] (fp32 or bf16, row i at element i * stride). */
ags_status ags_glu_store(const void *d_gate, int64_t gate_stride, const void *d_up,
                         int64_t up_stride, int32_t dtype, const ags_glu_weight *w,
                         void *hip_stream);

/* h [rows][h_stride] of h_dtype from x [rows, k] (bf16; any alignment and
 * stride, but rows that start at multiples of 16 bytes and a k that is a
 * multiple of 64 save a copy).  d_saved: g and u for the backward
 * pass, 3 bytes each in the order of the weight's rows, 3 lines bytes a row of x
 * (the upper 16 bits of all of them, bf16 values cut off, then the next 8 of
 * each), 16-byte aligned; or NULL.  rows up to 2^30. */
ags_status ags_glu_forward_workspace(int64_t rows, int64_t n, int64_t k, size_t *out_bytes);
ags_status ags_glu_forward(const void *d_x, int64_t rows, int64_t x_stride,
                           const ags_glu_weight *w, int32_t act, void *d_h, int32_t h_dtype,
                           int64_t h_stride, void *d_saved, void *d_workspace,
                           size_t workspace_bytes, void *hip_stream);

/* Gradients for dh [rows][dh_stride] (bf16).  d_saved: what the forward pass
 * saved, or NULL: g and u are computed again from x.  dx [rows][dx_stride] is
 * bf16, or NULL where it is not wanted; d_dgate and d_dup [n][dw_stride] are of
 * dw_dtype, both or neither, added to what is there with accumulate = 1 (in
 * fp32, one rounding).  With no rows they are zero (or left, with
 * accumulate). */
ags_status ags_glu_backward_workspace(int64_t rows, int64_t n, int64_t k, size_t *out_bytes);
ags_status ags_glu_backward(const void *d_dh, int64_t dh_stride, const void *d_x, int64_t rows,
                            int64_t x_stride, const void *d_saved, const ags_glu_weight *w,
                            int32_t act, void *d_dx, int64_t dx_stride, void *d_dgate,
                            void *d_dup, int32_t dw_dtype, int64_t dw_stride, int32_t accumulate,
                            void *d_workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* AGS_GLU_H */
