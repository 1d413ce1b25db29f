/*
 * libags orthogonalised updates: matrices brought near the nearest
 * orthogonal one by Newton-Schulz products, and the optimizer step made of it
 * (Muon), for the matrices of the flat buffers whose other layers AGS (ags.h)
 * updates.
 *
 * Orthogonalising U [rows, cols]: X = U / (|U| + eps), |U| the root of the
 * sum of squares, and then a number of steps
 *
 *   A = X X' (or X' X, whichever is smaller),  X <- a X + (b A + c A A) X
 *
 * with the step's a, b, c (X (b A + c A A) for X' X): singular values go the
 * way of s -> a s + b s^3 + c s^5.  The usual 3.4445, -4.7750, 2.0315 bring
 * those above 0.003 between 0.68 and 1.2 in five steps.
 *
 * The step, for the mean g of the K replica gradients:
 *
 *   m <- momentum m + g
 *   U = g + momentum m  (nesterov)  or  m
 *   w <- w (1 - lr weight_decay) - lr scale X
 *
 * X is held in fp32, norms are summed in fp64.  The products' operands are
 * rounded to fp16, scaled by powers of two, with fp32 sums: X carries no
 * rounding from step to step, whose error the steps would multiply by up to
 * a each; after five of the usual steps the result is off by 0.03 to 0.3 % of its
 * norm whatever the singular values (in bf16 throughout: up to 40 %), up to 1 %
 * where all but a few rows or columns are zero, as the roundings of few numbers do
 * not average out; after more, by up to 2 %.  Singular values that are zero take part
 * as those roundings: they stay below 1 % through eight of the usual steps, and from
 * about twelve on come out like any others.
 *
 * With a side of up to 16 the steps run in 64 bits on U U' alone, X = Q U is rounded to
 * fp32 once, and singular values that are zero stay zero.  Where the steps multiply
 * small ones by more than 2^18 in all (eleven usual steps), those below 2^-23 of |U|
 * count as zero.
 * Sums are added in an order that the sizes alone fix: equal inputs give equal
 * results bit for bit.
 * A NaN or an infinity makes its matrix NaN, no other; a zero matrix stays zero.
 *
 * Conventions as in ags.h: C linkage, ags_status results, arguments checked
 * on the host before any HIP call, then device pointers against their
 * allocations; the text of the last failed call on this thread from
 * ags_last_error(NULL); work goes on hip_stream and the call returns without
 * waiting.  A handle's calls share its workspace and are ordered as ags.h
 * describes (a call on another stream than the last one waits for it by an
 * event, except while a stream captures a graph); one thread at a time.  Graphs
 * that captured a handle's steps use its workspace too: their replays must not
 * overlap one another, nor the handle's other calls.
 */
#ifndef AGS_MUON_H
#define AGS_MUON_H

#include <stddef.h>
#include <stdint.h>

#include "ags.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AGS_MUON_MAX_STEPS 32

/* The steps' coefficients.  They must keep singular values of up to 1 below
 * 1.41, but for the last step's, and b s^2 + c s^4 below 3.99, the ranges that
 * fp16 operands are scaled for, with room for the operands' roundings: 5 |b| s^2 +
 * 8 |c| s^4 times s 2^-11 a step, s the largest (AGS_E_ARG). */
typedef struct {
    int32_t steps;          /* 1 .. AGS_MUON_MAX_STEPS                   */
    int32_t reserved;       /* must be 0                                 */
    const double *abc;      /* host [steps][3], read before the call returns */
    double eps;             /* >= 0; the usual value is 1e-7             */
} ags_muon_schedule;

/* Workspace (16-byte aligned) of ags_muon_orthogonalize (host only).
 * AGS_E_LAYOUT where rows or cols exceed 2^20, a matrix 2^31 elements, or the
 * batch 2^20 matrices. */
ags_status ags_muon_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols,
                                            size_t *out_bytes);

/* Each of `batch` matrices x [rows, cols] (of dtype, an ags_dtype; matrix i at
 * element i * x_batch_stride, its row j x_stride elements each) to out, of
 * out_dtype.  Nothing overlaps the output. */
ags_status ags_muon_orthogonalize(const void *d_x, int32_t dtype, int64_t batch, int64_t rows,
                                  int64_t cols, int64_t x_batch_stride, int64_t x_stride,
                                  const ags_muon_schedule *schedule, void *d_out, int32_t out_dtype,
                                  int64_t out_batch_stride, int64_t out_stride, void *d_workspace,
                                  size_t workspace_bytes, void *hip_stream);

/* A matrix of the flat buffers, its rows one after the other from element
 * `offset`, a multiple of AGS_ALIGN_ELEMS. */
typedef struct {
    int64_t offset;
    int64_t rows, cols;     /* >= 1                                      */
    double scale;           /* of its update, finite and >= 0            */
} ags_muon_matrix;

typedef struct {
    int32_t n_matrices;     /* >= 0                                      */
    int32_t K;              /* replicas, >= 1                            */
    const ags_muon_matrix *matrices; /* host array, copied at init; no two overlap */
    int64_t n_flat;         /* elements of w, m and a replica            */
    int32_t grad_dtype;     /* ags_dtype                                 */
    int32_t nesterov;       /* 0 or 1                                    */
    double lr;              /* finite, >= 0                              */
    double momentum;        /* 0 <= momentum < 1                         */
    double weight_decay;    /* finite, >= 0                              */
    ags_muon_schedule schedule;
} ags_muon_config;

typedef struct ags_muon_handle ags_muon_handle;

/* Bytes of device workspace ags_muon_init would allocate (host only): 8 an element of a
 * matrix, its rows padded to a multiple of 64, and 4 an element of its shorter side squared,
 * padded alike; for one with a side of up to 16 4 an element and 2048 for each
 * 128 of the longer side, 512 KiB at most; and tables of 16 bytes for each
 * block of a launch. */
ags_status ags_muon_workspace_bytes(const ags_muon_config *cfg, size_t *out_bytes);

/* A handle for w and m (device fp32 [n_flat], 16-byte aligned) on the current
 * device, which the steps update in place: the elements of the matrices, and
 * no others.  AGS_E_NOMEM as for ags_init. */
ags_status ags_muon_init(const ags_muon_config *cfg, float *d_w, float *d_m, void *hip_stream,
                         ags_muon_handle **out);

/* One step for the replica gradients d_grads [K][replica_stride], as for
 * ags_step. */
ags_status ags_muon_step(ags_muon_handle *h, const void *d_grads, int64_t replica_stride,
                         void *hip_stream);

/* The learning rate of the steps that run after this call, as ags_set_lr:
 * written on the handle's last stream, in force for eager steps and replayed
 * ones. */
ags_status ags_muon_set_lr(ags_muon_handle *h, double lr);

/* Free the handle and its workspace (waits for its last stream).  NULL is a
 * no-op. */
void ags_muon_destroy(ags_muon_handle *h);

#ifdef __cplusplus
}
#endif

#endif /* AGS_MUON_H */
