/*
 * libags gradient clipping: the norm of many gradient tensors and their
 * scaling to a bound, in the same library as the AGS step.  In
 * data-parallel training each worker clips its gradient before the average
 * (Tula, arXiv 2603.18112, Eq. (1c)), so the calls here take gradients as a
 * backward pass leaves them, many tensors of one or two types, and can
 * write them where ags_step reads them: the rows of the replica stack.
 *
 * For the elements x of group g's segments:
 *
 *   N_g = (sum x^2)^(1/2)  or  sum |x|  or  max |x|
 *   c_g = min(1, max_norm / (N_g + eps))
 *   out = x c_g
 *
 * One group is the global norm; a group for each replica clips each
 * worker's gradient by itself; a group for each layer clips layer by layer.
 * Sums are kept in fp64 and added in an order that the configuration alone
 * fixes, not the tensors' addresses: equal gradients give equal norms bit for
 * bit, and no fp32 value over- or underflows its square.  c_g is
 * rounded to fp32, the product x c_g to fp32, and that to a bf16 output's
 * type.  (A c_g below 2^-100 has 24 bits all the same: it multiplies in two
 * steps, the second by a power of two.)
 *
 * A NaN among a group's elements makes N_g and c_g NaN (so every output of
 * the group); an infinite one makes N_g infinite and c_g zero (finite
 * elements become 0, infinite ones NaN).  Nothing is hidden: the caller
 * reads N_g.  A group without elements has N_g = 0.
 *
 * Conventions as in ags.h: C linkage, ags_status results, nothing changed on
 * an argument error, the text of the last failed call on this thread from
 * ags_last_error(NULL); work goes on hip_stream and the call returns
 * without waiting; a handle's calls share its workspace and are ordered as
 * ags.h describes (a call on another stream than the last one waits for it
 * by an event, except while a stream captures a graph); one thread at a
 * time.
 */
#ifndef AGS_CLIP_H
#define AGS_CLIP_H

#include <stddef.h>
#include <stdint.h>

#include "ags.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { AGS_CLIP_L2 = 0, AGS_CLIP_L1 = 1, AGS_CLIP_MAX = 2 } ags_clip_kind;

/* One run of consecutive elements: [in_offset, in_offset + numel) of input
 * tensor in_base, which go to out_offset of output tensor out_base.  numel
 * may be 0.  out_base and out_offset are not read in a configuration
 * without outputs. */
typedef struct {
    int64_t numel;
    int64_t in_offset;
    int64_t out_offset;
    int32_t in_base;
    int32_t out_base;
    int32_t group;
    int32_t reserved; /* must be 0 */
} ags_clip_segment;

typedef struct {
    int32_t n_segments;
    const ags_clip_segment *segments; /* host array, copied at init          */
    int32_t n_in;                     /* input tensors, >= 0                 */
    const int32_t *in_dtypes;         /* ags_dtype of each (host, copied)    */
    int32_t n_out;                    /* output tensors; 0: in place only    */
    const int32_t *out_dtypes;
    int32_t n_groups;                 /* 1 .. 2^30                           */
    int32_t kind;                     /* ags_clip_kind                       */
    double eps;                       /* >= 0; the usual value is 1e-6       */
} ags_clip_config;

typedef struct ags_clip_handle ags_clip_handle;

/* Bytes of device workspace ags_clip_init would allocate (host only). */
ags_status ags_clip_workspace_bytes(const ags_clip_config *cfg, size_t *out_bytes);

/* A handle for gradients of these sizes, types and groups on the current
 * device.  It holds tables of sizes and a workspace, no addresses: each call
 * names its tensors.  Output segments of one tensor must not overlap
 * (AGS_E_LAYOUT).  AGS_E_NOMEM as for ags_init. */
ags_status ags_clip_init(const ags_clip_config *cfg, void *hip_stream, ags_clip_handle **out);

/* N_g of every group to d_norms (device fp32 [n_groups]).  d_in: host array
 * of n_in device pointers, aligned to their element type, read before the
 * call returns; a tensor no segment uses may be NULL. */
ags_status ags_clip_norm(ags_clip_handle *h, const void *const *d_in, float *d_norms,
                         void *hip_stream);

/* N_g to d_norms and the scaled elements to d_out (host array of n_out
 * device pointers), or in place with d_out NULL, where a group whose c_g is
 * 1 is left unwritten.  max_norm > 0.  Outputs must not overlap each other,
 * the inputs or d_norms (AGS_E_ARG); in place, input segments must not
 * overlap each other. */
ags_status ags_clip_apply(ags_clip_handle *h, const void *const *d_in, void *const *d_out,
                          double max_norm, float *d_norms, void *hip_stream);

/* Free the handle and its workspace (waits for its last stream).  NULL is a
 * no-op. */
void ags_clip_destroy(ags_clip_handle *h);

#ifdef __cplusplus
}
#endif

#endif /* AGS_CLIP_H */
