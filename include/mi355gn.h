/*
 * mi355gn -- the norm over all of a network's gradients, and clipping by it, for AMD MI355X (gfx950).  Part of the same
 * library as mi355conv.h.
 *
 *   norm = sqrt(sum over all tensors and elements of g^2)
 *   out  = factor g,   factor = limit / norm where norm > limit, else 1
 *
 * the step that Caffe's solvers take between accumulating parameter diffs (the paper's Appendix A and B) and applying them.
 * Squares and sums are held in fp64, and no square of a finite gradient overflows or vanishes.  The factor is held in fp64 for
 * fp64 tensors (below 2^-1022 with the bits that such numbers have) and rounded to 24 bits for the others, of any size, also
 * below fp32's normal numbers; their product with it is rounded to fp32 and once more to the tensor's type.  A norm of +inf (an
 * infinite gradient, or fp64 gradients whose norm itself is beyond fp64) has the factor 0, so an infinite gradient becomes NaN
 * and the others 0; one that is NaN compares as not above the limit, and the gradients stay as they are.
 *
 * Layouts: tensor i is counts[i] contiguous elements of dtypes[i] in DEVICE memory, on the element's own alignment; the arrays of
 * pointers are HOST memory and are read before the call returns.  outs[i] may be grads[i] itself (a factor of 1 then
 * leaves it untouched); otherwise outputs must not overlap inputs.  No tensor
 * may share memory with another one of the list.  Tensors that follow each other in memory, as views of one flat
 * buffer do, are taken together; the result does not depend on it but for the order of the sums.
 *
 * The workspace is 16-byte aligned.  Ownership, execution and errors as in mi355conv.h.  Every call only enqueues kernels (a pass each for
 * the sum and the product, of one launch for up to 96 runs of tensors that follow each other, and one between them for many partial
 * sums) and may be captured.  Equal calls give equal bits.
 */
#ifndef MI355GN_H
#define MI355GN_H

#include "mi355conv.h"
#include "mi355dtype.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t tensors;       /* 0 .. 2^18 */
  const int64_t* counts; /* >= 0 each, below 2^40 in all; read by gn_desc_create only */
  const int32_t* dtypes; /* MI355_F32, MI355_F16, MI355_BF16 or MI355_F64 each; read by gn_desc_create only */
} gn_params_t;

typedef struct gn_desc gn_desc_t;

/* Touches no device.  *out is written only on success.  CONV_ESHAPE: too many tensors or elements. */
int gn_desc_create(gn_desc_t** out, const gn_params_t* p);
int gn_desc_destroy(gn_desc_t* d);
int gn_desc_workspace_bytes(const gn_desc_t* d, size_t* bytes);
/* "clip=gn_sum+gn_scale(T=tensors)"; owned by d. */
const char* gn_desc_kernel_names(const gn_desc_t* d);

/* limit >= 0, +inf for the norm alone.  norm: one fp32 value in device memory, or NULL.  A tensor of no elements may be NULL. */
int gn_clip(const gn_desc_t* d, const void* const* grads, double limit, void* const* outs, float* norm, void* ws,
            size_t ws_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
