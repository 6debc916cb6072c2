/*
 * mi355q4 -- the InnerProduct layer's forward pass on weights of 4 bits with group scales, for AMD MI355X (gfx950).  Part of
 * the same library as mi355conv.h; mi355ip.h has the layer on fp32 weights, its gradients included.
 *
 * Semantics (as ip_forward, with w[o][i] = scales[o][i / group] value(codes[o][i])):
 *   z[n][o] = bias[o] + sum_i x[n][i] w[o][i];   y = relu ? max(z, 0) : z
 *   value(c) for c = 0 .. 15:  0 0.5 1 1.5 2 3 4 6  -0 -0.5 -1 -1.5 -2 -3 -4 -6     (one sign, two exponent, one mantissa bit)
 * Products with x are exact and summed in fp32 inside each group, the groups' sums times their scales in fp32; fp32 x takes part with all
 * of its 24 bits, but for those below 2^-133 (of inputs below 2^-110).  One rounding to y's type at the end.  A group's sum is taken
 * before its scale: it stays in fp32's range where |x| <= 2^118, and may be infinite or NaN beyond, whatever the scale.
 *
 * Made for batches of up to 64 rows, which read the weights once.  Larger ones are taken 64 rows at a time.
 *
 * Layouts, dense row-major DEVICE memory:
 *   x [m][k], bias [num_output], y [m][num_output]: the descriptor's type (fp32, fp16, bf16), on the element's own alignment
 *   codes : uint8 [num_output][ceil(k / 2)], input 2b in byte b's low half, 2b + 1 in its high half (ignored beyond k)
 *   scales: bf16 [num_output][ceil(k / group)]
 *   packed: q4_desc_packed_bytes bytes, 16-byte aligned: what q4_pack makes of codes and scales once, and q4_forward reads
 * The packed form depends on k, num_output and group alone: descriptors that agree in these share it.
 * Outputs must not overlap inputs or the workspace.
 *
 * The workspace is 16-byte aligned.  Ownership, execution and errors as in mi355conv.h.  Every call only enqueues kernels and may be
 * captured.  Equal calls give equal bits.  m may be 0: q4_forward is then a no-op.
 */
#ifndef MI355Q4_H
#define MI355Q4_H

#include "mi355conv.h"
#include "mi355dtype.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t m;          /* rows of the bottom blob, >= 0 */
  int32_t k;          /* inputs per row, >= 1 */
  int32_t num_output; /* >= 1 */
  int32_t dtype;      /* of x, bias and y: MI355_F32, MI355_F16 or MI355_BF16 */
  int32_t group;      /* inputs that share a scale: 32, 64 or 128 */
  int32_t bias_term;  /* 0 or 1 */
  int32_t relu;       /* 0 or 1 */
} q4_params_t;

typedef struct q4_desc q4_desc_t;

/* Touches no device.  *out is written only on success.  CONV_ESHAPE: 2^30 or more elements of x, w or y. */
int q4_desc_create(q4_desc_t** out, const q4_params_t* p);
int q4_desc_destroy(q4_desc_t* d);
/* Bytes of q4_forward's workspace (may be 0), and of the packed weights. */
int q4_desc_workspace_bytes(const q4_desc_t* d, size_t* bytes);
int q4_desc_packed_bytes(const q4_desc_t* d, size_t* bytes);
/* "fwd=..." -- the kernel variant chosen; owned by d. */
const char* q4_desc_kernel_names(const q4_desc_t* d);

int q4_pack(const q4_desc_t* d, const uint8_t* codes, const uint16_t* scales, void* packed, void* hip_stream);
/* bias must be NULL exactly when bias_term == 0. */
int q4_forward(const q4_desc_t* d, const void* x, const void* packed, const void* bias, void* y, void* ws, size_t ws_bytes,
               void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
