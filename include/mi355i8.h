/*
 * mi355i8 -- the InnerProduct layer in 8-bit integers with a scale for each row and each output, and its gradients from activations
 * kept in 8 bits, for AMD MI355X (gfx950).  Part of the same library as mi355conv.h; mi355ip.h has the layer on fp32 weights.
 *
 * A row r of numbers in 8 bits is whole numbers c_i in [-127, 127] and a scale s, and stands for s c_i:
 *   s    the smallest number of 8 significant bits with 127 s >= max |r_i|, at least 2^-126 (it is a bf16 number, held in fp32)
 *   c_i  the whole number nearest r_i / s, the even one of two
 * A row that holds a NaN or an infinity has the scale NaN and stands for NaN throughout.
 *
 * Semantics, with x ~ s_n c[n][i] and w ~ t_o v[o][i]:
 *   forward          z[n][o] = bias[o] + s_n t_o sum_i c[n][i] v[o][i];   y = relu ? max(z, 0) : z   (a NaN z is 0 then, as in mi355ip.h)
 *   backward filter  dw[o][i] = beta dw[o][i] + sum_n dz[n][o] s_n c[n][i];   db[o] = beta db[o] + sum_n dz[n][o]
 *   backward data    dx[n][i] = sum_o dz[n][o] t_o v[o][i]
 * The forward sum is exact in 32-bit integers; scales, bias and the rounding to y's type follow in fp32.  The gradients are those of the layer on
 * the rows and weights as they stand in 8 bits, the rounding to them counted as none.  dz s_n and dz t_o take part with all their bits for
 * bf16 dz and with 24 for fp16 and fp32 (but for bits below 2^-133), and products with the codes are exact; sums are fp32.  A dz whose product with a scale is 2^127 or
 * more gives results that are not finite.  dz is the top gradient after the ReLU's, as in mi355ip.h.  beta is 0 (overwrite) or 1 (accumulate).
 *
 * The codes and scales that i8_forward leaves are all of x that i8_backward_filter needs: the activations of a training step are kept in a
 * quarter of fp32's bytes.
 *
 * Layouts, row-major DEVICE memory:
 *   x, dx [m][k]   w [num_output][k]   y, dz [m][num_output]   bias [num_output]: the descriptor's type (fp32, fp16, bf16), dense, on the element's own
 *       alignment
 *   codes int8 [m][row], w_codes int8 [num_output][row]: row = i8_desc_row_bytes, k rounded up to 128; 0 beyond k; 16-byte aligned
 *   scale fp32 [m], w_scale fp32 [num_output]      dw fp32 [num_output][k]      db fp32 [num_output]
 * Outputs must not overlap inputs, the workspace or another output.
 *
 * The workspace is 16-byte aligned.  Ownership, execution and errors as in mi355conv.h.  Every call only enqueues kernels and may be
 * captured.  Equal calls give equal bits.  m may be 0: forward, quantise and backward data are then no-ops, and backward filter leaves beta
 * times what was there.
 */
#ifndef MI355I8_H
#define MI355I8_H

#include "mi355conv.h"
#include "mi355dtype.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t m;          /* rows of the bottom blob, >= 0 */
  int32_t k;          /* inputs per row, 1 .. 133120: 127^2 times as many fit 32 bits */
  int32_t num_output; /* >= 1 */
  int32_t dtype;      /* of x, w, bias, y, dz and dx: MI355_F32, MI355_F16 or MI355_BF16 */
  int32_t bias_term;  /* 0 or 1 */
  int32_t relu;       /* 0 or 1 */
} i8_params_t;

typedef struct i8_desc i8_desc_t;

/* Touches no device.  *out is written only on success.  CONV_ESHAPE: 2^30 or more elements of x, w or y, or more than 133120 inputs. */
int i8_desc_create(i8_desc_t** out, const i8_params_t* p);
int i8_desc_destroy(i8_desc_t* d);
/* Largest workspace any pass of this descriptor needs (may be 0), and the bytes of a row of codes. */
int i8_desc_workspace_bytes(const i8_desc_t* d, size_t* bytes);
int i8_desc_row_bytes(const i8_desc_t* d, size_t* bytes);
/* "fwd=...;bwd_filter=...;bwd_data=..." -- the kernel variants chosen; owned by d. */
const char* i8_desc_kernel_names(const i8_desc_t* d);

/* Weights, and rows of x, to 8 bits. */
int i8_pack(const i8_desc_t* d, const void* w, int8_t* w_codes, float* w_scale, void* hip_stream);
int i8_quantise(const i8_desc_t* d, const void* x, int8_t* codes, float* scale, void* hip_stream);
/* Writes codes and scale as i8_quantise does, and y; where x is NULL it takes them as i8_quantise has left them.  bias must be NULL exactly when
 * bias_term == 0. */
int i8_forward(const i8_desc_t* d, const void* x, const int8_t* w_codes, const float* w_scale, const void* bias, void* y,
               int8_t* codes, float* scale, void* ws, size_t ws_bytes, void* hip_stream);
/* db may be NULL (not wanted), and is when bias_term == 0. */
int i8_backward_filter(const i8_desc_t* d, const int8_t* codes, const float* scale, const void* dz, float* dw, float* db, float beta,
                       void* ws, size_t ws_bytes, void* hip_stream);
int i8_backward_data(const i8_desc_t* d, const int8_t* w_codes, const float* w_scale, const void* dz, void* dx, void* ws,
                     size_t ws_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
