/*
 * mi355sm -- drawing tokens over a large vocabulary under a temperature, top-k, top-p and min-p from given uniform numbers, for AMD
 * MI355X (gfx950).  Part of the same library as mi355conv.h; mi355lp.h scores the tokens and has the gradients.
 *
 * Semantics, for each row of logits x[0 .. vocab), with its own scale (1 / temperature), k, p, q and u:
 *   w_i = exp(scale (x_i - max x));   the order of tokens is by descending x, equal logits (-0 and +0 among them) by ascending index
 *   top_k   keeps the first k of the order               (all of them where k <= 0 or k >= vocab)
 *   top_p   keeps the shortest beginning of the order whose weight is at least p times that of what top_k keeps, one token at
 *           least                                        (no limit where p >= 1)
 *   min_p   keeps what has w_i >= min(q, 1)              (no limit where q <= 0)
 *   token   of what all three keep, in the order of the indices, the first whose weight, with those before it, is more than u times the whole
 *           (the last one of any weight where none is, as with u = 1)
 *   logp    ln(w_token / weight of what is kept): the log probability that it was drawn with
 * Without top_k the tokens are the same for every order of the limits; with it, top_k comes first.  top_k = 1 is the most likely token.
 * A logit of -inf is a banned token and is never drawn.  A row of nothing but -inf has nothing to draw: token -1, logp -inf.  A row that holds a NaN or
 * +inf, or whose scale is not in [2^-60, 2^60], u not in [0, 1], p or q NaN, has token -1 and logp NaN.  (A token of -1 counts for
 * nothing in mi355lp.h.)
 * Weights and their sums are held in 64 bits: a token differs from the formula's only where u or p meets a border within some 2^-44 of
 * the whole (vocab 2^-62 of it in rows of more than 2^18 logits), or q a weight within 2^-44 of it.  A weight below some 2^-995 counts as 0.
 *
 * Types and layouts: logits in the descriptor's type (fp32, fp16, bf16), rows `stride` elements apart (stride >= vocab where there is more than one
 * row) and dense inside, on the element's own alignment; dense [rows]: u, scale, top_p, min_p, logp fp32, top_k, token int32.  scale, top_k, top_p
 * and min_p may be NULL each: 1, and no limit.  They are read by the kernels, so that a captured call can be replayed with others.
 * No output may overlap an input, the workspace or another output.
 *
 * The workspace is 16-byte aligned.  Ownership, execution and errors as in mi355conv.h: caller-owned device memory and workspace, enqueued on the
 * caller's hipStream_t without synchronising; a conv_status_t comes back, and argument errors are found before anything is enqueued.
 * Every call only enqueues kernels and may be captured.  Results do not depend on timing: equal calls give equal bits.
 * rows == 0 is a no-op.
 */
#ifndef MI355SM_H
#define MI355SM_H

#include "mi355conv.h"
#include "mi355dtype.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t rows;  /* >= 0 */
  int32_t vocab; /* 1 .. 2^30 - 1 */
  int32_t dtype; /* of the logits: MI355_F32, MI355_F16 or MI355_BF16 */
} sm_params_t;

typedef struct sm_desc sm_desc_t;

/* Validates p, picks kernels and sizes the workspace; touches no device.  *out is written only on success.
 * CONV_ESHAPE: vocab of 2^30 or more. */
int sm_desc_create(sm_desc_t** out, const sm_params_t* p);
int sm_desc_destroy(sm_desc_t* d);
/* Bytes of sm_sample's workspace (may be 0). */
int sm_desc_workspace_bytes(const sm_desc_t* d, size_t* bytes);
/* "sample=..." -- the kernel variants chosen; owned by d. */
const char* sm_desc_kernel_names(const sm_desc_t* d);

/* logp may be NULL (not wanted). */
int sm_sample(const sm_desc_t* d, const void* logits, int64_t stride, const float* u, const float* scale, const int32_t* top_k,
              const float* top_p, const float* min_p, int32_t* token, float* logp, void* ws, size_t ws_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
