/*
 * mi355lp -- log probabilities of given tokens over a large vocabulary, with the entropy and the most likely
 * alternatives, and the gradient of a loss on them, for AMD MI355X (gfx950).  Part of the same library as mi355conv.h.
 *
 * The policy-gradient trainer of the paper (Appendix B, the Softmax model) for policies whose actions are tokens: what
 * pg_softmax_bottom_diff does with the probabilities of a few actions, without ever writing the probabilities down.
 *
 * Semantics, for each row of logits x[0 .. vocab):
 *   z = scale x          log p_i = z_i - log sum_j exp z_j          H = -sum_i p_i log p_i
 *   logp       log p_token                                 (0 where the token counts for nothing: outside [0, vocab))
 *   entropy    H, in nats
 *   top        the `top` largest logits in descending order as (log p, index); equal logits (-0 and +0 among them) in ascending order of
 *              their indices, NaN above everything
 *   d_logits   scale (w (1[i = token] - p_i) - u p_i (log p_i + H)),   w = d_logp, u = d_entropy: the derivatives of the
 *              loss by logp and entropy; w counts as 0 where the token counts for nothing, u = 0 where d_entropy is NULL
 * A logit of -inf is a banned token: p_i = 0, no part in the entropy, d_logits 0 (but for w scale if it is the token itself,
 * whose logp is -inf).  A row of nothing but -inf has no distribution: p = 0 throughout, logp -inf, entropy 0,
 * alternatives -inf in ascending order of indices, no gradient but w scale at the token.  A NaN or +inf makes the row's results NaN
 * (the indices of the alternatives stay defined).
 *
 * Types and layouts: logits and d_logits in the descriptor's type (fp32, fp16, bf16), rows `stride` elements apart
 * (stride >= vocab where there is more than one row) and dense inside, on the element's own alignment; everything else is dense fp32 or int32:
 *   token int32 [rows]   logp, entropy, d_logp, d_entropy [rows]   stats [rows][4]   top_logp, top_token (int32) [rows][top]
 * stats is what lp_forward leaves for lp_backward (reference exponent, log2 of the sum, entropy, exponent factor): of the same logits, by
 * a descriptor of the same vocab, dtype and scale.  The entropy is NaN if that descriptor's is 0: a gradient through it is then NaN, one
 * without it as usual.
 * Sums, maxima and gradients are held in fp32; a gradient is rounded once, to nearest, as it is stored.
 * d_logits may be logits itself (same base and stride); no other output may overlap an input, the workspace or another output.
 *
 * The workspace is 16-byte aligned.  Ownership, execution and errors as in mi355conv.h: caller-owned device memory and workspace, enqueued on the caller's
 * hipStream_t without synchronising; a conv_status_t comes back, and argument errors are found before anything is enqueued.
 * Every call only enqueues kernels and may be captured.  Results do not depend on timing: equal calls give equal bits.
 * rows == 0 is a no-op.
 */
#ifndef MI355LP_H
#define MI355LP_H

#include "mi355conv.h"
#include "mi355dtype.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t rows;    /* >= 0 */
  int32_t vocab;   /* 1 .. 2^30 - 1 */
  int32_t dtype;   /* of logits and d_logits: MI355_F32, MI355_F16 or MI355_BF16 */
  int32_t top;     /* alternatives of lp_forward: 0 .. min(64, vocab) */
  int32_t entropy; /* 0 or 1: whether entropies, or gradients through them, are wanted */
  float scale;     /* 1 / temperature: 2^-60 .. 2^60 */
} lp_params_t;

typedef struct lp_desc lp_desc_t;

/* Validates p, picks kernels and sizes the workspace; touches no device.  *out is written only on success.
 * CONV_ESHAPE: vocab of 2^30 or more. */
int lp_desc_create(lp_desc_t** out, const lp_params_t* p);
int lp_desc_destroy(lp_desc_t* d);
/* Largest workspace any pass of this descriptor needs, in bytes (may be 0). */
int lp_desc_workspace_bytes(const lp_desc_t* d, size_t* bytes);
/* "forward=...;backward=...;forward_backward=..." -- the kernel variants chosen; owned by d. */
const char* lp_desc_kernel_names(const lp_desc_t* d);

/* entropy is NULL if the descriptor's is 0 and may be NULL otherwise (not wanted), as may stats.  token and logp may be
 * NULL together.  top_logp and top_token are NULL exactly when top == 0. */
int lp_forward(const lp_desc_t* d, const void* logits, int64_t stride, const int32_t* token, float* logp, float* entropy,
               float* stats, float* top_logp, int32_t* top_token, void* ws, size_t ws_bytes, void* hip_stream);
/* stats from lp_forward on the same logits, as above.  d_entropy is NULL if the descriptor's entropy is 0 and may be NULL otherwise. */
int lp_backward(const lp_desc_t* d, const void* logits, int64_t stride, const int32_t* token, const float* stats,
                const float* d_logp, const float* d_entropy, void* d_logits, int64_t d_stride, void* hip_stream);
/* Both at once, where the derivatives are known before the call; logp and entropy may be NULL (not wanted). */
int lp_forward_backward(const lp_desc_t* d, const void* logits, int64_t stride, const int32_t* token, const float* d_logp,
                        const float* d_entropy, float* logp, float* entropy, void* d_logits, int64_t d_stride, void* ws,
                        size_t ws_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif
