/* gem_lm.h -- operators of a language model that asynchronous workers train with GEM (C
 * ABI, sm_103a): the layer that mixes time, the loss over a vocabulary, and the scoring of
 * what the model answers.
 *
 *   gem_glr_forward, gem_glr_backward     a gated linear recurrence over long sequences
 *   gem_distill                           the loss against a teacher's top logits, with its
 *                                         gradient
 *   gem_token_logp, gem_token_logp_grad   log probabilities of given tokens with entropy and
 *                                         the top alternatives, and their gradient
 *
 * They give the gradient of a worker's loss (Delta theta = -eta grad L(s_w), Algorithm 1 of
 * Hermans & Louppe, arXiv 1805.08469), which gem_commit then applies; the paper's own models
 * are those of gem_sim.h and gem_cnn.h, and it has no counterpart to these operators.
 *
 * Conventions shared by every call:
 *   - Return value: GEM_OK (0) or a negative gem_status.  Arguments are checked on the host;
 *     a call that fails a check launches nothing.  Calls hold no handle, allocate nothing and
 *     keep nothing of their data from one call for the next (only, for each kernel and device, that it may
 *     use the shared memory that it does, and how many of its clusters fit).
 *   - All pointers are device memory of the current device.  Work is asynchronous and ordered
 *     on `stream` (a cudaStream_t; NULL is the legacy default stream); the caller orders
 *     buffers that other streams use.  Calls can be captured into a CUDA graph.
 *   - Elements are fp32, bf16 or fp16 (gem_dtype), statistics and states fp32.  All arithmetic
 *     is fp32, rounded once when an output of 16 bits is stored; exponentials over rows, those of 16-bit
 *     gates and the gates' quotients are the GPU's approximations (2 units in the last place and what rounding
 *     the argument adds; a quotient 1).  Results do not depend on
 *     timing: sums are taken in an order that the sizes fix.
 *   - Strides and row pitches count elements.  Tensors need the alignment of their element
 *     type, no more (aligned rows are read with wider loads).
 *   - No kernel waits on another.  Blocks of a cluster of gem_glr_* wait for one another's maps for at
 *     most two seconds; where a wait ran out, every state and gradient that rests on what did not come, and
 *     all that later steps hand on, are NaN, resets or not.
 *   - Outputs overlap neither inputs nor one another except where a call says so.  A size of
 *     zero is valid and leaves nothing to do.
 */
#ifndef GEM_LM_H
#define GEM_LM_H

#include <stddef.h>
#include <stdint.h>

#include "gem.h"

#ifdef __cplusplus
extern "C" {
#endif

enum gem_dtype { GEM_F32 = 0, GEM_BF16 = 1, GEM_F16 = 2 };

/* A [B][T][D] tensor whose D channels lie side by side: element (b, t, d) at data[b * stride_b
 * + t * stride_t + d].  Views such as the halves of one projection's [B][T][2 D] output, or
 * [T][B][D] storage, are given by their strides. */
typedef struct {
  void* data;
  int64_t stride_b, stride_t;
} gem_seq_t;

/* Gated linear recurrence.  With the gate a = sigmoid(f), elementwise over channels,
 *
 *   GEM_GLR_LERP   h_t = a_t h_{t-1} + (1 - a_t) x_t
 *   GEM_GLR_ADD    h_t = a_t h_{t-1} + x_t
 *
 * from h_{-1} = h0.  f below -80 counts as -80 (a = 2e-35), so that an infinite state, or gradient, stays
 * infinite until a reset. */
enum gem_glr_form { GEM_GLR_LERP = 0, GEM_GLR_ADD = 1 };

/* Steps between the states that gem_glr_forward saves for gem_glr_backward. */
#define GEM_GLR_CHUNK 16

/* Floats of the `saved` buffer, [B][ceil(T / GEM_GLR_CHUNK)][D]; -1 for a negative size. */
int64_t gem_glr_saved_count(int64_t B, int64_t T, int64_t D);

/* The recurrence over x and f (B sequences of T steps and D channels, of type dtype) into h.
 *   h0 [B][D] fp32, NULL: zeros.
 *   lengths [B] int32, NULL: all T.  Sequence b has lengths[b] steps (clipped to 0..T): past
 *     them x and f are not used, h is 0 and the state stays.
 *   reset [B][T] bytes, NULL: none.  Where it is not 0, the state before the step counts as
 *     0, whatever it holds (packed documents).
 *   h_last [B][D] fp32, may be NULL and may be h0: the state after the last step, so that a
 *     call can go on where another ended; serving is a call with T = 1 for each token.
 *   saved, may be NULL: gem_glr_saved_count floats, the state before steps 0, 16, 32, ... for
 *     gem_glr_backward (a rounded h would cost the gate's gradient its precision). */
int gem_glr_forward(int dtype, int form, int64_t B, int64_t T, int64_t D, const gem_seq_t* x,
                    const gem_seq_t* f, const float* h0, const int32_t* lengths,
                    const uint8_t* reset, const gem_seq_t* h, float* h_last, float* saved,
                    void* stream);

/* Gradients of the recurrence: dh is the gradient with respect to h, dh_last [B][D] fp32 (NULL:
 * zeros) that with respect to h_last; x, f, lengths, reset and form are those of the forward
 * call and saved is what it saved.  With g_t = dh_t + a_{t+1} g_{t+1}, where a counts as 0 at a
 * reset and g of the last step also receives dh_last,
 *
 *   GEM_GLR_LERP   dx_t = (1 - a_t) g_t   df_t = a_t (1 - a_t) g_t (h_{t-1} - x_t)
 *   GEM_GLR_ADD    dx_t = g_t             df_t = a_t (1 - a_t) g_t h_{t-1}
 *
 * and dh0 [B][D] fp32 (may be NULL, may be dh_last) = a_0 g_0.  Past lengths[b] dh is not used
 * and dx and df are 0. */
int gem_glr_backward(int dtype, int form, int64_t B, int64_t T, int64_t D, const gem_seq_t* x,
                     const gem_seq_t* f, const int32_t* lengths, const uint8_t* reset,
                     const float* saved, const gem_seq_t* dh, const float* dh_last,
                     const gem_seq_t* dx, const gem_seq_t* df, float* dh0, void* stream);

/* Most top entries of a row (gem_distill, gem_token_logp). */
#define GEM_TOP_MAX 256

/* Distillation from a teacher's top logits: for each of N rows of V student logits (row n at
 * logits + n * ld) the loss, and its gradient, against K entries of the teacher,
 *
 *   L = (1 - alpha) tau^2 [sum_k q_k (log q_k - log p_k) + q_rest (log q_rest - log p_rest)]
 *       + alpha (-log p1_label)
 *
 * with p = softmax(logits / tau), p1 = softmax(logits), tau = temperature.
 *   top_idx, top_logits [N][K]: the teacher's entries; an index outside [0, V) or a logit of
 *     -inf is an entry that is absent.  Entries with the same index add up in the gradient; the
 *     loss has a term for each.  A row without entries has no teacher: its first term is 0.
 *   teacher_lse [N] fp32.  NULL: q = softmax of the row's K entries / tau, q_rest = 0.  Else
 *     q_k = exp(top_logits_k / tau - teacher_lse), where teacher_lse is the teacher's
 *     log-sum-exp of all logits / tau (its rounding is q's relative error, |teacher_lse| 2^-24: give
 *     logits without an offset), and q_rest = max(0, 1 - sum q) is compared with p_rest,
 *     the student's mass outside the entries, as one class; where p_rest is 0 that class is
 *     left out.
 *   labels [N] int32 (required when alpha > 0, not read otherwise): < 0: the row has no label
 *     and no second term; >= V: the row's loss and gradient are NaN.
 *   alpha = 1: labels only; the teacher's arrays are checked, but not read.
 *   row_scale [N] fp32, NULL: ones.  The gradient of row n is multiplied by row_scale[n]
 *     (1 / rows for a mean, a loss scale, a mask).  A row whose scale is 0 is not read: its loss
 *     is 0 and its gradient zeros.
 *   loss [N] fp32: L of each row (not multiplied by row_scale).
 *   grad (row n at grad + n * grad_ld, type dtype), may be NULL and may be logits with grad_ld
 *     = ld: row_scale[n] dL/dlogits.
 * A student logit of -inf has p = 0: its gradient is that of the formula, and the loss is +inf
 * where the teacher gives it mass.  A logit of NaN or +inf makes its row's loss and gradient NaN.
 * The first term's rounding, some 2^-20, is multiplied by tau^2 in the loss and by tau (of p and q)
 * in the gradient.  Requires 0 <= K <= GEM_TOP_MAX, 1e-20 <=
 * temperature <= 1e20, 0 <= alpha <= 1, 1 <= V <= 2^30, N <= 2^27,
 * ld >= V (or 0: one row of logits for all), grad_ld >= V. */
int gem_distill(int dtype, int64_t N, int64_t V, const void* logits, int64_t ld, int K,
                const int32_t* top_idx, const float* top_logits, const float* teacher_lse,
                const int32_t* labels, const float* row_scale, float temperature, float alpha,
                float* loss, void* grad, int64_t grad_ld, void* stream);

/* Log probabilities: for each of N rows of V logits, with p = softmax(logits / temperature),
 *   logp [N] (may be NULL; else tokens [N] int32 is required): log p of tokens[n]; 0 where
 *     tokens[n] < 0 (no token), NaN where tokens[n] >= V.
 *   entropy [N] (may be NULL): -sum p log p; terms with p = 0 count as 0.
 *   lse [N] (may be NULL): log-sum-exp of logits / temperature (gem_token_logp_grad reads it;
 *     gem_distill takes a teacher's).
 *   top_idx, top_logp [N][K] (K = 0: not written): the K largest logits' indices, descending,
 *     equal ones by ascending index, and their log p.  NaN orders above everything.
 * A row whose logits are all -inf has lse -inf, entropy 0 and every log p -inf; in a row with a
 * NaN or +inf logit every value is NaN (logp stays 0 where there is no token; the indices are those of the
 * order above).  Requires 0
 * <= K <= min(V, GEM_TOP_MAX), 1e-20 <= temperature <= 1e20, V >= 1, ld >= V or 0. */
int gem_token_logp(int dtype, int64_t N, int64_t V, const void* logits, int64_t ld,
                   const int32_t* tokens, float temperature, int K, float* logp,
                   float* entropy, float* lse, int32_t* top_idx, float* top_logp, void* stream);

/* Gradient of logp and entropy of gem_token_logp with respect to the logits,
 *
 *   grad_j = (dlogp ([j = token] - p_j) - dentropy p_j (log p_j + entropy)) / temperature
 *
 * with dlogp [N] and dentropy [N] (either may be NULL: zeros), and lse [N] and, with dentropy,
 * entropy [N] as that call wrote them.  (In a row whose |lse| is 128 or more, where the rounding of lse would
 * show in p, maximum and sum are found again from the logits, which takes longer.)  A row without a
 * token has no first term; one with a token >= V gets NaN (both as dlogp is given).  grad may be
 * logits with grad_ld = ld. */
int gem_token_logp_grad(int dtype, int64_t N, int64_t V, const void* logits, int64_t ld,
                        const int32_t* tokens, float temperature, const float* lse,
                        const float* entropy, const float* dlogp, const float* dentropy,
                        void* grad, int64_t grad_ld, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GEM_LM_H */
