/* gem_lm.h -- operators of a language model that asynchronous workers train with GEM (C
 * ABI, sm_103a): the embedding, the layers that mix time, the losses over a vocabulary, and the
 * scoring of what the model answers.
 *
 *   gem_embed, gem_embed_grad             rows of the embedding table for tokens, and the
 *                                         table's gradient
 *   gem_conv_forward, gem_conv_backward   a short causal convolution of each channel
 *   gem_ssm_forward, gem_ssm_backward     a selective state space scan
 *   gem_glr_forward, gem_glr_backward     a gated linear recurrence over long sequences
 *   gem_distill                           the loss against a teacher's top logits, with its
 *                                         gradient
 *   gem_policy                            the clipped policy loss of sampled tokens with a KL
 *                                         term and an entropy bonus, with its gradient
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
 *     use the shared memory that it does, and how many of its clusters fit).  A workspace is the caller's; what it
 *     holds before and after a call does not matter, and calls that may run at once need one each.
 *   - All pointers are device memory of the current device.  Work is asynchronous and ordered
 *     on `stream` (a cudaStream_t; NULL is the legacy default stream); the caller orders
 *     buffers that other streams use.  Calls can be captured into a CUDA graph.
 *   - Elements are fp32, bf16 or fp16 (gem_dtype), statistics and states fp32.  All arithmetic
 *     is fp32, rounded once when an output of 16 bits is stored; exponentials over rows, those of 16-bit
 *     gates, all of the convolution's and the scan's (gates, softplus, decays) and the gates' quotients are the
 *     GPU's approximations (2 units in the last place and what rounding the argument adds, so that the softplus of v
 *     below -10 is off by |v| 2^-24 of itself; a quotient 1), 0 below 2^-126.  Results do not depend on
 *     timing: sums are taken in an order that the sizes fix (the embedding gradient's: the tokens).
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

/* Clipped policy loss: for each of N rows of V logits, with p = softmax(logits / temperature),
 * logp = log p of the row's token, H = -sum p log p and r = exp(logp - old_logp), the loss
 *
 *   L = max(-r A, -min(max(r, 1 - clip_low), 1 + clip_high) A) + kl (exp(d) - d - 1) - bonus H,
 *       d = ref_logp - logp,
 *
 * and its gradient, with D = -r A where the first of the two terms is the larger or equal one, else 0, less
 * kl (exp(d) - 1),
 *
 *   dL/dlogits_j = (D ([j = token] - p_j) + bonus p_j (log p_j + H)) / temperature.
 *
 *   tokens [N] int32: the sampled tokens; < 0: the row has none, its loss is 0 and its gradient zeros;
 *     >= V: its loss, logp and gradient are NaN.
 *   old_logp [N] fp32: the tokens' log probabilities when they were sampled (gem_token_logp);
 *     advantage [N] fp32: A of each; ref_logp [N] fp32 (required when kl > 0, not read otherwise):
 *     those under the reference model.
 *   row_scale [N] fp32, NULL: ones.  The gradient of row n is multiplied by row_scale[n].  A row whose
 *     scale is 0 (a prompt's, padding) is not read: its loss, logp and entropy are 0, its gradient zeros.
 *   loss [N] fp32: L of each row (not multiplied by row_scale); logp, entropy [N] fp32, may be NULL: logp and H
 *     (0 in a row without a token).
 *   grad (row n at grad + n * grad_ld, type dtype), may be NULL and may be logits with grad_ld =
 *     ld: row_scale[n] dL/dlogits.
 * A logit of -inf has p = 0, and no gradient unless it is the token's; a logit of NaN or +inf, or a row of -inf
 * alone, makes its row's loss and gradient NaN; so may a KL term past fp32 (d above 88, or a token without any
 * probability).  Requires 0 <= clip_low <= 1, 0 <= clip_high, kl and bonus finite and
 * kl >= 0, 1e-20 <= temperature <= 1e20, 1 <= V <= 2^30, N <= 2^27, ld >= V (or 0), grad_ld >= V. */
int gem_policy(int dtype, int64_t N, int64_t V, const void* logits, int64_t ld,
               const int32_t* tokens, const float* old_logp, const float* advantage,
               const float* ref_logp, const float* row_scale, float temperature, float clip_low,
               float clip_high, float kl, float bonus, float* loss, float* logp, float* entropy,
               void* grad, int64_t grad_ld, void* stream);

/* Embedding: out[n] = scale table[tokens[n]] for N tokens (int32), rows of D elements: row v of the
 * table at table + v * table_ld (type table_dtype), row n of out at out + n * out_ld (type dtype; rounded
 * once).  A token < 0 has no row: zeros; one >= V gives NaN.  Requires N <= 2^27, 1 <= V <= 2^30, D <= 2^23, pitches from
 * D to 2^30. */
int gem_embed(int table_dtype, int dtype, int64_t N, int64_t V, int64_t D, const void* table,
              int64_t table_ld, const int32_t* tokens, float scale, void* out, int64_t out_ld,
              void* stream);

/* Bytes of gem_embed_grad's workspace; -1 for a size out of range. */
int64_t gem_embed_workspace(int64_t N, int64_t V, int64_t D);

/* Gradient of the embedding with respect to the table: dtable[v] = scale sum dout[n] over the n
 * with tokens[n] = v, from dout (row n at dout + n * dout_ld, type dtype), into dtable (row v at
 * dtable + v * dtable_ld, type grad_dtype).  Tokens outside [0, V) have no row and are left out, dout
 * unread.
 *   accumulate = 0: all V rows are written, those without a token with zeros.
 *   accumulate = 1: the sum is added to what dtable holds (a table that is also the output layer);
 *     rows without a token are not touched.
 *   workspace: gem_embed_workspace bytes, 16-byte aligned, in use until the call's work is done.
 * Sums are fp32, in the order of n and of pieces of it that the tokens alone fix.  Where an fp32 dtable is added to,
 * what is added, what it holds there and their sum count as 0 below 2^-126. */
int gem_embed_grad(int dtype, int grad_dtype, int64_t N, int64_t V, int64_t D, const void* dout,
                   int64_t dout_ld, const int32_t* tokens, float scale, int accumulate,
                   void* dtable, int64_t dtable_ld, void* workspace, void* stream);

enum gem_conv_form { GEM_CONV_LINEAR = 0, GEM_CONV_SILU = 1 };

/* Short causal convolution of each channel over time:
 *
 *   p_t = bias + sum_{k < W} weight_k x_{t - W + 1 + k},   y_t = p_t (GEM_CONV_LINEAR) or p_t sigmoid(p_t)
 *
 * over x (B sequences of T steps and D channels, of type dtype) into y; 2 <= W <= 4, D <= 2^30.
 *   weight [D][W], bias [D] fp32 (NULL: zeros).
 *   state [B][W - 1][D] fp32, NULL: zeros: the W - 1 inputs before the first step, oldest first.
 *   lengths [B] int32, NULL: all T.  Sequence b has lengths[b] steps (clipped to 0..T): past
 *     them x is not used and y is 0.
 *   reset [B][T] bytes, NULL: none.  Where it is not 0, every input before the step counts as 0 from
 *     then on, whatever it holds (packed documents).
 *   state_last [B][W - 1][D] fp32, may be NULL and may be state: the last W - 1 inputs, so that a call
 *     can go on where another ended (serving: T = 1 for each token). */
int gem_conv_forward(int dtype, int form, int64_t B, int64_t T, int64_t D, int W, const gem_seq_t* x,
                     const float* weight, const float* bias, const float* state,
                     const int32_t* lengths, const uint8_t* reset, const gem_seq_t* y,
                     float* state_last, void* stream);

/* Floats of gem_conv_backward's workspace; -1 for a size out of range. */
int64_t gem_conv_workspace(int64_t B, int64_t T, int64_t D, int W);

/* Gradients of the convolution: dy is the gradient with respect to y, dstate_last [B][W - 1][D] fp32
 * (NULL: zeros) that with respect to state_last; x, weight, bias, state, lengths, reset and form are
 * those of the forward call.  Writes dx (0 past lengths[b]), dweight [D][W], dbias [D] and dstate [B][W -
 * 1][D] fp32 (any of the last three may be NULL; dstate must not be dstate_last).  workspace: gem_conv_workspace floats,
 * in use until the call's work is done. */
int gem_conv_backward(int dtype, int form, int64_t B, int64_t T, int64_t D, int W,
                      const gem_seq_t* x, const float* weight, const float* bias,
                      const float* state, const int32_t* lengths, const uint8_t* reset,
                      const gem_seq_t* dy, const float* dstate_last, const gem_seq_t* dx,
                      float* dweight, float* dbias, float* dstate, float* workspace, void* stream);

/* Selective state space scan.  Each of D channels has N states; with step = softplus(dt + dt_bias)
 * (softplus != 0) or dt + dt_bias, per channel and step,
 *
 *   h_t[n] = exp(step_t A[n]) h_{t-1}[n] + step_t x_t b_t[n]
 *   y_t    = (sum_n c_t[n] h_t[n] + skip x_t) z_t sigmoid(z_t)
 *
 * from h_{-1} = h0.  b and c are shared by the D / G channels of each of G groups. */
typedef struct {
  int64_t B, T, D;
  int32_t N, G;              /* 1 <= N <= GEM_SSM_STATES; G divides D; D, G N <= 2^30 */
  int32_t softplus;
  gem_seq_t x, dt;           /* [B][T][D] */
  gem_seq_t b, c;            /* [B][T][G][N], the last two dimensions side by side */
  gem_seq_t z;               /* [B][T][D]; data NULL: no gate, y is the sum alone */
  const float* A;            /* [D][N] */
  const float* skip;         /* [D], NULL: zeros */
  const float* dt_bias;      /* [D], NULL: zeros */
  const int32_t* lengths;    /* [B], NULL: all T; past lengths[b] (clipped to 0..T) x, dt, b, c and z are not used, y is 0
                                and the state stays */
  const uint8_t* reset;      /* [B][T], NULL: none; where it is not 0, the state before the step counts as 0,
                                whatever it holds */
} gem_ssm_t;

/* Most states of a channel. */
#define GEM_SSM_STATES 64
/* Steps between the states that gem_ssm_forward saves for gem_ssm_backward. */
#define GEM_SSM_CHUNK 16

/* Floats of the `saved` buffer, [B][ceil(T / GEM_SSM_CHUNK)][D][N]; -1 for a size out of range. */
int64_t gem_ssm_saved_count(int64_t B, int64_t T, int64_t D, int N);

/* Floats of the workspace of gem_ssm_forward (backward = 0), or of one that serves both calls (backward =
 * 1); may be 0; -1 for a size out of range.  Most of the latter, where a group has more than 32 channels (16 for more than
 * 32 states), are the blocks' parts of db and dc: B T D floats for up to 16 states, 2 B T D for up to 32, 8 B T D for up to 64. */
int64_t gem_ssm_workspace(int64_t B, int64_t T, int64_t D, int N, int G, int backward);

/* The scan into y [B][T][D], of type dtype as x, dt, b, c and z.
 *   h0 [B][D][N] fp32, NULL: zeros.
 *   h_last [B][D][N] fp32, may be NULL and may be h0: the state after the last step (serving is a call with
 *     T = 1 for each token).
 *   saved, may be NULL: gem_ssm_saved_count floats, the state before steps 0, 16, 32, ... for
 *     gem_ssm_backward; those past a sequence's end are not written.
 *   workspace: gem_ssm_workspace floats (NULL where that is 0), in use until the call's work is done.
 * A state or step that is not finite stays so until a reset, but an infinite state may become NaN where
 * exp(step A) is 0 in fp32, and a state of 0 where it is infinite. */
int gem_ssm_forward(int dtype, const gem_ssm_t* in, const float* h0, const gem_seq_t* y,
                    float* h_last, float* saved, float* workspace, void* stream);

/* What gem_ssm_backward writes: gradients of the inputs of the same names, [D], [D][N] and [B][D][N] ones
 * fp32 (each may be NULL), those of sequences of type dtype, 0 past lengths[b] (dz only with a gate). */
typedef struct {
  gem_seq_t dx, ddt, db, dc, dz;
  float *dA, *dskip, *ddt_bias, *dh0;
} gem_ssm_grad_t;

/* Gradients of the scan: dy is the gradient with respect to y, dh_last [B][D][N] fp32 (NULL: zeros) that
 * with respect to h_last; in is that of the forward call and saved is what it saved.  dh0 may be
 * dh_last. */
int gem_ssm_backward(int dtype, const gem_ssm_t* in, const float* saved, const gem_seq_t* dy,
                     const float* dh_last, const gem_ssm_grad_t* out, float* workspace,
                     void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GEM_LM_H */
