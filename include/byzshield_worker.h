/*
 * byzshield_worker.h -- operators of a worker's training step (C-ABI of libbyzshield, one MI355X).
 *
 * The server of byzshield.h compares the r copies of a file's gradient bit by bit, so honest
 * workers have to compute the same bits.  The operators here do: calls of the same sizes and type on
 * the same values give the same bits, wherever their tensors lie and whatever their pitches are (no
 * atomics, every sum in a fixed order, launch shapes chosen by sizes and type alone).  A file within a
 * call of more rows or samples is a call of other sizes: copies have to be computed by calls alike.
 * None mixes the samples of a file (the preference loss those of a pair alone), and all of them enqueue work and nothing else.
 *
 * Conventions (beyond those of byzshield.h)
 *   - Device pointers of the current device; `stream` is a hipStream_t passed as void*.  No
 *     allocation, no host synchronisation; calls can be captured into HIP graphs.
 *   - Values of type `dtype`; statistics, losses, parameters of the norm and their gradients are
 *     fp32.  Sums are held in fp32 or more, each output is rounded once.
 *   - Pitches and strides count elements.  Any alignment to the element's size works; 16-byte
 *     aligned bases with pitches of whole 16 bytes are faster (the feed-forward of more than 16 tokens copies others first).
 *   - Sizes of zero are valid and give what is left (no output, or zero gradients).
 *   - Outputs do not overlap inputs unless a function says so.
 */
#ifndef BYZSHIELD_WORKER_H
#define BYZSHIELD_WORKER_H

#include "byzshield.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum byz_dtype { BYZ_F32 = 0, BYZ_BF16 = 1, BYZ_F16 = 2 } byz_dtype;

typedef enum byz_act {
    BYZ_ACT_NONE = 0,   /* z                                    */
    BYZ_ACT_RELU = 1,   /* max(z, 0); derivative 0 at 0; a NaN stays one */
    BYZ_ACT_SILU = 2,   /* z / (1 + exp(-z))                    */
    BYZ_ACT_GELU = 3,   /* z (1 + erf(z / sqrt 2)) / 2          */
    BYZ_ACT_SIGMOID = 4 /* 1 / (1 + exp(-z))                    */
} byz_act;

/* ------------------------------------------------------- group norm with an activation */

/*
 * Features of n samples, p positions (height * width) and c channels, channels last: value
 * (i, q, j) of x is x[i * x_sample + q * x_pixel + j], x_pixel >= c.  The channels form `groups`
 * groups of c / groups neighbours.  With mean and variance (biased) over a group's positions and
 * channels of one sample,
 *     y = act((x - mean) * rstd * gamma[j] + beta[j]),   rstd = 1 / sqrt(var + eps).
 * gamma and beta (c each) may be NULL (ones, zeros).  mean and rstd: n * groups each, both are
 * written.  y may be x itself with the same strides.
 */
size_t byz_group_norm_workspace_bytes(int64_t n, int64_t p, int64_t c, int groups, int dtype);
int byz_group_norm(const void *x, int64_t x_sample, int64_t x_pixel, int64_t n, int64_t p, int64_t c,
                   int groups, int dtype, const float *gamma, const float *beta, float eps, int act,
                   void *y, int64_t y_sample, int64_t y_pixel, float *mean, float *rstd,
                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * Its gradients for dy, from x and the call's mean and rstd: dx, and dgamma and dbeta (c each, sums
 * over samples and positions; both or neither may be NULL).  dx may be dy itself with the same strides.
 */
size_t byz_group_norm_backward_workspace_bytes(int64_t n, int64_t p, int64_t c, int groups, int dtype);
int byz_group_norm_backward(const void *dy, int64_t dy_sample, int64_t dy_pixel, const void *x,
                            int64_t x_sample, int64_t x_pixel, int64_t n, int64_t p, int64_t c,
                            int groups, int dtype, const float *gamma, const float *beta,
                            const float *mean, const float *rstd, int act, void *dx,
                            int64_t dx_sample, int64_t dx_pixel, float *dgamma, float *dbeta,
                            void *workspace, size_t workspace_bytes, void *stream);

/* ----------------------------------------------- distillation from a teacher's top logits */

#define BYZ_MAX_TEACHER 1024 /* most entries of a teacher's row */

/*
 * Row i of the student has `vocab` logits s (pitch ld); the teacher gives k entries of it (pitch
 * teacher_ld): logits t[j] and their places index[j].  A negative index is no entry.  With
 * p = softmax of t / temperature over the entries that are there, q = softmax of s / temperature
 * over the whole vocabulary,
 *     loss[i] = temperature^2 * sum_j p_j (log p_j - log q_index[j]),  lse[i] = log sum_v exp(s_v / temperature).
 * Entries with p_j = 0 add nothing (whatever the student has there); entries at one place add up.  A row without any
 * entry, or whose entries are all -inf, has loss 0 and gradient 0 whatever its logits are.  A student
 * logit of -inf is a banned one: q = 0 there.  An index of vocab or more makes the row's loss NaN,
 * and its gradient.  lse may be NULL.  temperature > 0; 1 <= k <= BYZ_MAX_TEACHER.
 */
int byz_distill_loss(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                     const float *teacher, const int32_t *index, int k, int64_t teacher_ld,
                     float temperature, float *loss, float *lse, void *stream);

/*
 * The gradient for dloss (one value a row), from the call's lse:
 *     dlogits[i, v] = dloss[i] * temperature * (q_v - sum of p_j with index[j] = v).
 * q has the rounding of lse to fp32 (2^-19 of it at most: a row with |lse| > 64 is summed again, at the price of a second
 * pass over it).
 * dlogits (pitch dlogits_ld, type dtype) may be the logits themselves with the same pitch.
 */
int byz_distill_loss_backward(const float *dloss, const void *logits, int64_t rows, int64_t vocab,
                              int64_t ld, int dtype, const float *teacher, const int32_t *index, int k,
                              int64_t teacher_ld, const float *lse, float temperature, void *dlogits,
                              int64_t dlogits_ld, void *stream);

/* Loss and gradient in one call, for a dloss that is known beforehand (the weight of a row in a mean): the logits
 * are read once where a row fits a compute unit.  The outputs of the two calls but for rounding (the gradient without that of
 * lse); lse may be NULL. */
size_t byz_distill_loss_step_workspace_bytes(int64_t rows, int64_t vocab, int k, int dtype);
int byz_distill_loss_step(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                          const float *teacher, const int32_t *index, int k, int64_t teacher_ld,
                          const float *dloss, float temperature, float *loss, float *lse,
                          void *dlogits, int64_t dlogits_ld, void *workspace, size_t workspace_bytes,
                          void *stream);

/* ------------------------------------------------------------- gated feed-forward block */

/*
 * m tokens of k values (x, pitch x_ld), two weights of n rows of k values (pitch w_ld), bf16 or fp16:
 *     gate = x w_gate^T,  up = x w_up^T,  h = act(gate) * up
 * in one kernel; the products are summed in fp32 and h (pitch h_ld) comes from the unrounded sums.
 * gate_out and up_out (m x n, pitch gate_ld; both or neither may be NULL) keep the sums for the
 * backward pass.  fp32 is BYZ_EUNSUPPORTED.  The workspace is for more than 16 tokens whose x or weights have to be
 * copied first: k not a multiple of 8, or rows that do not start at 16-byte boundaries; else it may be NULL.
 */
size_t byz_gated_ffn_workspace_bytes(int64_t m, int64_t k, int64_t n, int dtype);
int byz_gated_ffn(const void *x, int64_t x_ld, const void *w_gate, const void *w_up, int64_t w_ld,
                  int64_t m, int64_t k, int64_t n, int dtype, int act, void *h, int64_t h_ld,
                  float *gate_out, float *up_out, int64_t gate_ld, void *workspace,
                  size_t workspace_bytes, void *stream);

/*
 * Its gradients for dh (m x n, pitch dh_ld) from the saved gate and up (pitch gate_ld):
 *     dup = dh * act(gate),  dgate = dh * up * act'(gate)      (rounded to the type once)
 *     dx = dgate w_gate + dup w_up,  dw_gate = dgate^T x,  dw_up = dup^T x
 * dx has pitch dx_ld, dw_gate and dw_up pitch dw_ld; dx or both dw may be NULL.  The workspace has room for copies of x and
 * the weights, which a call whose k is a multiple of 8 and whose rows of x and weights all start at 16-byte boundaries does not
 * need: it takes the aligned size.
 */
size_t byz_gated_ffn_backward_workspace_bytes(int64_t m, int64_t k, int64_t n, int dtype);
size_t byz_gated_ffn_backward_aligned_workspace_bytes(int64_t m, int64_t k, int64_t n, int dtype);
int byz_gated_ffn_backward(const void *dh, int64_t dh_ld, const void *x, int64_t x_ld,
                           const void *w_gate, const void *w_up, int64_t w_ld, const float *gate,
                           const float *up, int64_t gate_ld, int64_t m, int64_t k, int64_t n, int dtype,
                           int act, void *dx, int64_t dx_ld, void *dw_gate, void *dw_up, int64_t dw_ld,
                           void *workspace, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------ dropout */

/*
 * y = x / (1 - p) where a value stays, 0 where it is dropped (whatever it is), of `rows` rows of `cols` values (pitches x_ld, y_ld).
 * Its gradient is the same call on dy.  No mask is stored: value (i, j) stays if 16 random bits of
 * Philox 4x32-10 (key: seed; counter: j / 8, first_row + i, and the 64-bit sum of offset and *offset_at) are p 2^16 or more, p 2^16
 * rounded to a whole number, whose p is also the scale's.  So the copies of a file drop the same values if they give
 * the same seed, offset and first_row; calls of one step need offsets of their own.
 * offset_at (device, 8-byte aligned) may be NULL: a captured call takes another offset at each replay from it.
 * 0 <= p <= 1, first_row + rows <= 2^32, cols < 2^31.  y may be x itself with the same pitch.
 */
int byz_dropout(const void *x, int64_t rows, int64_t cols, int64_t x_ld, int dtype, float p, uint64_t seed,
                uint64_t offset, const int64_t *offset_at, int64_t first_row, void *y, int64_t y_ld, void *stream);

/* --------------------------------------- a block's output joins the residual, and norms */

typedef enum byz_norm { BYZ_NORM_NONE = 0, BYZ_NORM_RMS = 1, BYZ_NORM_LAYER = 2 } byz_norm;

typedef struct byz_residual_form {
    int32_t post, pre; /* byz_norm */
    float eps, scale, p;
    uint64_t seed, offset; /* of the dropout, as in byz_dropout */
    const int64_t *offset_at;
    int64_t first_row;
} byz_residual_form;

/*
 * For each of `rows` rows of `cols` values of the residual x and a block's output h:
 *     u = norm_post(h) * post_weight + post_bias
 *     out = x + scale * gate * dropout(u)
 *     y = norm_pre(out) * pre_weight + pre_bias
 * with norm(v) = (v - mean) / sqrt(var + eps) for BYZ_NORM_LAYER (var biased), v / sqrt(mean of v^2 + eps) for BYZ_NORM_RMS, v
 * for BYZ_NORM_NONE; y is of the unrounded sum.  gate_rows rows one after the other share a row of gate, which has
 * ceil(rows / gate_rows) rows, and one at least, of cols values (gate_rows = rows: one for all).  Weights and biases (cols each) and gate may be NULL
 * (ones, zeros, ones).  Without a pre norm there is no y, and no pre_weight or pre_bias.  h NULL: no block, y = norm_pre(x), no out.
 * stats: rows * 4, mean and 1 / sqrt(...) of both norms (0 and 1 where there is none); it may be NULL if no gradients are
 * wanted.  out may be x or h with the same pitch, but the backward call needs both.  cols < 2^31.
 */
int byz_residual_norm(const void *x, int64_t x_ld, const void *h, int64_t h_ld, int64_t rows, int64_t cols, int dtype,
                      const byz_residual_form *form, const float *post_weight, const float *post_bias, const float *gate,
                      int64_t gate_rows, const float *pre_weight, const float *pre_bias, void *out, int64_t out_ld, void *y,
                      int64_t y_ld, float *stats, void *stream);

/*
 * Its gradients for dout and dy (either may be NULL: zeros), from the call's x, h and stats: dx and dh (no dh without h), and those of
 * the vectors, fp32 sums over the rows, each of which may be NULL; d_gate has gate's shape.  The workspace is that of the call's gate_rows, and
 * of gate_rows = rows without a gate.
 */
size_t byz_residual_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int dtype, int64_t gate_rows);
int byz_residual_norm_backward(const void *dout, int64_t dout_ld, const void *dy, int64_t dy_ld, const void *x, int64_t x_ld,
                               const void *h, int64_t h_ld, const float *stats, int64_t rows, int64_t cols, int dtype,
                               const byz_residual_form *form, const float *post_weight, const float *post_bias,
                               const float *gate, int64_t gate_rows, const float *pre_weight, void *dx, int64_t dx_ld,
                               void *dh, int64_t dh_ld, float *d_post_weight, float *d_post_bias, float *d_gate,
                               float *d_pre_weight, float *d_pre_bias, void *workspace, size_t workspace_bytes,
                               void *stream);

/* ------------------------------------------------ losses of tokens' log-probabilities */

/*
 * Row i has `vocab` logits z (pitch ld) and a token label[i]; a negative label is no token: log-probability, loss and
 * gradient 0, whatever the logits are.
 *     logp[i] = z_label / temperature - log sum_v exp(z_v / temperature),  q = softmax of z / temperature
 * A logit of -inf is a banned one: q = 0 there, logp = -inf if it is the label's.  A label of vocab or more makes the row NaN, and
 * its gradient.  stats: rows * 2, the row's largest logit m and log sum_v exp((z_v - m) / temperature), for the backward calls
 * (0 and 0 where all are banned or there is no token); where it is an output it may be NULL.  temperature >= 2^-64; vocab < 2^31.
 * All calls of this section take a workspace of byz_token_loss_workspace_bytes.  dlogits (pitch dlogits_ld, type dtype)
 * may be the logits themselves with the same pitch.
 */
size_t byz_token_loss_workspace_bytes(int64_t rows, int64_t vocab, int dtype);

/* Log-probabilities, and their gradient dlogits[i, v] = dlogp[i] / temperature * ((v = label) - q_v). */
int byz_token_logp(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, const int32_t *label,
                   float temperature, float *logp, float *stats, void *workspace, size_t workspace_bytes, void *stream);
int byz_token_logp_backward(const float *dlogp, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                            const int32_t *label, const float *stats, float temperature, void *dlogits, int64_t dlogits_ld,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * The clipped policy loss with a KL term, of each token: with a = advantage, r = exp(logp - old), g = ref - logp,
 *     loss = -min(r a, clamp(r, 1 - clip_low, 1 + clip_high) a) + kl (exp(g) - 1 - g)
 * old, advantage and ref hold a value a row (ref may be NULL if kl is 0).  The gradient of the first term is that of -r a where r is
 * within the bound on its side (at the bound too), else 0.  0 <= clip_low <= 1, 0 <= clip_high, 0 <= kl.
 * The step makes loss and gradient in one call for a dloss that is known beforehand (the weight of a token in a mean): the logits
 * are read once where a row fits a compute unit.
 */
int byz_policy_loss(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, const int32_t *label,
                    const float *old, const float *advantage, const float *ref, float clip_low, float clip_high, float kl,
                    float temperature, float *loss, float *logp, float *stats, void *workspace, size_t workspace_bytes,
                    void *stream);
int byz_policy_loss_backward(const float *dloss, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                             const int32_t *label, const float *old, const float *advantage, const float *ref,
                             float clip_low, float clip_high, float kl, float temperature, const float *stats,
                             void *dlogits, int64_t dlogits_ld, void *workspace, size_t workspace_bytes, void *stream);
int byz_policy_loss_step(const float *dloss, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                         const int32_t *label, const float *old, const float *advantage, const float *ref,
                         float clip_low, float clip_high, float kl, float temperature, float *loss, float *logp,
                         void *dlogits, int64_t dlogits_ld, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The preference loss of pairs of sequences: sequence s has the rows bounds[s] .. bounds[s + 1] - 1 (bounds: 2 pairs + 1, not
 * falling, within 0 .. rows), sequences 2 i and 2 i + 1 are the chosen and the rejected one of pair i.  With sums[s] the
 * sum of logp over s, and ref[s] the same of a reference model (NULL: zeros),
 *     margin = beta ((sums - ref)[2 i] - (sums - ref)[2 i + 1]),  sigma(x) = 1 / (1 + exp(-x))
 *     loss[i] = -(1 - smoothing) log sigma(margin) - smoothing log sigma(-margin),  slope[i] = d loss / d margin
 * Rows of no sequence are in no loss, and their gradient is 0.  A pair whose bounds fall or leave 0 .. rows has a NaN loss and
 * slope, and what gradient its rows get is not specified.
 * sums (2 pairs) and slope (pairs, for the backward call) may be NULL.  0 <= smoothing <= 1; beta is finite.
 */
int byz_preference_loss(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, const int32_t *label,
                        const int32_t *bounds, int64_t pairs, const float *ref, float beta, float smoothing,
                        float temperature, float *loss, float *sums, float *slope, float *stats, void *workspace,
                        size_t workspace_bytes, void *stream);
int byz_preference_loss_backward(const float *dloss, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                 const int32_t *label, const int32_t *bounds, int64_t pairs, const float *slope,
                                 float beta, float temperature, const float *stats, void *dlogits, int64_t dlogits_ld,
                                 void *workspace, size_t workspace_bytes, void *stream);
int byz_preference_loss_step(const float *dloss, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                             const int32_t *label, const int32_t *bounds, int64_t pairs, const float *ref, float beta,
                             float smoothing, float temperature, float *loss, float *sums, void *dlogits,
                             int64_t dlogits_ld, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BYZSHIELD_WORKER_H */
