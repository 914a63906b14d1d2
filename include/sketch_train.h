/*
 * sketch_train.h -- operators of a language model's training step around the
 * sketches (C ABI, same conventions as sketch.h).
 *
 * Data attribution sketches the gradient of a loss, and an intrinsic-dimension
 * run steps omega on the sketched gradient of one.  These entry points are the
 * parts of such a step that lie outside the model's blocks: the embedding
 * lookup and its gradient (per example, as sketch_apply takes it, or summed),
 * the log-probabilities of given tokens, from logits or from hidden states and the
 * output matrix, the clipped policy loss and the preference loss with their
 * gradients, dropout, the balance loss of a router, and AdamW over a parameter
 * list.
 *
 * Conventions: return 0 or a negative SK_E* code (sketch_last_error() gives
 * the message); arguments are validated before any device work is queued;
 * device pointers are plain HIP addresses on `device`, aligned to their
 * element; work is queued on `stream` (a hipStream_t, NULL = legacy default);
 * nothing here synchronises, allocates device memory (but creation) or uses
 * floating-point atomics: results are bitwise deterministic.  Values held in
 * device memory (ids, offsets) cannot be refused by the call: ids outside
 * [0, vocab) are the masked entries described at each operator, and offsets are
 * clamped to [0, rows].  Inputs may not overlap outputs unless said otherwise.
 */
#ifndef SK_SKETCH_TRAIN_H
#define SK_SKETCH_TRAIN_H

#include <stdint.h>

#include "sketch.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SK_I32 = 0, SK_I64 = 1 } sk_index; /* type of ids and offsets */

/*
 * Embedding lookup: out[t] = scale * weight[ids[t]] for t < n, rounded once to
 * out_dtype.  An id outside [0, vocab) gives a row of zeros (padding, or an id
 * of another shard of the vocabulary).
 *   weight   [vocab, width], row stride ld >= width elements.
 *   out      [n, width] contiguous.
 */
int sketch_embed(const void *weight, sk_dtype dtype, int64_t vocab, int64_t width, int64_t ld, const void *ids,
                 sk_index index, int64_t n, float scale, void *out, sk_dtype out_dtype, int32_t device, void *stream);

/*
 * Gradient of the lookup: for each of `batch` groups of n tokens
 *   out[v] (+)= scale * sum over t with ids[t] = v of dy[t]
 * with the sum in fp32, rounded once to out_dtype; ids outside [0, vocab) add
 * nothing.  The order of a sum is set by the ids, the sizes and the types: that of
 * t for up to 1024 tokens a group and 64 MB of out; else that of t in pieces of
 * the sorted tokens (16, 32 or 64, by batch * n * width), then the pieces, every
 * fourth of them in a sum of its own.  The same call gives the same bits; the
 * gradient of one text may differ in its last bits with the batch it is part of.
 * batch > 1 gives one gradient per example.  Rows that no id names are zeroed
 * (accumulate = 0) or kept (accumulate = 1).
 *   dy       [batch, n, width], row stride ld >= width elements.
 *   out      [batch, vocab, width] contiguous.
 *   work     sketch_embed_grad_work_bytes(batch, n, width) bytes, 256-byte aligned.
 * SK_EUNSUPPORTED for vocab > 2^20, batch > 2^18, batch * n >= 2^28, width > 2^24 or
 * about batch * n * width > 2^37.
 */
int64_t sketch_embed_grad_work_bytes(int64_t batch, int64_t n, int64_t width);
int sketch_embed_grad(const void *dy, sk_dtype dtype, int64_t ld, const void *ids, sk_index index, int64_t batch,
                      int64_t n, int64_t vocab, int64_t width, float scale, void *out, sk_dtype out_dtype,
                      int32_t accumulate, void *work, int64_t work_bytes, int32_t device, void *stream);

/*
 * Logits of `rows` positions with their targets, common to the losses.
 *   data     [rows, vocab], row stride ld >= vocab elements.
 *   targets  [rows]; a target outside [0, vocab) masks its position: the row of
 *            logits is not read, its log-probability counts as 0 and its
 *            gradient is a row of zeros.
 *   scale    in [2^-120, 2^127]: the softmax is that of scale * data
 *            (1 / temperature).
 * vocab < 2^31.
 */
typedef struct {
  const void *data;
  const void *targets;
  int64_t rows, vocab, ld;
  float scale;
  sk_dtype dtype;
  sk_index index;
  int32_t device;
} sk_logits;

/*
 * logp[t] = log softmax(scale x_t)[targets[t]] (fp32).  stats [rows, 2] fp32
 * (NULL if not wanted): the row's largest logit m and sum exp(scale (x - m)), what
 * sketch_token_logp_grad needs (0, 0 at masked rows).  A row without a logit above -inf has
 * logp = -inf and a gradient of zeros; NaN and +inf follow the formula.
 */
int sketch_token_logp(const sk_logits *x, float *logp, float *stats, void *stream);

/*
 * dlogits[t] = scale * dlogp[t] * (onehot(targets[t]) - softmax(scale x_t)) in
 * the type of the logits (row stride ld_out), from the stats of
 * sketch_token_logp.  Rows with dlogp = 0 are not read.  dlogits may be the
 * logits themselves (same ld).
 */
int sketch_token_logp_grad(const sk_logits *x, const float *stats, const float *dlogp, void *dlogits, int64_t ld_out,
                           void *stream);

/*
 * Clipped policy loss with a divergence term, per token t
 *   r    = exp(logp - old_logp)
 *   l_t  = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *          + kl_coef (exp(ref_logp - logp) - (ref_logp - logp) - 1)
 *   loss = sum_t weights[t] l_t     (summed in fp64)
 * and, where dlogits is not NULL, d loss / d logits in the type of the logits,
 * in the same pass over them.  Positions with a masked target or weight 0 are
 * not read and count as l_t = 0, logp = 0.
 *   ref_logp   NULL if kl_coef = 0.
 *   loss       one float; logp, token_loss  [rows] fp32 (l_t, unweighted).
 * dlogits may be the logits themselves (same ld).
 */
int sketch_policy_loss(const sk_logits *x, const float *old_logp, const float *advantages, const float *weights,
                       const float *ref_logp, float clip_low, float clip_high, float kl_coef, float *loss, float *logp,
                       float *token_loss, void *dlogits, int64_t ld_out, void *stream);

/*
 * Preference loss over pairs of texts: text i holds rows offsets[i] ..
 * offsets[i + 1] - 1, the even texts are chosen over the odd ones that follow.
 *   s_i  = sum over its unmasked rows of logp     (the mean if `average`)
 *   d_p  = (s_2p - s_2p+1) - the same of ref_logp (fp64 sums of logp - ref_logp)
 *   l_p  = -(1 - smoothing) log sigmoid(beta d_p) - smoothing log sigmoid(-beta d_p)
 *   loss = mean over pairs of l_p
 * and, where dlogits is not NULL, d loss / d logits in the type of the logits.
 *   offsets    [2 pairs + 1], ascending; rows outside all texts get zeros.
 *   ref_logp   [rows] fp32 (not read at masked rows).
 *   loss       one float; seq_logp [2 pairs], pair_loss [pairs] fp32.
 *   work       sketch_preference_work_bytes(rows) bytes, 16-byte aligned.
 * dlogits may be the logits themselves (same ld).
 */
int64_t sketch_preference_work_bytes(int64_t rows);
int sketch_preference_loss(const sk_logits *x, const void *offsets, sk_index offsets_index, int64_t pairs,
                           const float *ref_logp, float beta, float smoothing, int32_t average, float *loss,
                           float *seq_logp, float *pair_loss, void *dlogits, int64_t ld_out, void *work,
                           int64_t work_bytes, void *stream);

/*
 * Hidden states of `rows` positions, the output matrix that turns them into
 * logits x_t = weight hidden_t, and their targets.  The logits are formed in
 * pieces and never kept.
 *   hidden   [rows, width], row stride ld_hidden >= width elements.
 *   weight   [vocab, width], row stride ld_weight >= width elements.
 *   targets, scale  as in sk_logits; of a masked position the hidden state is
 *            not read either.
 * dtype is that of hidden and weight.  SK_EUNSUPPORTED for rows > 2^20, vocab > 2^22
 * or width > 2^16.
 */
typedef struct {
  const void *hidden;
  const void *weight;
  const void *targets;
  int64_t rows, vocab, width, ld_hidden, ld_weight;
  float scale;
  sk_dtype dtype;
  sk_index index;
  int32_t device;
} sk_linear;

/*
 * logp[t] = log softmax(scale x_t)[targets[t]] (fp32) and stats [rows, 2] fp32
 * (NULL if not wanted), as sketch_token_logp gives them for these logits.  Sums are
 * fp32.  bf16 products are exact; of fp32 inputs (more than 16 rows) each product is
 * taken from two numbers of 11 bits an operand: 22 bits, what lies below 2^-38 of the
 * largest entry of a row of hidden or weight is lost, and infinities and NaNs give
 * NaNs in what they reach.
 *   work     sketch_linear_logp_work_bytes(x) bytes (0 if x is refused), 256-byte
 *            aligned.
 */
int64_t sketch_linear_logp_work_bytes(const sk_linear *x);
int sketch_linear_logp(const sk_linear *x, float *logp, float *stats, void *work, int64_t work_bytes, void *stream);

/*
 * The gradient of sum_t dlogp[t] logp[t] from the stats of sketch_linear_logp:
 * with g_t = scale dlogp[t] (onehot(targets[t]) - softmax(scale x_t)),
 *   dhidden[t] = sum_v g_tv weight[v]        (the type of hidden; masked rows get
 *                zeros, row stride ld_dhidden; NULL if not wanted)
 *   dweight[b][v] (+)= sum over the rows t of example b of g_tv hidden[t]
 *                [batch, vocab, width] contiguous, NULL if not wanted: rows are
 *                `batch` examples of rows / batch each, batch > 1 gives one gradient
 *                per example.  Of fp32 weights it is fp32, of bf16 weights either.
 * Sums are fp32 and rounded once.  bf16 inputs: g is rounded to bf16 before the
 * products, and what the targets' entries have lost is returned to both gradients; up
 * to 256 rows, and with dweight in fp32 up to 256 rows an example, g takes two bf16
 * (2^-16).  fp32 inputs: products as above; of dweight[b][v] what lies below 2^-37 of
 * its largest |g_tv| max |hidden[t]| is lost, of dhidden[t] what lies below 2^-36 of
 * dlogp[t] times the largest entry of weight.  A weight that is not finite gives NaNs.
 * Rows with dlogp = 0 are masked.  Outputs may not overlap inputs.
 *   work     sketch_linear_logp_grad_work_bytes(x, batch, dhidden wanted, dweight
 *            wanted) bytes (0 if refused), 256-byte aligned.
 * SK_EUNSUPPORTED for batch > 2^14.
 */
int64_t sketch_linear_logp_grad_work_bytes(const sk_linear *x, int64_t batch, int32_t dhidden, int32_t dweight);
int sketch_linear_logp_grad(const sk_linear *x, int64_t batch, const float *stats, const float *dlogp, void *dhidden,
                            int64_t ld_dhidden, void *dweight, sk_dtype dweight_dtype, int32_t accumulate, void *work,
                            int64_t work_bytes, void *stream);

/*
 * Dropout with a mask that is drawn again wherever it is needed:
 *   out_i = residual_i + (u_i >= t ? x_i 65536 / (65536 - t) : 0),  t = floor(65536 p + 1/2)
 * for element i = row * width + column of x, in fp32 and rounded once.  u_i is half
 * (i mod 2) of word (i / 2 mod 4) of the Philox4x32-10 block with counter
 * (i / 8, step, site, SK_STREAM_DROPOUT) under the key of `seed`: p counts in
 * steps of 2^-16, and what is dropped may be anything.  The gradient with respect
 * to x is the same call with dy in the place of x and without residual (that one's
 * gradient is dy).
 *   x, residual (NULL if none), out  [rows, width] of one type, row strides >= width
 *   p        in [0, 1]; p that rounds to t = 65536 drops everything.
 *   step_at  NULL, or one int64 in device memory whose low 32 bits stand for step
 *            (a captured graph that is replayed draws a new mask when it changes)
 *   step, site  in [0, 2^32)
 * out may be x or residual (same row stride).  SK_EUNSUPPORTED for more than 2^35
 * elements.
 */
#define SK_STREAM_DROPOUT 13
int sketch_dropout(const void *x, sk_dtype dtype, int64_t rows, int64_t width, int64_t ld, const void *residual,
                   int64_t ld_residual, void *out, int64_t ld_out, double p, uint64_t seed, int64_t step,
                   const int64_t *step_at, int64_t site, int32_t device, void *stream);

/*
 * Balance loss of a router over E = `experts` from the logits of its tokens and the
 * k ids it has chosen for each:
 *   c_e = ids equal to e (counts),  n = tokens with an id in [0, E)
 *   P_e = mean over those tokens of softmax(logits)_e (probs),  f_e = c_e / (n k)
 *   loss = coef E sum_e f_e P_e  (coef where f or P is even)
 *   dlogits_te = coef E / n p_te (f_e - sum_e' f_e' p_te')
 * (c_e has no gradient).  A token without an id in [0, E) is masked: its logits may
 * be anything, its gradient is a row of zeros.  An id counts as often as it stands.
 * With n = 0 everything is 0.  A row of -inf alone counts with probabilities 0.
 *   logits   [tokens, E], row stride ld >= E;  ids [tokens, k] contiguous
 *   loss, probs [E]  fp32;  counts [E] int64
 *   dlogits  NULL, or the type of the logits, row stride ld_out; may be the logits
 *            themselves (same ld)
 *   work     sketch_balance_work_bytes(experts) bytes, 16-byte aligned
 * SK_EUNSUPPORTED for experts > 2048, k > 1024 or 2^31 ids.
 */
int64_t sketch_balance_work_bytes(int64_t experts);
int sketch_balance_loss(const void *logits, sk_dtype dtype, int64_t tokens, int64_t experts, int64_t ld, const void *ids,
                        sk_index index, int64_t k, float coef, float *loss, int64_t *counts, float *probs, void *dlogits,
                        int64_t ld_out, void *work, int64_t work_bytes, int32_t device, void *stream);

/*
 * AdamW over a list of parameter tensors, one launch for up to 160 of them:
 *   g = g s;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
 *   p = p (1 - lr wd_l) - lr / (1 - b1^step) m / (sqrt(v / (1 - b2^step)) + eps)
 * in fp32, each product and sum of the two moments rounded by itself, so that
 * they can be reproduced bit by bit.  s is grad_scale, times
 * min(1, max_norm / (norm + 1e-6)) where max_norm > 0, norm = |grad_scale| times
 * the 2-norm of all gradients (fp64 sums).  A step whose s is not finite
 * changes nothing.
 *
 * Moments are held in 64-element blocks of each tensor (a tensor's last block
 * is padded with zeros), by concatenation in list order:
 *   SK_ADAMW_F32   fp32.
 *   SK_ADAMW_8BIT  one byte an element and one exponent byte E + 127 a block.
 *     m: sign, 4 exponent bits, 3 mantissa bits; v: 5 exponent bits, 3 mantissa
 *     bits.  The fields (e, f) stand for 2^(E + e - top) (1 + f / 8), e = 0 for
 *     2^(E + 1 - top) f / 8, with top = 15 (m), 31 (v).  E is the exponent of
 *     the block's largest value, one more where that has a mantissa above 1.875
 *     (so that nothing is cut off at the top).  Values are rounded up or down
 *     at random so that the expected value is exact (an average with b2 = 0.999
 *     changes by less than half a step at a time and would stand still under
 *     rounding to nearest): the 20 fp32 mantissa bits below the code get
 *     16 u + 8 added and are cut off, u the high (m) or low (v) half of word
 *     (i mod 4) of the Philox4x32-10 block with counter
 *     (i / 4, step, l, SK_STREAM_ADAMW) under the key of `seed`, for element i
 *     of tensor l.  A block that holds an infinity or NaN has exponent byte 255
 *     and stands for NaNs.
 * step, lr and the other numbers of a call are taken when it is made: a captured
 * graph repeats that very step, its bias corrections and its random words, at
 * every replay.  A replay stands for training only where that is meant; a step of
 * its own number is a call of its own.
 *
 * Parameters in bf16 without a master copy are rounded the same way: the 16
 * bits that are cut off get u added, half (i mod 2) of word (i / 2 mod 4) of
 * the block with counter (i / 8, step, l, SK_STREAM_ADAMW_P).  To a NaN nothing is
 * added.
 */
#define SK_STREAM_ADAMW 11
#define SK_STREAM_ADAMW_P 12
typedef enum { SK_ADAMW_F32 = 0, SK_ADAMW_8BIT = 1 } sk_adamw_state;
typedef struct sk_adamw sk_adamw;

/* numel, decay: host arrays of n_tensors element counts (1 .. 2^34 - 1) and
 * factors of weight_decay (NULL: 1 for all).  The handle owns only its tables
 * and the partial sums of the norm. */
int sketch_adamw_create(const int64_t *numel, const float *decay, int32_t n_tensors, sk_adamw_state state,
                        uint64_t seed, int32_t device, sk_adamw **out);
/* Elements of one moment (a multiple of 64; the exponents of SK_ADAMW_8BIT are
 * a 64th of it). */
int64_t sketch_adamw_state_elems(const sk_adamw *h);

/* One step's numbers; the pointers are device memory of the handle's device.
 * lr weight_decay, lr / (1 - beta1^step) and eps must be finite in fp32, and an
 * eps above 0 must not become 0 there (SK_EINVAL). */
typedef struct {
  int64_t step;            /* 1, 2, .. < 2^32 */
  double lr, beta1, beta2, eps, weight_decay;
  double max_norm;         /* 0: no clipping */
  const float *grad_scale; /* one float, or NULL for 1 */
  float *norm;             /* one float, or NULL; written if max_norm > 0 */
  void *m, *v;             /* fp32 or bytes, sketch_adamw_state_elems entries, 256-byte aligned */
  uint8_t *m_exp, *v_exp;  /* SK_ADAMW_8BIT only */
} sk_adamw_step;
/* params, grads, masters: host arrays of n_tensors device pointers, read during
 * the call; params of `pdtype`, grads of `gdtype`, contiguous.  masters (NULL
 * if none): fp32 copies that the step is taken on, each parameter then being
 * its master rounded to nearest. */
int sketch_adamw_apply(sk_adamw *h, const sk_adamw_step *a, void *const *params, sk_dtype pdtype,
                       const void *const *grads, sk_dtype gdtype, float *const *masters, void *stream);
/* The values that moments in 8 bits stand for, fp32, state_elems entries each. */
int sketch_adamw_moments(sk_adamw *h, const uint8_t *m, const uint8_t *m_exp, const uint8_t *v, const uint8_t *v_exp,
                         float *m_out, float *v_out, void *stream);
/* Free the handle (synchronises its device).  NULL is a no-op. */
void sketch_adamw_destroy(sk_adamw *h);

#ifdef __cplusplus
}
#endif

#endif /* SK_SKETCH_TRAIN_H */
