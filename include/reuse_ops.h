/*
 * reuse_ops — operators around a policy net on MI355X (gfx950): layer norm, the
 * gated delta rule (a memory per stream that is carried from frame to frame), the
 * sampling of actions, the norm of a residual stream, the log-probabilities a
 * policy is trained on, a short convolution over a stream's last tokens and the
 * selective scan (a memory that decays by an amount of each token's own), in the
 * library of reuse_net.h.
 *
 * A policy over many streams of frames (Sec. 1: multiple input frames; Sec. 2:
 * actions and REINFORCE) normalises each frame's features, carries a memory
 * from one frame of a stream to its next, and draws an action from its logits;
 * with the backward calls the gradients reach the net's logits, where
 * reuse_net_backward takes over.
 *
 * Conventions are those of reuse_net.h: rn_status results, device pointers
 * owned by the caller, no device allocation and no host synchronisation here,
 * everything enqueued on hip_stream, nothing launched on an argument error
 * (reuse_ops_last_error() then describes it, for the calling thread).  The
 * calls keep no state, may be captured into a HIP graph and may run from
 * several threads.  Sums, states and statistics are float32 or wider whatever
 * the data type; results are rounded to it once.  All results are
 * deterministic: the same inputs give the same bits.
 *
 * dtype is RN_F32 or RN_BF16 and is that of the arrays given as void *.
 * A stride counts elements from one row (token) to the next; within a row
 * elements are contiguous.  Arrays need the alignment of their element type
 * only; calls are fastest where rows begin on 16 bytes.
 */
#ifndef REUSE_OPS_H
#define REUSE_OPS_H

#include "reuse_net.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Text of the calling thread's last error from a call below ("" if none). */
const char *reuse_ops_last_error(void);

/* ---- layer norm ----
 *
 *   mean = sum_j x_j / width, var = sum_j (x_j - mean)^2 / width,
 *   rstd = 1 / sqrt(var + eps), y_j = (x_j - mean) rstd weight_j + bias_j.
 */

/* y for `rows` rows of `width` elements (rows >= 0, width >= 1).
 *   dev_weight, dev_bias: [width] float32, or NULL for 1 and 0.
 *   dev_stats: NULL, or [rows][2] float32 that receives each row's mean and
 *              rstd for the backward call.
 * y may be x itself (same stride). */
rn_status reuse_ops_layer_norm(int64_t rows, int32_t width, const void *dev_x, int64_t x_stride, rn_dtype dtype,
                               const float *dev_weight, const float *dev_bias, float eps, void *dev_y,
                               int64_t y_stride, float *dev_stats, void *hip_stream);

/* Device scratch bytes the backward call needs for these sizes when it writes
 * weight or bias gradients (0 if a size is out of range). */
size_t reuse_ops_layer_norm_backward_scratch_bytes(int64_t rows, int32_t width);

/* Gradients of J given dy = dJ/dy: with t_j = dy_j weight_j and xh = (x - mean) rstd,
 *   dx_j = rstd (t_j - mean(t) - xh_j mean(t xh)),
 *   dweight_j = sum over rows dy_j xh_j,  dbias_j = sum over rows dy_j.
 *   dev_stats:   [rows][2] from the forward call.
 *   dev_dweight, dev_dbias: [width] float32 or NULL (not wanted); accumulate = 0
 *                overwrites them, accumulate != 0 adds to them.  No rows: zeros.
 *   dev_scratch: 256-byte aligned, at least the bytes above (NULL if neither
 *                gradient is wanted).
 * dx may be dy or x itself (same stride). */
rn_status reuse_ops_layer_norm_backward(int64_t rows, int32_t width, const void *dev_dy, int64_t dy_stride,
                                        const void *dev_x, int64_t x_stride, rn_dtype dtype, const float *dev_weight,
                                        const float *dev_stats, void *dev_dx, int64_t dx_stride, float *dev_dweight,
                                        float *dev_dbias, int32_t accumulate, void *dev_scratch, size_t scratch_bytes,
                                        void *hip_stream);

/* ---- sampling ---- */

/* Settings of a sampling call: each is one value for every row, or an array on
 * the device with a value per row where the pointer is not NULL. */
typedef struct {
    float temperature;            /* > 0; 0 or less, NaN, or below 1.4e-37: greedy (the largest logit, the
                                     lowest index of equal ones) */
    int32_t top_k;                /* keep the k largest logits; 0 or less: all */
    float top_p;                  /* keep the fewest that hold this share of the probability, one at least */
    float min_p;                  /* keep those with at least this share of the largest one's probability */
    const float *dev_temperature; /* [n] or NULL */
    const int32_t *dev_top_k;
    const float *dev_top_p;
    const float *dev_min_p;
} rn_sample_params;

#define RN_SAMPLE_MAX_VOCAB (1 << 20)

/* Draw one of `vocab` choices for each of n rows of logits with the given
 * random numbers u in [0, 1).
 *
 * With m the row's largest logit and c = log2(e) / temperature (float32):
 *   z_i = (l_i - m) c,  w_i = 2^31 2^(z_i) rounded to a whole number,
 * and the choices that stay are, in this order, the top_k largest, those with
 * 2^(z_i) >= min_p, and of these, from the largest down, each one before which
 * less than top_p of their summed weight lies (the first always stays).  Equal
 * logits rank by index.  The draw is the first choice, in index order, at which
 * the running sum of the weights that stay exceeds floor(u total).  Weights are
 * whole numbers, so sums have one value in any order and the draw depends on
 * the inputs alone; a choice less likely than 2^-32 of the likeliest is never
 * drawn.
 *
 *   dev_tokens:   [n] int32 choices.
 *   dev_logprobs: NULL, or [n] float32: log of the drawn choice's share of the
 *                 weights that stay, (z - log2(total 2^-31)) ln 2; 0 if greedy.
 * A NaN logit counts as -infinity; where the largest is +infinity only equal
 * ones stay; a row of nothing but -infinity gives -1 and -infinity.  u below 0
 * or NaN counts as 0, 1 and above draws the last that stays.
 * 1 <= vocab <= RN_SAMPLE_MAX_VOCAB, n >= 0. */
rn_status reuse_ops_sample(int32_t n, int32_t vocab, const void *dev_logits, int64_t stride, rn_dtype dtype,
                           const float *dev_u, const rn_sample_params *params, int32_t *dev_tokens,
                           float *dev_logprobs, void *hip_stream);

/* ---- gated delta rule ----
 *
 * A head's memory is a matrix S [dk][dv].  For each token with key k, query q
 * [dk], value v [dv], log decay g (<= 0) and write strength beta:
 *   S <- exp(g) S;  S <- S + beta k (v - S^T k)^T;  out = scale S^T q.
 * Value head h uses key head h / (heads_v / heads_k).  Keys of unit length keep
 * the memory bounded for beta in [0, 2].  g = -infinity empties the memory (an
 * episode that begins), if what it holds is finite.
 *
 * Values that are not finite (in float32 also finite ones from 3.39e38 on, which
 * round to infinity in bfloat16) reach what the rule makes of them, as NaN or
 * infinity, and nothing else: a token's q its out; an element of its v, or of the
 * first memory, that column of out and of the memory from there on; its k, g or
 * beta all columns from there on.  The gradients of a sequence that has such a
 * value, or gets one in dout or dfinal, may be NaN throughout; other sequences'
 * are not touched.
 */

#define RN_DELTA_MAX_DIM 128
#define RN_DELTA_CHUNK 64

typedef struct {
    int32_t n;                    /* sequences (streams), 0..65535 */
    int32_t heads_k, heads_v;     /* heads_v a multiple of heads_k */
    int32_t dk, dv;               /* 1..RN_DELTA_MAX_DIM */
    int64_t tokens;               /* tokens of all sequences, 0..2^31 - 1 */
    rn_dtype dtype;               /* of q, k, v and out */
    float scale;
    /* Elements from a token to the next; heads are contiguous within a token
     * (q, k: [heads_k][dk], v: [heads_v][dv]).  Below 2^23. */
    int64_t q_stride, k_stride, v_stride;
    /* Not 0: every sequence has tokens / n of them, and seq_off will be NULL.  The
     * sizes below are then those of the way such sequences take; 0 allows for any
     * lengths. */
    int32_t even;
} rn_delta_shape;

/* One token for each of n streams (tokens = n), the memory updated in place.
 *   dev_g, dev_beta:  [n][heads_v] float32.
 *   dev_state:        [slots][heads_v][dk][dv] float32 (NULL without slots).
 *   dev_stream_ids:   [n] distinct slots, or NULL for 0..n-1.  A stream whose id
 *                     is outside 0..slots-1 is left out and its out is 0.
 *   dev_out:          [n][heads_v][dv] dtype, contiguous. */
rn_status reuse_ops_delta_step(const rn_delta_shape *shape, const void *dev_q, const void *dev_k, const void *dev_v,
                               const float *dev_g, const float *dev_beta, const int32_t *dev_stream_ids,
                               int32_t slots, float *dev_state, void *dev_out, void *hip_stream);

/* Bytes of the buffer a forward call leaves for the backward call, and of the
 * scratch each call needs (0 if the shape is not supported; every size is at
 * least 256).  Where a call has 32 tokens a sequence on average or fewer, sequences
 * of up to 32 go token by token and take no scratch in the forward call.  All
 * others are taken by chunks of RN_DELTA_CHUNK tokens, each of which takes 37 KiB a
 * value head, and a key head 12 KiB (bfloat16) or 36 KiB (float32) for dk up to 32,
 * twice that up to 64, four times above; in the backward call also a memory.
 * seq_off is not known when the sizes are asked for: without `even` they allow for
 * as many chunks as any lengths can have. */
size_t reuse_ops_delta_saved_bytes(const rn_delta_shape *shape);
size_t reuse_ops_delta_scratch_bytes(const rn_delta_shape *shape);
size_t reuse_ops_delta_backward_scratch_bytes(const rn_delta_shape *shape);

/* All tokens of n sequences packed one after another: sequence i owns tokens
 * [seq_off[i], seq_off[i+1]), possibly none.
 *   dev_seq_off: [n+1] int32, seq_off[0] = 0, ascending, seq_off[n] = tokens; or
 *                NULL: every sequence has tokens / n.
 *   dev_state:   [n][heads_v][dk][dv] float32 memories before the first token, or
 *                NULL for zeros.
 *   dev_final:   the same after the last token, or NULL (not wanted).  It may be
 *                dev_state.
 *   dev_out:     [tokens][heads_v][dv] dtype, contiguous.
 *   dev_saved:   NULL, or reuse_ops_delta_saved_bytes bytes for the backward call.
 *   dev_scratch: reuse_ops_delta_scratch_bytes bytes; saved and scratch are
 *                256-byte aligned. */
rn_status reuse_ops_delta_forward(const rn_delta_shape *shape, const void *dev_q, const void *dev_k,
                                  const void *dev_v, const float *dev_g, const float *dev_beta,
                                  const int32_t *dev_seq_off, const float *dev_state, float *dev_final, void *dev_out,
                                  void *dev_saved, size_t saved_bytes, void *dev_scratch, size_t scratch_bytes,
                                  void *hip_stream);

/* Gradients of J given dout = dJ/dout and dfinal = dJ/dfinal (NULL: 0), for the
 * inputs and the saved buffer of a forward call.
 *   dev_dout:           [tokens][heads_v][dv] dtype, contiguous.
 *   dev_dq, dev_dk:     [tokens][heads_k][dk] dtype, contiguous, summed over the
 *                       value heads that share a key head.
 *   dev_dv:             [tokens][heads_v][dv] dtype, contiguous.
 *   dev_dg, dev_dbeta:  [tokens][heads_v] float32.
 *   dev_dstate:         [n][heads_v][dk][dv] float32, or NULL (not wanted).
 * dev_dstate must not be dev_dfinal. */
rn_status reuse_ops_delta_backward(const rn_delta_shape *shape, const void *dev_q, const void *dev_k,
                                   const void *dev_v, const float *dev_g, const float *dev_beta,
                                   const int32_t *dev_seq_off, const void *dev_saved, size_t saved_bytes,
                                   const void *dev_dout, const float *dev_dfinal, void *dev_dq, void *dev_dk,
                                   void *dev_dv, float *dev_dg, float *dev_dbeta, float *dev_dstate, void *dev_scratch,
                                   size_t scratch_bytes, void *hip_stream);

/* ---- residual norm ----
 *
 *   total_j = x_j + residual_j (float32, rounded to dtype; x_j itself without a residual),
 *   rstd = 1 / sqrt(sum_j total_j^2 / width + eps),  y_j = total_j rstd weight_j,
 * the norm being that of the rounded total, which is what the backward call and the
 * next layer see.  In 8 bits (e4m3, largest value 448), with t_j = total_j weight_j
 * rounded to float32 and m = max_j |t_j|:
 *   q_j = t_j (448 / m) rounded to nearest even (0 where m is 0),  scale = m rstd / 448,
 * so that y_j = q_j scale to half a step of e4m3, and q depends on no order of sums.
 * A row that holds NaN or infinity (or so large values that its sum of squares is
 * infinite) has the y of these formulas, a scale of NaN and any q.  Squares are float32:
 * those of values below 2^-75 are 0, beside eps or not.
 */

/* `rows` rows of `width` elements (rows >= 0, width >= 1); results are contiguous.
 *   dev_residual: NULL, or rows at residual_stride.
 *   dev_weight:   [width] float32, or NULL for 1.
 *   dev_y:        [rows][width] dtype, or NULL (not wanted).
 *   dev_q, dev_scales: [rows][width] e4m3 and [rows] float32, both or neither.
 *   dev_total:    [rows][width] dtype, or NULL; NULL without a residual.
 *   dev_rstd:     [rows] float32 for the backward call, or NULL.
 * y or total may be x or the residual itself where that is contiguous. */
rn_status reuse_ops_rms_norm(int64_t rows, int32_t width, const void *dev_x, int64_t x_stride, rn_dtype dtype,
                             const void *dev_residual, int64_t residual_stride, const float *dev_weight, float eps,
                             void *dev_y, void *dev_q, float *dev_scales, void *dev_total, float *dev_rstd,
                             void *hip_stream);

/* Device scratch bytes the backward call needs for these sizes when it writes
 * weight gradients (0 if a size is out of range). */
size_t reuse_ops_rms_norm_backward_scratch_bytes(int64_t rows, int32_t width);

/* Gradients of J given dy = dJ/dy and dtotal = dJ/dtotal (NULL: 0), the latter by
 * what else the total goes into: with t_j = dy_j weight_j and n_j = total_j rstd,
 *   dx_j = dtotal_j + rstd (t_j - n_j mean(t n)),  dweight_j = sum over rows dy_j n_j;
 * the residual's gradient is dx too.
 *   dev_total:   x of a forward call without a residual, its total otherwise.
 *   dev_rstd:    [rows] from the forward call.
 *   dev_dx:      [rows][width] dtype, contiguous; may be dy, total or dtotal itself
 *                where that is contiguous.
 *   dev_dweight: [width] float32 or NULL (not wanted); accumulate = 0 overwrites it,
 *                accumulate != 0 adds to it.  No rows: zeros.
 *   dev_scratch: 256-byte aligned, at least the bytes above (NULL if dweight is not
 *                wanted). */
rn_status reuse_ops_rms_norm_backward(int64_t rows, int32_t width, const void *dev_dy, int64_t dy_stride,
                                      const void *dev_total, int64_t total_stride, rn_dtype dtype,
                                      const float *dev_weight, const float *dev_rstd, const void *dev_dtotal,
                                      int64_t dtotal_stride, void *dev_dx, float *dev_dweight, int32_t accumulate,
                                      void *dev_scratch, size_t scratch_bytes, void *hip_stream);

/* ---- log-probabilities of given choices ----
 *
 * For each of n rows of `vocab` logits l and the choice t that was made, with
 *   p_i = exp(l_i / temperature) / sum_j exp(l_j / temperature):
 *   logprob = log p_t,  entropy = -sum_i p_i log p_i (0 log 0 = 0),
 * and the `top` choices of the largest logits with their log-probabilities, from the
 * largest down, the lowest index first of equal ones.
 *
 * A logit of -infinity has p = 0: a choice that is not allowed.  A row of nothing
 * else gives logprob -infinity, entropy 0 and gradients of 0.  A row with NaN or
 * +infinity gives NaN everywhere but in top_tokens, where NaN ranks as -infinity.
 * A t outside 0..vocab-1 gives logprob 0, without a gradient; the entropy is as ever.
 */

#define RN_LOGPROBS_MAX_TOP 64

/* Device scratch bytes of the call for these sizes, whatever its dtype (0 if one is out of range, never less than
 * 256 otherwise). */
size_t reuse_ops_log_probs_scratch_bytes(int32_t n, int32_t vocab, int32_t top);

/*   dev_logits:       n rows at `stride`; 1 <= vocab <= RN_SAMPLE_MAX_VOCAB, n >= 0.
 *   dev_tokens:       [n] int32 choices.
 *   temperature:      above 0 (4.3e-39 and more, so that 1.44 / temperature is finite), finite.
 *   dev_logprobs, dev_entropy: [n] float32 or NULL (not wanted).
 *   dev_top_tokens, dev_top_logprobs: [n][top] int32 and float32, 0 <= top <=
 *                     min(vocab, RN_LOGPROBS_MAX_TOP); NULL if top is 0.
 *   dev_stats:        NULL, or [n][4] float32 for the backward call: the largest
 *                     logit, 1 / sum_j exp((l_j - largest) / temperature), the
 *                     logarithm of that sum, the entropy.
 *   dev_scratch:      256-byte aligned, at least the bytes above. */
rn_status reuse_ops_log_probs(int32_t n, int32_t vocab, const void *dev_logits, int64_t stride, rn_dtype dtype,
                              const int32_t *dev_tokens, float temperature, int32_t top, float *dev_logprobs,
                              float *dev_entropy, int32_t *dev_top_tokens, float *dev_top_logprobs, float *dev_stats,
                              void *dev_scratch, size_t scratch_bytes, void *hip_stream);

/* Gradient of J given dJ/dlogprob and dJ/dentropy ([n] float32 each, NULL: 0):
 *   dl_i = (dlogprob ([i = t] - p_i) - dentropy p_i (log p_i + entropy)) / temperature.
 *   dev_stats:   from the forward call of the same logits and temperature.
 *   dev_dlogits: [n][vocab] dtype at dlogits_stride; may be logits itself at its stride. */
rn_status reuse_ops_log_probs_backward(int32_t n, int32_t vocab, const void *dev_logits, int64_t stride,
                                       rn_dtype dtype, const int32_t *dev_tokens, float temperature,
                                       const float *dev_stats, const float *dev_dlogprobs, const float *dev_dentropy,
                                       void *dev_dlogits, int64_t dlogits_stride, void *hip_stream);

/* ---- short causal convolution ----
 *
 * Each channel by itself, over a sequence's tokens x_t:
 *   pre_t = bias + sum_(k < taps) weight_k x_(t - taps + 1 + k),
 *   out_t = pre_t / (1 + exp(-pre_t)) (silu), or pre_t.
 * What lies before the sequence's first token is its window: the taps - 1 inputs
 * before, the oldest first.
 */

#define RN_CONV_MAX_TAPS 4

typedef struct {
    int32_t n;                    /* sequences (streams), 0..65535 */
    int32_t channels;             /* 1..65536 */
    int32_t taps;                 /* 1..RN_CONV_MAX_TAPS */
    int64_t tokens;               /* tokens of all sequences, 0..2^31 - 64 */
    rn_dtype dtype;               /* of x, out and the windows */
    int32_t silu;                 /* not 0: out = silu(pre) */
    int64_t x_stride;             /* elements from a token to the next, below 2^23 */
} rn_conv_shape;

/* One token for each of n streams (tokens = n), the windows updated in place.
 *   dev_weight:     [channels][taps] float32;  dev_bias: [channels] float32 or NULL (0).
 *   dev_window:     [slots][taps - 1][channels] dtype (NULL without slots); not used where
 *                   taps is 1.
 *   dev_stream_ids: [n] distinct slots, or NULL for 0..n-1.  A stream whose id is
 *                   outside 0..slots-1 is left out and its out is 0.
 *   dev_out:        [n][channels] dtype, contiguous; may be x itself where that is. */
rn_status reuse_ops_causal_conv_step(const rn_conv_shape *shape, const void *dev_x, const float *dev_weight,
                                     const float *dev_bias, const int32_t *dev_stream_ids, int32_t slots,
                                     void *dev_window, void *dev_out, void *hip_stream);

/* All tokens of n sequences packed one after another.
 *   dev_seq_off: [n+1] int32, ascending, or NULL: every sequence has tokens / n.  Tokens
 *                behind seq_off[n] (a padded batch) are no sequence's: their results
 *                are left as they were, and they have no part in any other's.
 *   dev_window:  [n][taps - 1][channels] dtype before the first token, or NULL for 0.
 *   dev_final:   the same after the last token, or NULL; not dev_window.
 *   dev_out:     [tokens][channels] dtype, contiguous; not x. */
rn_status reuse_ops_causal_conv(const rn_conv_shape *shape, const void *dev_x, const float *dev_weight,
                                const float *dev_bias, const int32_t *dev_seq_off, const void *dev_window,
                                void *dev_final, void *dev_out, void *hip_stream);

/* Device scratch bytes of the backward call (0 if the shape is out of range). */
size_t reuse_ops_causal_conv_backward_scratch_bytes(const rn_conv_shape *shape);

/* Gradients of J given dout = dJ/dout and dfinal = dJ/dfinal (NULL: 0).
 *   dev_dout:    [tokens][channels] dtype, contiguous.
 *   dev_dfinal:  [n][taps - 1][channels] dtype or NULL.
 *   dev_dx:      [tokens][channels] dtype, contiguous; neither x nor dout.
 *   dev_dweight, dev_dbias: [channels][taps] and [channels] float32.
 *   dev_dwindow: [n][taps - 1][channels] dtype or NULL (not wanted); not dfinal.
 *   dev_scratch: 256-byte aligned. */
rn_status reuse_ops_causal_conv_backward(const rn_conv_shape *shape, const void *dev_x, const float *dev_weight,
                                         const float *dev_bias, const int32_t *dev_seq_off, const void *dev_window,
                                         const void *dev_dout, const void *dev_dfinal, void *dev_dx,
                                         float *dev_dweight, float *dev_dbias, void *dev_dwindow, void *dev_scratch,
                                         size_t scratch_bytes, void *hip_stream);

/* ---- selective scan ----
 *
 * A channel c carries a state of `states` numbers h.  For each token, with its input
 * u, its step size and, of the channel's group, b and c:
 *   s = softplus(dt + dt_bias), or dt + dt_bias,
 *   h_i <- exp(s a_i) h_i + s b_i u,
 *   y = sum_i c_i h_i + d u,  out = y z / (1 + exp(-z)), or y without z.
 * Group g has channels g channels / groups and on.  With a <= 0 the states stay
 * bounded.  s = 0 leaves the state as it is, whatever a is: an infinite a counts as the
 * largest number of its sign, so that -infinity empties a state at every token whose s is
 * above 0, with a da of 0 and no part in ds.
 *
 * Values that are not finite reach what the rule makes of them, as NaN or infinity,
 * and nothing else: u, dt and z of a channel that channel's out, and u and dt its
 * state, from that token on; b and c those of all channels of the group.  A value
 * in one sequence reaches no other's results; dA, dD and the bias' gradient, which
 * are sums over all tokens, it does reach.
 */

#define RN_SCAN_MAX_STATES 64
#define RN_SCAN_KEEP 16

typedef struct {
    int32_t n;                    /* sequences (streams), 0..65535 */
    int32_t channels, groups;     /* channels 1..65536, a multiple of groups */
    int32_t states;               /* 1..RN_SCAN_MAX_STATES */
    int64_t tokens;               /* tokens of all sequences, 0..2^31 - 1 */
    rn_dtype dtype;               /* of u, dt, b, c, z and out */
    int32_t softplus;             /* not 0: s = softplus(dt + dt_bias) */
    /* Elements from a token to the next, below 2^23 (z_stride: not used without z).
     * Within a token elements are contiguous (u, dt, z: [channels], b, c:
     * [groups][states]). */
    int64_t u_stride, dt_stride, b_stride, c_stride, z_stride;
} rn_scan_shape;

/* What a scan reads beside the shape. */
typedef struct {
    const void *u, *dt, *b, *c;
    const float *a;               /* [channels][states] */
    const float *d;               /* [channels], or NULL for 0 */
    const void *z;                /* or NULL: out = y */
    const float *dt_bias;         /* [channels], or NULL for 0 */
} rn_scan_inputs;

/* One token for each of n streams (tokens = n), the states updated in place.
 *   dev_state:      [slots][channels][states] float32 (NULL without slots).
 *   dev_stream_ids: [n] distinct slots, or NULL for 0..n-1.  A stream whose id is
 *                   outside 0..slots-1 is left out and its out is 0.
 *   dev_out:        [n][channels] dtype, contiguous; may be u itself where that is. */
rn_status reuse_ops_scan_step(const rn_scan_shape *shape, const rn_scan_inputs *in, const int32_t *dev_stream_ids,
                              int32_t slots, float *dev_state, void *dev_out, void *hip_stream);

/* Bytes of the buffer a forward call leaves for the backward call (a state per
 * RN_SCAN_KEEP tokens and sequence), and of the scratch each call needs (0 if the
 * shape is not supported; every size is at least 256). */
size_t reuse_ops_scan_saved_bytes(const rn_scan_shape *shape);
size_t reuse_ops_scan_scratch_bytes(const rn_scan_shape *shape);
size_t reuse_ops_scan_backward_scratch_bytes(const rn_scan_shape *shape);

/* All tokens of n sequences packed one after another.
 *   dev_seq_off: as reuse_ops_causal_conv's.
 *   dev_state:   [n][channels][states] float32 before the first token, or NULL for 0.
 *   dev_final:   the same after the last token, or NULL; it may be dev_state.
 *   dev_out:     [tokens][channels] dtype, contiguous; not one of the inputs.
 *   dev_saved:   NULL, or reuse_ops_scan_saved_bytes bytes for the backward call.
 *   dev_scratch: reuse_ops_scan_scratch_bytes bytes; saved and scratch are 256-byte
 *                aligned. */
rn_status reuse_ops_scan_forward(const rn_scan_shape *shape, const rn_scan_inputs *in, const int32_t *dev_seq_off,
                                 const float *dev_state, float *dev_final, void *dev_out, void *dev_saved,
                                 size_t saved_bytes, void *dev_scratch, size_t scratch_bytes, void *hip_stream);

/* Where a backward call's gradients go: like what they are the gradients of, but
 * contiguous.  dz, dd, ddt_bias and dstate may be NULL (not wanted); dz is NULL
 * without z. */
typedef struct {
    void *du, *ddt, *db, *dc, *dz;
    float *da, *dd, *ddt_bias, *dstate;
} rn_scan_grads;

/* Gradients of J given dout = dJ/dout ([tokens][channels] dtype, contiguous) and
 * dfinal = dJ/dfinal (NULL: 0), for the inputs and the saved buffer of a forward
 * call.  No gradient lies over dout or an input; dstate is not dfinal. */
rn_status reuse_ops_scan_backward(const rn_scan_shape *shape, const rn_scan_inputs *in, const int32_t *dev_seq_off,
                                  const void *dev_saved, size_t saved_bytes, const void *dev_dout,
                                  const float *dev_dfinal, const rn_scan_grads *grads, void *dev_scratch,
                                  size_t scratch_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
