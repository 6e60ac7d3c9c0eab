/*
 * reuse_ops — operators around a policy net on MI355X (gfx950): layer norm, the
 * gated delta rule (a memory per stream that is carried from frame to frame)
 * and the sampling of actions, in the library of reuse_net.h.
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
 *   dev_state:        [slots][heads_v][dk][dv] float32.
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

#ifdef __cplusplus
}
#endif
#endif
