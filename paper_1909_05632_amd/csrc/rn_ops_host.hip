// C ABI of the operators (include/reuse_ops.h): argument checks, scratch layout,
// launches.  Nothing throws and nothing aborts.
#include "rn_ops.hpp"

#include <cstdio>

namespace {

using namespace rn;

constexpr size_t kAlign = 256;

// Fixed storage, so that reporting an error allocates nothing.
thread_local char g_error[160] = "";

rn_status fail(rn_status s, const char *why) {
    snprintf(g_error, sizeof g_error, "%s", why);
    return s;
}

rn_status launched(hipError_t e) {
    if (e == hipSuccess) return RN_OK;
    snprintf(g_error, sizeof g_error, "launch failed: %s", hipGetErrorString(e));
    return RN_EHIP;
}

rn_status need_bytes(const char *what, size_t need) {
    snprintf(g_error, sizeof g_error, "%s too small: need %zu bytes", what, need);
    return RN_ENOSPACE;
}

size_t round_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
bool known(rn_dtype d) { return d == RN_F32 || d == RN_BF16; }
bool misaligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % kAlign != 0; }

constexpr int64_t kMaxRows = int64_t(1) << 40, kMaxStride = 1 << 23;
constexpr int kMaxWidth = 1 << 30, kMaxHeads = 1024, kMaxSequences = 65535;

// ------------------------------------------------------------------ delta rule

const char *bad_shape(const rn_delta_shape *s) {
    if (!s) return "shape is NULL";
    if (s->n < 0 || s->n > kMaxSequences) return "n must be 0..65535";
    if (s->heads_k < 1 || s->heads_v < 1 || s->heads_v > kMaxHeads || s->heads_v % s->heads_k)
        return "heads_v must be 1..1024 and a multiple of heads_k";
    if (s->dk < 1 || s->dv < 1) return "dk and dv must be 1 or more";
    if (s->tokens < 0 || s->tokens > INT32_MAX) return "tokens must be 0..2^31 - 1";
    if (s->n == 0 && s->tokens > 0) return "tokens without sequences";
    if (s->even && s->n > 0 && s->tokens % s->n) return "of even sequences, tokens must be a multiple of n";
    if (!known(s->dtype)) return "dtype must be RN_F32 or RN_BF16";
    if (s->tokens > 1 && (s->q_stride < (int64_t)s->heads_k * s->dk || s->k_stride < (int64_t)s->heads_k * s->dk ||
                          s->v_stride < (int64_t)s->heads_v * s->dv))
        return "a token stride is smaller than its token";
    if (s->tokens > 1 && (s->q_stride >= kMaxStride || s->k_stride >= kMaxStride || s->v_stride >= kMaxStride))
        return "token strides must be below 2^23";
    return nullptr;
}

bool too_wide(const rn_delta_shape *s) { return s->dk > RN_DELTA_MAX_DIM || s->dv > RN_DELTA_MAX_DIM; }

struct DeltaSizes {
    size_t kept, states, tokens;          // bytes of before; after; [tokens][hv][dv] float32
    size_t keys, inverse, decay;          // of kf, qf, kt or qt; mf or pf; dec
    size_t map;
};

DeltaSizes sizes(const rn_delta_shape *s, bool even) {
    const size_t slots = (size_t)delta_slots(s->tokens, s->n, even), heads = s->heads_v;
    const bool bf16 = s->dtype == RN_BF16;
    return {round_up((size_t)delta_kept_slots(s->tokens, s->n) * heads * s->dk * s->dv * 4),
            round_up(slots * heads * s->dk * s->dv * 4),
            round_up((size_t)s->tokens * heads * s->dv * 4),
            round_up(slots * s->heads_k * 4 * delta_ksteps(s->dk) * delta_planes(bf16) * 1024),
            round_up(slots * heads * 6 * 3 * 1024), round_up(slots * heads * 3 * RN_DELTA_CHUNK * 4), round_up(slots * 16)};
}

size_t forward_bytes(const rn_delta_shape *s, bool even) {
    const DeltaSizes z = sizes(s, even);
    return 3 * z.keys + 2 * z.inverse + z.decay + kAlign;
}

size_t backward_bytes(const rn_delta_shape *s, bool even) {
    const DeltaSizes z = sizes(s, even);
    return 3 * z.keys + 2 * z.inverse + z.decay + z.states + z.tokens + z.map + kAlign;
}

DeltaArgs delta_args(const rn_delta_shape *s, const void *q, const void *k, const void *v, const float *g,
                     const float *beta) {
    DeltaArgs a{};
    a.n = s->n, a.hk = s->heads_k, a.hv = s->heads_v, a.dk = s->dk, a.dv = s->dv;
    a.tokens = s->tokens;
    a.scale = s->scale;
    a.qs = s->q_stride, a.ks = s->k_stride, a.vs = s->v_stride;
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta;
    return a;
}

rn_status check_delta(const rn_delta_shape *s, const void *q, const void *k, const void *v, const float *g,
                      const float *beta) {
    if (const char *why = bad_shape(s)) return fail(RN_EINVAL, why);
    if (too_wide(s)) return fail(RN_EUNSUPPORTED, "dk and dv above 128 have no kernel");
    if (s->tokens > 0 && (!q || !k || !v || !g || !beta)) return fail(RN_EINVAL, "q, k, v, g and beta must not be NULL");
    return RN_OK;
}

}  // namespace

extern "C" {

const char *reuse_ops_last_error(void) { return g_error; }

rn_status reuse_ops_layer_norm(int64_t rows, int32_t width, const void *x, int64_t x_stride, rn_dtype dtype,
                               const float *weight, const float *bias, float eps, void *y, int64_t y_stride,
                               float *stats, void *stream) {
    if (rows < 0 || rows > kMaxRows || width < 1 || width > kMaxWidth)
        return fail(RN_EINVAL, "rows must be 0..2^40 and width 1..2^30");
    if (!known(dtype)) return fail(RN_EINVAL, "dtype must be RN_F32 or RN_BF16");
    if (rows == 0) return RN_OK;
    if (!x || !y) return fail(RN_EINVAL, "x and y must not be NULL");
    if (rows > 1 && (x_stride < width || y_stride < width))
        return fail(RN_EINVAL, "a row stride is smaller than its row");
    if (!(eps >= 0.f)) return fail(RN_EINVAL, "eps must be 0 or more");
    NormArgs a{};
    a.rows = rows, a.width = width;
    a.x = x, a.y = y;
    a.xs = x_stride, a.ys = y_stride;
    a.weight = weight, a.bias = bias, a.eps = eps, a.stats = stats;
    return launched(launch_norm(a, dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

size_t reuse_ops_layer_norm_backward_scratch_bytes(int64_t rows, int32_t width) {
    if (rows < 0 || rows > kMaxRows || width < 1 || width > kMaxWidth) return 0;
    return round_up((size_t)norm_blocks(rows, width) * 2 * (size_t)width * 4);
}

rn_status reuse_ops_layer_norm_backward(int64_t rows, int32_t width, const void *dy, int64_t dy_stride, const void *x,
                                        int64_t x_stride, rn_dtype dtype, const float *weight, const float *stats,
                                        void *dx, int64_t dx_stride, float *dweight, float *dbias, int32_t accumulate,
                                        void *scratch, size_t scratch_bytes, void *stream) {
    if (rows < 0 || rows > kMaxRows || width < 1 || width > kMaxWidth)
        return fail(RN_EINVAL, "rows must be 0..2^40 and width 1..2^30");
    if (!known(dtype)) return fail(RN_EINVAL, "dtype must be RN_F32 or RN_BF16");
    const bool sums = dweight || dbias;
    if (rows == 0 && !sums) return RN_OK;
    if (rows > 0 && (!dy || !x || !stats || !dx)) return fail(RN_EINVAL, "dy, x, stats and dx must not be NULL");
    if (rows > 1 && (dy_stride < width || x_stride < width || dx_stride < width))
        return fail(RN_EINVAL, "a row stride is smaller than its row");
    if (sums) {
        if (!scratch) return fail(RN_EINVAL, "scratch is NULL");
        if (misaligned(scratch)) return fail(RN_EINVAL, "scratch must be 256-byte aligned");
        const size_t need = reuse_ops_layer_norm_backward_scratch_bytes(rows, width);
        if (scratch_bytes < need) return need_bytes("scratch", need);
    }
    NormArgs a{};
    a.rows = rows, a.width = width;
    a.x = x, a.dy = dy, a.y = dx;
    a.xs = x_stride, a.dys = dy_stride, a.ys = dx_stride;
    a.weight = weight, a.stats = const_cast<float *>(stats);
    a.blocks = rows > 0 ? norm_blocks(rows, width) : 0;
    a.part = sums ? static_cast<float *>(scratch) : nullptr;
    a.dweight = dweight, a.dbias = dbias, a.accumulate = accumulate;
    return launched(launch_norm_backward(a, dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_sample(int32_t n, int32_t vocab, const void *logits, int64_t stride, rn_dtype dtype,
                           const float *u, const rn_sample_params *params, int32_t *tokens, float *logprobs,
                           void *stream) {
    if (n < 0) return fail(RN_EINVAL, "n must be 0 or more");
    if (vocab < 1 || vocab > RN_SAMPLE_MAX_VOCAB) return fail(RN_EINVAL, "vocab must be 1..2^20");
    if (!known(dtype)) return fail(RN_EINVAL, "dtype must be RN_F32 or RN_BF16");
    if (!params) return fail(RN_EINVAL, "params is NULL");
    if (n == 0) return RN_OK;
    if (!logits || !u || !tokens) return fail(RN_EINVAL, "logits, u and tokens must not be NULL");
    if (n > 1 && stride < vocab) return fail(RN_EINVAL, "the row stride is smaller than a row");
    SampleArgs a{n, vocab, logits, stride, u, *params, tokens, logprobs};
    return launched(launch_sample(a, dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_delta_step(const rn_delta_shape *shape, const void *q, const void *k, const void *v,
                               const float *g, const float *beta, const int32_t *ids, int32_t slots, float *state,
                               void *out, void *stream) {
    if (rn_status s = check_delta(shape, q, k, v, g, beta)) return s;
    if (shape->tokens != shape->n) return fail(RN_EINVAL, "a step takes one token a stream: tokens must be n");
    if (slots < 0 || (!ids && slots < shape->n)) return fail(RN_EINVAL, "fewer slots than streams");
    if (shape->n == 0) return RN_OK;
    if (!state || !out) return fail(RN_EINVAL, "state and out must not be NULL");
    DeltaArgs a = delta_args(shape, q, k, v, g, beta);
    a.ids = ids, a.slots = slots, a.final_state = state, a.out = out;
    return launched(launch_delta_step(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

size_t reuse_ops_delta_saved_bytes(const rn_delta_shape *shape) {
    if (bad_shape(shape) || too_wide(shape)) return 0;
    const DeltaSizes z = sizes(shape, shape->even);
    return z.kept + z.tokens + kAlign;
}

size_t reuse_ops_delta_scratch_bytes(const rn_delta_shape *shape) {
    if (bad_shape(shape) || too_wide(shape)) return 0;
    return forward_bytes(shape, shape->even);
}

size_t reuse_ops_delta_backward_scratch_bytes(const rn_delta_shape *shape) {
    if (bad_shape(shape) || too_wide(shape)) return 0;
    return backward_bytes(shape, shape->even);
}

rn_status reuse_ops_delta_forward(const rn_delta_shape *shape, const void *q, const void *k, const void *v,
                                  const float *g, const float *beta, const int32_t *seq_off, const float *state,
                                  float *final_state, void *out, void *saved, size_t saved_bytes, void *scratch,
                                  size_t scratch_bytes, void *stream) {
    if (rn_status s = check_delta(shape, q, k, v, g, beta)) return s;
    if (shape->even && seq_off) return fail(RN_EINVAL, "even sequences have no seq_off");
    if (!seq_off && shape->n > 0 && shape->tokens % shape->n)
        return fail(RN_EINVAL, "without seq_off, tokens must be a multiple of n");
    if (shape->n == 0) return RN_OK;
    if (shape->tokens > 0 && !out) return fail(RN_EINVAL, "out must not be NULL");
    if (misaligned(saved) || misaligned(scratch)) return fail(RN_EINVAL, "saved and scratch must be 256-byte aligned");
    if (saved && saved_bytes < reuse_ops_delta_saved_bytes(shape))
        return need_bytes("saved", reuse_ops_delta_saved_bytes(shape));
    if (!scratch) return fail(RN_EINVAL, "scratch is NULL");
    const size_t need = forward_bytes(shape, !seq_off);
    if (scratch_bytes < need) return need_bytes("scratch", need);
    const DeltaSizes z = sizes(shape, !seq_off);
    char *kept = static_cast<char *>(saved), *at = static_cast<char *>(scratch);
    DeltaArgs a = delta_args(shape, q, k, v, g, beta);
    a.off = seq_off, a.state = state, a.final_state = final_state, a.out = out;
    a.kf = reinterpret_cast<uint16_t *>(at);
    a.qf = reinterpret_cast<uint16_t *>(at += z.keys);
    a.kt = reinterpret_cast<uint16_t *>(at += z.keys);
    a.mf = reinterpret_cast<uint16_t *>(at += z.keys);
    a.pf = reinterpret_cast<uint16_t *>(at += z.inverse);
    a.dec = reinterpret_cast<float *>(at += z.inverse);
    if (saved) {
        a.before = reinterpret_cast<float *>(kept);
        a.err = reinterpret_cast<float *>(kept + z.kept);
    }
    return launched(launch_delta_forward(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_delta_backward(const rn_delta_shape *shape, const void *q, const void *k, const void *v,
                                   const float *g, const float *beta, const int32_t *seq_off, const void *saved,
                                   size_t saved_bytes, const void *dout, const float *dfinal, void *dq, void *dk,
                                   void *dv, float *dg, float *dbeta, float *dstate, void *scratch,
                                   size_t scratch_bytes, void *stream) {
    if (rn_status s = check_delta(shape, q, k, v, g, beta)) return s;
    if (shape->even && seq_off) return fail(RN_EINVAL, "even sequences have no seq_off");
    if (!seq_off && shape->n > 0 && shape->tokens % shape->n)
        return fail(RN_EINVAL, "without seq_off, tokens must be a multiple of n");
    if (shape->n == 0) return RN_OK;
    if (shape->tokens > 0 && (!dout || !dq || !dk || !dv || !dg || !dbeta))
        return fail(RN_EINVAL, "dout and the gradients must not be NULL");
    if (dstate && dstate == dfinal) return fail(RN_EINVAL, "dstate must not be dfinal");
    if (!saved || !scratch) return fail(RN_EINVAL, "saved and scratch must not be NULL");
    if (misaligned(saved) || misaligned(scratch)) return fail(RN_EINVAL, "saved and scratch must be 256-byte aligned");
    if (saved_bytes < reuse_ops_delta_saved_bytes(shape)) return need_bytes("saved", reuse_ops_delta_saved_bytes(shape));
    const size_t need = backward_bytes(shape, !seq_off);
    if (scratch_bytes < need) return need_bytes("scratch", need);
    const DeltaSizes z = sizes(shape, !seq_off);
    char *kept = const_cast<char *>(static_cast<const char *>(saved)), *at = static_cast<char *>(scratch);
    DeltaArgs a = delta_args(shape, q, k, v, g, beta);
    a.off = seq_off;
    a.before = reinterpret_cast<float *>(kept);
    a.err = reinterpret_cast<float *>(kept + z.kept);
    a.dout = dout, a.dfinal = dfinal;
    a.kf = reinterpret_cast<uint16_t *>(at);
    a.kt = reinterpret_cast<uint16_t *>(at += z.keys);
    a.qt = reinterpret_cast<uint16_t *>(at += z.keys);
    a.mf = reinterpret_cast<uint16_t *>(at += z.keys);
    a.pf = reinterpret_cast<uint16_t *>(at += z.inverse);
    a.dec = reinterpret_cast<float *>(at += z.inverse);
    a.after = reinterpret_cast<float *>(at += z.decay);
    a.dwrite = reinterpret_cast<float *>(at += z.states);
    a.map = reinterpret_cast<int32_t *>(at += z.tokens);
    a.dq = dq, a.dkey = dk, a.dval = dv, a.dg = dg, a.dbeta = dbeta, a.dstate = dstate;
    return launched(launch_delta_backward(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
