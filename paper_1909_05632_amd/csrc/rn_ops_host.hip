// C ABI of the operators (include/reuse_ops.h): argument checks, scratch layout,
// launches.  Nothing throws and nothing aborts.
#include "rn_ops.hpp"

#include <cmath>
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
constexpr int kMaxWidth = 1 << 30, kMaxHeads = 1024, kMaxSequences = 65535, kMaxChannels = 65536;

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

// ------------------------------------------------------------------ log-probabilities

const char *bad_logp(int32_t n, int32_t vocab, int32_t top) {
    if (n < 0) return "n must be 0 or more";
    if (vocab < 1 || vocab > RN_SAMPLE_MAX_VOCAB) return "vocab must be 1..2^20";
    if (top < 0 || top > RN_LOGPROBS_MAX_TOP || top > vocab) return "top must be 0..64 and no more than vocab";
    return nullptr;
}

constexpr float kLog2e = 1.4426950408889634f;

bool bad_temperature(float t) { return !(t > 0.f) || !(t < HUGE_VALF) || !(kLog2e / t < HUGE_VALF); }

LogpArgs logp_args(int32_t n, int32_t vocab, const void *logits, int64_t stride, const int32_t *tokens,
                   float temperature, float *stats) {
    LogpArgs a{};
    a.n = n, a.vocab = vocab;
    a.logits = logits, a.stride = stride, a.tokens = tokens;
    a.c = kLog2e / temperature, a.inv_t = 1.f / temperature;
    a.stats = stats;
    return a;
}

// ------------------------------------------------------------------ short convolution

const char *bad_conv(const rn_conv_shape *s) {
    if (!s) return "shape is NULL";
    if (s->n < 0 || s->n > kMaxSequences) return "n must be 0..65535";
    if (s->channels < 1 || s->channels > kMaxChannels) return "channels must be 1..65536";
    if (s->taps < 1 || s->taps > RN_CONV_MAX_TAPS) return "taps must be 1..4";
    // The kernels count some tokens past the last in 32 bits.
    if (s->tokens < 0 || s->tokens > INT32_MAX - 63) return "tokens must be 0..2^31 - 64";
    if (s->n == 0 && s->tokens > 0) return "tokens without sequences";
    if (!known(s->dtype)) return "dtype must be RN_F32 or RN_BF16";
    if (s->tokens > 1 && s->x_stride < s->channels) return "a token stride is smaller than its token";
    if (s->tokens > 1 && s->x_stride >= kMaxStride) return "token strides must be below 2^23";
    return nullptr;
}

CausalArgs conv_args(const rn_conv_shape *s, const void *x, const float *weight, const float *bias) {
    CausalArgs a{};
    a.n = s->n, a.channels = s->channels, a.taps = s->taps, a.silu = s->silu;
    a.tokens = s->tokens, a.xs = s->x_stride;
    a.even = s->n > 0 ? (int)(s->tokens / s->n) : 0;
    a.x = x, a.weight = weight, a.bias = bias;
    return a;
}

// ------------------------------------------------------------------ selective scan

const char *bad_scan(const rn_scan_shape *s) {
    if (!s) return "shape is NULL";
    if (s->n < 0 || s->n > kMaxSequences) return "n must be 0..65535";
    if (s->channels < 1 || s->channels > kMaxChannels || s->groups < 1 || s->channels % s->groups)
        return "channels must be 1..65536 and a multiple of groups";
    if (s->states < 1) return "states must be 1 or more";
    if (s->tokens < 0 || s->tokens > INT32_MAX) return "tokens must be 0..2^31 - 1";
    if (s->n == 0 && s->tokens > 0) return "tokens without sequences";
    if (!known(s->dtype)) return "dtype must be RN_F32 or RN_BF16";
    const int64_t bc = (int64_t)s->groups * s->states;
    if (s->tokens > 1 && (s->u_stride < s->channels || s->dt_stride < s->channels || s->b_stride < bc || s->c_stride < bc))
        return "a token stride is smaller than its token";
    if (s->tokens > 1 && (s->u_stride >= kMaxStride || s->dt_stride >= kMaxStride || s->b_stride >= kMaxStride ||
                          s->c_stride >= kMaxStride))
        return "token strides must be below 2^23";
    return nullptr;
}

bool too_many_states(const rn_scan_shape *s) { return s->states > RN_SCAN_MAX_STATES; }

struct ScanSizes {
    int64_t blocks, chunks, walkers;
    int log_chunk;
    size_t kept, packed, ends, sums;      // bytes
    size_t part_bc, part_a, part_d;
};

ScanSizes scan_sizes(const rn_scan_shape *s, bool backward) {
    ScanSizes z{};
    const size_t row = (size_t)s->channels * 4, states = row * s->states, own = row * ((s->states + 3) / 4 * 4);
    z.blocks = scan_blocks(s->channels, s->groups);
    z.log_chunk = scan_log_chunk(s->tokens, s->n, s->channels, s->groups, backward);
    z.chunks = (s->tokens >> z.log_chunk) + s->n;
    z.walkers = scan_walkers(z.chunks, z.blocks);
    z.kept = round_up(scan_kept_slots(s->tokens, s->n) * own);
    // Calls may need it by the address of bfloat16 b and c, which is not known here.
    if (const int padded = scan_padded(s->states); s->dtype == RN_BF16 || padded != s->states)
        z.packed = round_up((size_t)s->tokens * s->groups * 2 * padded * 4);
    const size_t ends = scan_ends(s->tokens, z.log_chunk);
    z.ends = round_up(ends * own), z.sums = round_up(ends * row);
    if (backward) {
        z.part_bc = round_up((size_t)z.blocks * s->tokens * 2 * s->states * 4);
        z.part_a = round_up(z.walkers * states), z.part_d = round_up(z.walkers * 2 * row);
    }
    return z;
}

size_t scan_bytes(const ScanSizes &z) {
    return z.packed + z.ends + z.sums + z.part_bc + z.part_a + z.part_d + kAlign;
}

bool is_input(const rn_scan_inputs *in, const void *p) {
    return p && (p == in->u || p == in->dt || p == in->b || p == in->c || p == in->z);
}

bool on_16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

rn_status check_scan(const rn_scan_shape *s, const rn_scan_inputs *in) {
    if (const char *why = bad_scan(s)) return fail(RN_EINVAL, why);
    if (too_many_states(s)) return fail(RN_EUNSUPPORTED, "states above 64 have no kernel");
    if (!in) return fail(RN_EINVAL, "the inputs are NULL");
    if (s->tokens > 0 && (!in->u || !in->dt || !in->b || !in->c)) return fail(RN_EINVAL, "u, dt, b and c must not be NULL");
    if (!in->a) return fail(RN_EINVAL, "a must not be NULL");
    if (in->z && s->tokens > 1 && s->z_stride < s->channels) return fail(RN_EINVAL, "a token stride is smaller than its token");
    if (in->z && s->tokens > 1 && s->z_stride >= kMaxStride) return fail(RN_EINVAL, "token strides must be below 2^23");
    return RN_OK;
}

ScanArgs scan_args(const rn_scan_shape *s, const rn_scan_inputs *in, const int32_t *seq_off, const ScanSizes &z,
                   void *scratch) {
    ScanArgs a{};
    a.n = s->n, a.channels = s->channels, a.groups = s->groups, a.states = s->states, a.softplus = s->softplus;
    a.tokens = s->tokens;
    a.u = in->u, a.dt = in->dt, a.b = in->b, a.c = in->c, a.z = in->z;
    a.us = s->u_stride, a.dts = s->dt_stride, a.bs = s->b_stride, a.cs = s->c_stride, a.zs = in->z ? s->z_stride : 0;
    a.a = in->a, a.d = in->d, a.dt_bias = in->dt_bias;
    a.off = seq_off;
    a.whole_states = s->states % 4 == 0 && on_16(a.a);
    a.even = s->n > 0 ? (int)(s->tokens / s->n) : 0;
    a.blocks = z.blocks, a.log_chunk = z.log_chunk, a.chunks = z.chunks, a.walkers = z.walkers;
    a.parts = (seq_off || s->n == 0 ? s->tokens : a.even) > a.chunk();
    a.padded = scan_padded(s->states);
    char *at = static_cast<char *>(scratch);
    a.packed = reinterpret_cast<float *>(at);
    a.ends = reinterpret_cast<float *>(at + z.packed);
    a.sums = reinterpret_cast<float *>(at + z.packed + z.ends);
    return a;
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

rn_status reuse_ops_rms_norm(int64_t rows, int32_t width, const void *x, int64_t x_stride, rn_dtype dtype,
                             const void *residual, int64_t residual_stride, const float *weight, float eps, void *y,
                             void *q, float *scales, void *total, float *rstd, void *stream) {
    if (rows < 0 || rows > kMaxRows || width < 1 || width > kMaxWidth)
        return fail(RN_EINVAL, "rows must be 0..2^40 and width 1..2^30");
    if (!known(dtype)) return fail(RN_EINVAL, "dtype must be RN_F32 or RN_BF16");
    if (!(eps >= 0.f)) return fail(RN_EINVAL, "eps must be 0 or more");
    if (total && !residual) return fail(RN_EINVAL, "without a residual there is no total: it must be NULL");
    if (rows == 0) return RN_OK;
    if (!x) return fail(RN_EINVAL, "x must not be NULL");
    if (!y && !q) return fail(RN_EINVAL, "y and q must not both be NULL");
    if (!q != !scales) return fail(RN_EINVAL, "q and scales go together: one of them is NULL");
    if (rows > 1 && (x_stride < width || (residual && residual_stride < width)))
        return fail(RN_EINVAL, "a row stride is smaller than its row");
    if (y && y == total) return fail(RN_EINVAL, "y and total must be two arrays");
    if (rows > 1 && (((y == x || total == x) && x_stride != width) ||
                     (residual && (y == residual || total == residual) && residual_stride != width)))
        return fail(RN_EINVAL, "a result lies over an input that is not contiguous");
    RmsArgs a{};
    a.rows = rows, a.width = width;
    a.x = x, a.residual = residual;
    a.xs = x_stride, a.rs = residual ? residual_stride : 0;
    a.weight = weight, a.eps = eps;
    a.y = y, a.q = static_cast<uint8_t *>(q), a.scales = scales, a.total = total, a.rstd = rstd;
    return launched(launch_rms(a, dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

size_t reuse_ops_rms_norm_backward_scratch_bytes(int64_t rows, int32_t width) {
    if (rows < 0 || rows > kMaxRows || width < 1 || width > kMaxWidth) return 0;
    return round_up((size_t)norm_blocks(rows, width) * (size_t)width * 4);
}

rn_status reuse_ops_rms_norm_backward(int64_t rows, int32_t width, const void *dy, int64_t dy_stride,
                                      const void *total, int64_t total_stride, rn_dtype dtype, const float *weight,
                                      const float *rstd, const void *dtotal, int64_t dtotal_stride, void *dx,
                                      float *dweight, int32_t accumulate, void *scratch, size_t scratch_bytes,
                                      void *stream) {
    if (rows < 0 || rows > kMaxRows || width < 1 || width > kMaxWidth)
        return fail(RN_EINVAL, "rows must be 0..2^40 and width 1..2^30");
    if (!known(dtype)) return fail(RN_EINVAL, "dtype must be RN_F32 or RN_BF16");
    if (rows == 0 && !dweight) return RN_OK;
    if (rows > 0 && (!dy || !total || !rstd || !dx)) return fail(RN_EINVAL, "dy, total, rstd and dx must not be NULL");
    if (rows > 1 && (dy_stride < width || total_stride < width || (dtotal && dtotal_stride < width)))
        return fail(RN_EINVAL, "a row stride is smaller than its row");
    if (rows > 1 && ((dx == dy && dy_stride != width) || (dx == total && total_stride != width) ||
                     (dx == dtotal && dtotal_stride != width)))
        return fail(RN_EINVAL, "a result lies over an input that is not contiguous");
    if (dweight) {
        if (!scratch) return fail(RN_EINVAL, "scratch is NULL");
        if (misaligned(scratch)) return fail(RN_EINVAL, "scratch must be 256-byte aligned");
        const size_t need = reuse_ops_rms_norm_backward_scratch_bytes(rows, width);
        if (scratch_bytes < need) return need_bytes("scratch", need);
    }
    RmsArgs a{};
    a.rows = rows, a.width = width;
    a.x = total, a.dy = dy, a.dtotal = dtotal, a.y = dx;
    a.xs = total_stride, a.dys = dy_stride, a.dts = dtotal ? dtotal_stride : 0;
    a.weight = weight, a.rstd = const_cast<float *>(rstd);
    a.blocks = rows > 0 ? norm_blocks(rows, width) : 0;
    a.part = dweight ? static_cast<float *>(scratch) : nullptr;
    a.dweight = dweight, a.accumulate = accumulate;
    return launched(launch_rms_backward(a, dtype == RN_BF16, static_cast<hipStream_t>(stream)));
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

size_t reuse_ops_log_probs_scratch_bytes(int32_t n, int32_t vocab, int32_t top) {
    if (bad_logp(n, vocab, top)) return 0;
    size_t most = 0;
    for (const bool bf16 : {false, true}) {
        const size_t parts = (size_t)logp_parts(n, vocab, top, bf16);
        const size_t need = parts > 1 ? round_up(n * parts * 12) + round_up(n * parts * top * 8) : 0;
        if (need > most) most = need;
    }
    return most < kAlign ? kAlign : most;
}

rn_status reuse_ops_log_probs(int32_t n, int32_t vocab, const void *logits, int64_t stride, rn_dtype dtype,
                              const int32_t *tokens, float temperature, int32_t top, float *logprobs, float *entropy,
                              int32_t *top_tokens, float *top_logprobs, float *stats, void *scratch,
                              size_t scratch_bytes, void *stream) {
    if (const char *why = bad_logp(n, vocab, top)) return fail(RN_EINVAL, why);
    if (!known(dtype)) return fail(RN_EINVAL, "dtype must be RN_F32 or RN_BF16");
    if (bad_temperature(temperature)) return fail(RN_EINVAL, "temperature must be above 0 and finite");
    if (n == 0) return RN_OK;
    if (!logits || !tokens) return fail(RN_EINVAL, "logits and tokens must not be NULL");
    if (top > 0 && (!top_tokens || !top_logprobs)) return fail(RN_EINVAL, "top_tokens and top_logprobs must not be NULL");
    if (n > 1 && stride < vocab) return fail(RN_EINVAL, "the row stride is smaller than a row");
    if (!scratch) return fail(RN_EINVAL, "scratch is NULL");
    if (misaligned(scratch)) return fail(RN_EINVAL, "scratch must be 256-byte aligned");
    const size_t need = reuse_ops_log_probs_scratch_bytes(n, vocab, top);
    if (scratch_bytes < need) return need_bytes("scratch", need);
    LogpArgs a = logp_args(n, vocab, logits, stride, tokens, temperature, stats);
    a.top = top;
    a.logprobs = logprobs, a.entropy = entropy, a.top_tokens = top_tokens, a.top_logprobs = top_logprobs;
    a.parts = logp_parts(n, vocab, top, dtype == RN_BF16);
    a.part_sums = static_cast<float *>(scratch);
    a.part_keys = reinterpret_cast<uint64_t *>(static_cast<char *>(scratch) + round_up((size_t)n * a.parts * 12));
    return launched(launch_logp(a, dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_log_probs_backward(int32_t n, int32_t vocab, const void *logits, int64_t stride, rn_dtype dtype,
                                       const int32_t *tokens, float temperature, const float *stats,
                                       const float *dlogprobs, const float *dentropy, void *dlogits,
                                       int64_t dlogits_stride, void *stream) {
    if (const char *why = bad_logp(n, vocab, 0)) return fail(RN_EINVAL, why);
    if (!known(dtype)) return fail(RN_EINVAL, "dtype must be RN_F32 or RN_BF16");
    if (bad_temperature(temperature)) return fail(RN_EINVAL, "temperature must be above 0 and finite");
    if (n == 0) return RN_OK;
    if (!logits || !tokens || !stats || !dlogits)
        return fail(RN_EINVAL, "logits, tokens, stats and dlogits must not be NULL");
    if (n > 1 && (stride < vocab || dlogits_stride < vocab))
        return fail(RN_EINVAL, "the row stride is smaller than a row");
    if (n > 1 && dlogits == logits && dlogits_stride != stride)
        return fail(RN_EINVAL, "dlogits over logits must have the same stride");
    LogpArgs a = logp_args(n, vocab, logits, stride, tokens, temperature, const_cast<float *>(stats));
    a.dlogprobs = dlogprobs, a.dentropy = dentropy, a.dlogits = dlogits, a.dstride = dlogits_stride;
    return launched(launch_logp_backward(a, dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_causal_conv_step(const rn_conv_shape *shape, const void *x, const float *weight, const float *bias,
                                     const int32_t *ids, int32_t slots, void *window, void *out, void *stream) {
    if (const char *why = bad_conv(shape)) return fail(RN_EINVAL, why);
    if (shape->tokens != shape->n) return fail(RN_EINVAL, "a step takes one token a stream: tokens must be n");
    if (slots < 0 || (!ids && slots < shape->n)) return fail(RN_EINVAL, "fewer slots than streams");
    if (shape->n == 0) return RN_OK;
    if (!x || !weight || !out || (shape->taps > 1 && slots > 0 && !window))
        return fail(RN_EINVAL, "x, weight, window and out must not be NULL");
    if (out == x && shape->n > 1 && shape->x_stride != shape->channels)
        return fail(RN_EINVAL, "a result lies over an input that is not contiguous");
    if (out == window) return fail(RN_EINVAL, "out and the windows must be two arrays");
    CausalArgs a = conv_args(shape, x, weight, bias);
    a.ids = ids, a.slots = slots, a.final_window = window, a.out = out;
    return launched(launch_causal_step(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_causal_conv(const rn_conv_shape *shape, const void *x, const float *weight, const float *bias,
                                const int32_t *seq_off, const void *window, void *final_window, void *out,
                                void *stream) {
    if (const char *why = bad_conv(shape)) return fail(RN_EINVAL, why);
    if (!seq_off && shape->n > 0 && shape->tokens % shape->n)
        return fail(RN_EINVAL, "without seq_off, tokens must be a multiple of n");
    if (shape->n == 0) return RN_OK;
    if (shape->tokens > 0 && (!x || !weight || !out)) return fail(RN_EINVAL, "x, weight and out must not be NULL");
    if (out && out == x) return fail(RN_EINVAL, "out must not be x");
    if (final_window && final_window == window) return fail(RN_EINVAL, "the final windows must not be the first ones");
    CausalArgs a = conv_args(shape, x, weight, bias);
    a.off = seq_off, a.window = window, a.final_window = final_window, a.out = out;
    return launched(launch_causal(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

size_t reuse_ops_causal_conv_backward_scratch_bytes(const rn_conv_shape *shape) {
    if (bad_conv(shape)) return 0;
    return round_up((size_t)causal_parts(shape->tokens, shape->channels) * shape->channels * (shape->taps + 1) * 4) + kAlign;
}

rn_status reuse_ops_causal_conv_backward(const rn_conv_shape *shape, const void *x, const float *weight,
                                         const float *bias, const int32_t *seq_off, const void *window,
                                         const void *dout, const void *dfinal, void *dx, float *dweight, float *dbias,
                                         void *dwindow, void *scratch, size_t scratch_bytes, void *stream) {
    if (const char *why = bad_conv(shape)) return fail(RN_EINVAL, why);
    if (!seq_off && shape->n > 0 && shape->tokens % shape->n)
        return fail(RN_EINVAL, "without seq_off, tokens must be a multiple of n");
    if (shape->tokens > 0 && (!x || !dout || !dx)) return fail(RN_EINVAL, "x, dout and dx must not be NULL");
    if (!weight || !dweight || !dbias) return fail(RN_EINVAL, "weight, dweight and dbias must not be NULL");
    if (dx && (dx == x || dx == dout)) return fail(RN_EINVAL, "dx must be neither x nor dout");
    if (dwindow && (dwindow == dfinal || dwindow == window))
        return fail(RN_EINVAL, "dwindow must be neither dfinal nor the windows");
    if (!scratch) return fail(RN_EINVAL, "scratch is NULL");
    if (misaligned(scratch)) return fail(RN_EINVAL, "scratch must be 256-byte aligned");
    const size_t need = reuse_ops_causal_conv_backward_scratch_bytes(shape);
    if (scratch_bytes < need) return need_bytes("scratch", need);
    CausalArgs a = conv_args(shape, x, weight, bias);
    a.off = seq_off, a.window = window;
    a.dout = dout, a.dfinal = dfinal, a.dx = dx, a.dwindow = dwindow, a.dweight = dweight, a.dbias = dbias;
    a.part = static_cast<float *>(scratch);
    return launched(launch_causal_backward(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_scan_step(const rn_scan_shape *shape, const rn_scan_inputs *in, const int32_t *ids, int32_t slots,
                              float *state, void *out, void *stream) {
    if (rn_status s = check_scan(shape, in)) return s;
    if (shape->tokens != shape->n) return fail(RN_EINVAL, "a step takes one token a stream: tokens must be n");
    if (slots < 0 || (!ids && slots < shape->n)) return fail(RN_EINVAL, "fewer slots than streams");
    if (shape->n == 0) return RN_OK;
    if ((slots > 0 && !state) || !out) return fail(RN_EINVAL, "state and out must not be NULL");
    if (shape->n > 1 && ((out == in->u && shape->u_stride != shape->channels) ||
                         (out == in->dt && shape->dt_stride != shape->channels) ||
                         (out == in->z && shape->z_stride != shape->channels)))
        return fail(RN_EINVAL, "a result lies over an input that is not contiguous");
    if (out == in->b || out == in->c) return fail(RN_EINVAL, "out must be neither b nor c");
    ScanArgs a = scan_args(shape, in, nullptr, scan_sizes(shape, false), nullptr);
    a.whole_states = a.whole_states && on_16(state);
    a.ids = ids, a.slots = slots, a.final_state = state, a.out = out;
    return launched(launch_scan_step(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

size_t reuse_ops_scan_saved_bytes(const rn_scan_shape *shape) {
    if (bad_scan(shape) || too_many_states(shape)) return 0;
    return scan_sizes(shape, false).kept + kAlign;
}

size_t reuse_ops_scan_scratch_bytes(const rn_scan_shape *shape) {
    if (bad_scan(shape) || too_many_states(shape)) return 0;
    return scan_bytes(scan_sizes(shape, false));
}

size_t reuse_ops_scan_backward_scratch_bytes(const rn_scan_shape *shape) {
    if (bad_scan(shape) || too_many_states(shape)) return 0;
    return scan_bytes(scan_sizes(shape, true));
}

rn_status reuse_ops_scan_forward(const rn_scan_shape *shape, const rn_scan_inputs *in, const int32_t *seq_off,
                                 const float *state, float *final_state, void *out, void *saved, size_t saved_bytes,
                                 void *scratch, size_t scratch_bytes, void *stream) {
    if (rn_status s = check_scan(shape, in)) return s;
    if (!seq_off && shape->n > 0 && shape->tokens % shape->n)
        return fail(RN_EINVAL, "without seq_off, tokens must be a multiple of n");
    if (shape->n == 0) return RN_OK;
    if (shape->tokens > 0 && !out) return fail(RN_EINVAL, "out must not be NULL");
    if (misaligned(saved) || misaligned(scratch)) return fail(RN_EINVAL, "saved and scratch must be 256-byte aligned");
    const ScanSizes z = scan_sizes(shape, false);
    if (saved && saved_bytes < z.kept + kAlign) return need_bytes("saved", z.kept + kAlign);
    if (!scratch) return fail(RN_EINVAL, "scratch is NULL");
    const size_t need = scan_bytes(z);
    if (scratch_bytes < need) return need_bytes("scratch", need);
    if (shape->tokens > 0 && is_input(in, out)) return fail(RN_EINVAL, "out must not be one of the inputs");
    ScanArgs a = scan_args(shape, in, seq_off, z, scratch);
    a.whole_states = a.whole_states && on_16(state) && on_16(final_state);
    a.state = state, a.final_state = final_state, a.out = out, a.kept = static_cast<float *>(saved);
    return launched(launch_scan(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_scan_backward(const rn_scan_shape *shape, const rn_scan_inputs *in, const int32_t *seq_off,
                                  const void *saved, size_t saved_bytes, const void *dout, const float *dfinal,
                                  const rn_scan_grads *grads, void *scratch, size_t scratch_bytes, void *stream) {
    if (rn_status s = check_scan(shape, in)) return s;
    if (!seq_off && shape->n > 0 && shape->tokens % shape->n)
        return fail(RN_EINVAL, "without seq_off, tokens must be a multiple of n");
    if (!grads) return fail(RN_EINVAL, "the gradients are NULL");
    if (shape->tokens > 0 && (!dout || !grads->du || !grads->ddt || !grads->db || !grads->dc))
        return fail(RN_EINVAL, "dout and the gradients of u, dt, b and c must not be NULL");
    if (!grads->da) return fail(RN_EINVAL, "da must not be NULL");
    if (grads->dz && !in->z) return fail(RN_EINVAL, "dz without z");
    if (grads->dstate && grads->dstate == dfinal) return fail(RN_EINVAL, "dstate must not be dfinal");
    if (!saved || !scratch) return fail(RN_EINVAL, "saved and scratch must not be NULL");
    if (misaligned(saved) || misaligned(scratch)) return fail(RN_EINVAL, "saved and scratch must be 256-byte aligned");
    const ScanSizes z = scan_sizes(shape, true);
    if (saved_bytes < z.kept + kAlign) return need_bytes("saved", z.kept + kAlign);
    const size_t need = scan_bytes(z);
    if (scratch_bytes < need) return need_bytes("scratch", need);
    if (shape->tokens > 0)
        for (const void *p : {grads->du, grads->ddt, grads->db, grads->dc, grads->dz})
            if (is_input(in, p) || (p && p == dout)) return fail(RN_EINVAL, "a gradient lies over dout or an input");
    ScanArgs a = scan_args(shape, in, seq_off, z, scratch);
    a.whole_states = a.whole_states && on_16(dfinal) && on_16(grads->dstate);
    a.kept = static_cast<float *>(const_cast<void *>(saved));
    a.dout = dout, a.dfinal = dfinal;
    a.du = grads->du, a.ddt = grads->ddt, a.db = grads->db, a.dc = grads->dc, a.dz = grads->dz;
    a.da = grads->da, a.dd = grads->dd, a.ddt_bias = grads->ddt_bias, a.dstate = grads->dstate;
    char *at = static_cast<char *>(scratch) + z.packed + z.ends + z.sums;
    a.part_bc = reinterpret_cast<float *>(at);
    a.part_a = reinterpret_cast<float *>(at += z.part_bc);
    a.part_d = reinterpret_cast<float *>(at += z.part_a);
    return launched(launch_scan_backward(a, shape->dtype == RN_BF16, static_cast<hipStream_t>(stream)));
}

rn_status reuse_ops_delta_step(const rn_delta_shape *shape, const void *q, const void *k, const void *v,
                               const float *g, const float *beta, const int32_t *ids, int32_t slots, float *state,
                               void *out, void *stream) {
    if (rn_status s = check_delta(shape, q, k, v, g, beta)) return s;
    if (shape->tokens != shape->n) return fail(RN_EINVAL, "a step takes one token a stream: tokens must be n");
    if (slots < 0 || (!ids && slots < shape->n)) return fail(RN_EINVAL, "fewer slots than streams");
    if (shape->n == 0) return RN_OK;
    if ((slots > 0 && !state) || !out) return fail(RN_EINVAL, "state and out must not be NULL");
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
