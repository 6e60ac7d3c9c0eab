// The gated delta rule over short sequences, token by token.
//
// Forward, with S the memory and a = e^g:
//   err = v - a S^T k,  S <- a S + k (beta err)^T,  out = scale S^T q.
// Backward, with D the gradient of the memory, from the last token on:
//   D <- D + scale q dout^T,  x = D^T k (the gradient of beta err),
//   D <- a (D - k (beta x)^T).
// The inputs' gradients (k_delta_short_grad) follow from err, x and the first
// memory by the sums over pairs of tokens that are written down in rn_delta_bwd.hip.
//
// A wave owns 16 columns: lane l column l % 16, rows R (l / 16) .. + R - 1, in its
// registers from the first token to the last.  Sums over the rows are R
// multiply-adds and two swaps of lanes; nothing passes between waves but k and q,
// which the block stages in LDS, all tokens at once.  Bound by those
// multiply-adds (4 R a token and wave; 256 episodes of 16 tokens and 4 heads of
// 64 x 64 take 9 us of them) and by the memories' bytes: those episodes take 20 us
// for 50 MB forward and 19 back.
#include "rn_delta.hpp"

namespace rn {
namespace {

using namespace ops;

constexpr int kWaves = 4;

// Sum over the four lanes that share a column.
__device__ inline float over_rows(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <int R>
struct Stage {
    static constexpr int K = 4 * R;
    float k[kShort][K], q[kShort][K], v[kShort][kWaves * 16];
    float a[kShort], beta[kShort];
};

// A sequence's tokens: k, scale q, the values (forward) or their gradients, e^g
// and beta.  Rows past dk and columns past dv are 0.  A pass's loads are all on
// their way before the first is waited for: one pass does for 16 tokens up to dk 64.
// VEC: dk, dv and strides multiples of 4, rows on that.
template <class T, int R, bool VEC>
__device__ inline void fill(const DeltaArgs &a, Stage<R> &s, const void *v, int64_t vs, int h, int hk, int v0, Span span) {
    constexpr int PER = VEC ? 4 : 1, TP = kWaves * 64 / R;              // tokens of k and q a pass
    const __amdgpu_buffer_rsrc_t pk = rsrc_of(static_cast<const T *>(a.k) + (int64_t)span.begin * a.ks + hk * a.dk);
    const __amdgpu_buffer_rsrc_t pq = rsrc_of(static_cast<const T *>(a.q) + (int64_t)span.begin * a.qs + hk * a.dk);
    const __amdgpu_buffer_rsrc_t pv = rsrc_of(static_cast<const T *>(v) + (int64_t)span.begin * vs + h * a.dv + v0);
    const int d = threadIdx.x % R * 4, c = threadIdx.x % 16 * 4;
    for (int p = 0; p * (TP < 16 ? TP : 16) < span.len; ++p) {
        const int tk = p * TP + threadIdx.x / R, tv = p * 16 + threadIdx.x / 16;
        Pack<T, PER> fk[4 / PER], fq[4 / PER], fv[4 / PER];
#pragma unroll
        for (int e = 0; e < 4; e += PER) {
            const bool in = tk < span.len && d + e < a.dk;
            fk[e / PER] = load_if<Pack<T, PER>>(in, pk, sizeof(T) * (tk * (uint32_t)a.ks + d + e));
            fq[e / PER] = load_if<Pack<T, PER>>(in, pq, sizeof(T) * (tk * (uint32_t)a.qs + d + e));
            fv[e / PER] = load_if<Pack<T, PER>>(tv < span.len && v0 + c + e < a.dv, pv, sizeof(T) * (tv * (uint32_t)vs + c + e));
        }
        f32x4 k, q, w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            k[e] = to_float(fk[e / PER].v[e % PER]), q[e] = to_float(fq[e / PER].v[e % PER]) * a.scale;
            w[e] = to_float(fv[e / PER].v[e % PER]);
        }
        if (tk < kShort) {
            *reinterpret_cast<f32x4 *>(&s.k[tk][d]) = k;
            *reinterpret_cast<f32x4 *>(&s.q[tk][d]) = q;
        }
        if (tv < kShort) *reinterpret_cast<f32x4 *>(&s.v[tv][c]) = w;
    }
    if ((int)threadIdx.x < span.len) {
        const int64_t i = (int64_t)(span.begin + threadIdx.x) * a.hv + h;
        s.a[threadIdx.x] = expf(a.g[i]);
        s.beta[threadIdx.x] = a.beta[i];
    }
}

template <int R>
__device__ inline void row_of(const float *p, float (&f)[R]) {      // R consecutive floats, on 16 bytes
#pragma unroll
    for (int i = 0; i < R; i += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i + j] = v[j];
    }
}

template <int R>
__device__ inline float dot(const float (&x)[R], const float (&y)[R]) {
    float p[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < R; ++i) p[i % 4] = fmaf(x[i], y[i], p[i % 4]);
    return (p[0] + p[1]) + (p[2] + p[3]);
}

// A head's memory [dk][dv] at one column, this lane's R rows.
template <int R>
__device__ inline void load_memory(const DeltaArgs &a, const float *m, int row0, int col, float (&S)[R]) {
    const __amdgpu_buffer_rsrc_t p = rsrc_of(m);
#pragma unroll
    for (int i = 0; i < R; ++i) S[i] = load_if<float>(m && row0 + i < a.dk && col < a.dv, p, 4 * ((row0 + i) * a.dv + col));
}
template <int R>
__device__ inline void store_memory(const DeltaArgs &a, float *m, int row0, int col, const float (&S)[R]) {
    const __amdgpu_buffer_rsrc_t p = rsrc_of(m);
#pragma unroll
    for (int i = 0; i < R; ++i) store_if(row0 + i < a.dk && col < a.dv, p, 4 * ((row0 + i) * a.dv + col), S[i]);
}

template <class T, int R, bool SAVE, bool VEC>
__global__ __launch_bounds__(kWaves * 64) void k_delta_short(DeltaArgs a) {
    __shared__ __align__(16) Stage<R> st;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int seq = blockIdx.y, h = blockIdx.x % a.hv, hk = h / (a.hv / a.hk);
    const Span span = span_of(a, seq);
    if (span.len > a.short_len) return;
    const int v0 = blockIdx.x / a.hv * kWaves * 16, vc = wave * 16 + r, col = v0 + vc, row0 = g * R;
    const int64_t mem = ((int64_t)seq * a.hv + h) * a.dk * a.dv;
    float S[R];
    load_memory<R>(a, a.state ? a.state + mem : nullptr, row0, col, S);
    fill<T, R, VEC>(a, st, a.v, a.vs, h, hk, v0, span);
    __syncthreads();
    if constexpr (SAVE)
        if (span.len > 0)
            store_memory<R>(a, a.before + ((int64_t)kept_slot_of(span.begin, seq) * a.hv + h) * a.dk * a.dv, row0, col, S);
    for (int t = 0; t < span.len; ++t) {
        float k[R], q[R];
        row_of<R>(&st.k[t][row0], k);
        const float e = st.a[t], err = st.v[t][vc] - e * over_rows(dot<R>(k, S)), w = st.beta[t] * err;
        row_of<R>(&st.q[t][row0], q);
#pragma unroll
        for (int i = 0; i < R; ++i) S[i] = fmaf(e, S[i], k[i] * w);
        const float o = over_rows(dot<R>(q, S));
        const int64_t to = ((int64_t)(span.begin + t) * a.hv + h) * a.dv + col;
        if (col < a.dv) {
            if (g == 0) static_cast<T *>(a.out)[to] = from_float<T>(o);
            if (SAVE && g == 1) a.err[to] = err;
        }
    }
    if (a.final_state) store_memory<R>(a, a.final_state + mem, row0, col, S);
}

template <class T, int R, bool VEC>
__global__ __launch_bounds__(kWaves * 64) void k_delta_short_bwd(DeltaArgs a) {
    __shared__ __align__(16) Stage<R> st;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int seq = blockIdx.y, h = blockIdx.x % a.hv, hk = h / (a.hv / a.hk);
    const Span span = span_of(a, seq);
    if (span.len > a.short_len) return;
    const int v0 = blockIdx.x / a.hv * kWaves * 16, vc = wave * 16 + r, col = v0 + vc, row0 = g * R;
    const int64_t mem = ((int64_t)seq * a.hv + h) * a.dk * a.dv;
    float D[R];
    load_memory<R>(a, a.dfinal ? a.dfinal + mem : nullptr, row0, col, D);
    fill<T, R, VEC>(a, st, a.dout, (int64_t)a.hv * a.dv, h, hk, v0, span);
    __syncthreads();
    for (int t = span.len - 1; t >= 0; --t) {
        float k[R], q[R];
        row_of<R>(&st.q[t][row0], q);
        row_of<R>(&st.k[t][row0], k);
        const float o = st.v[t][vc], e = st.a[t];
#pragma unroll
        for (int i = 0; i < R; ++i) D[i] = fmaf(q[i], o, D[i]);
        const float x = over_rows(dot<R>(k, D)), w = st.beta[t] * x;
#pragma unroll
        for (int i = 0; i < R; ++i) D[i] = e * fmaf(-k[i], w, D[i]);
        if (g == 0 && col < a.dv) a.dwrite[((int64_t)(span.begin + t) * a.hv + h) * a.dv + col] = x;
    }
    if (a.dstate) store_memory<R>(a, a.dstate + mem, row0, col, D);
}

// The inputs' gradients of a sequence that is one chunk, all of it on the float32
// matrix cores: operands of 16 or 32 tokens are too few for the split into bf16
// planes to pay.  A block takes a sequence and a key head and adds the value heads
// that share it; wave w owns the memory's row tiles w, w + 4.  The tokens' rows lie
// in LDS, S and dS' are read once, as operands as they lie in memory.  Bound by
// those bytes: 256 episodes of 16 tokens and 4 heads of 64 x 64, 24 us for 67 MB, 2.8
// TB/s (56 us by chunks, whose operands it does without).
template <class T, int NT, int TT, bool VEC>
__global__ __launch_bounds__(kWaves * 64, NT * TT == 1 ? 4 : 2) void k_delta_short_grad(DeltaArgs a) {
    constexpr int rows = 16 * TT;                       // tokens there is room for
    extern __shared__ __align__(16) float lds[];
    __shared__ double cs[64];
    __shared__ float beta[64], dc[kWaves][kShort], extra[kWaves];
    const int seq = blockIdx.y, hk = blockIdx.x, group = a.hv / a.hk;
    const Span span = span_of(a, seq);
    const int len = span.len;
    if (len == 0 || len > a.short_len) return;
    const int dvp = (a.dv + 31) / 32 * 32, ldV = dvp + 4, ldX = rows + 4;
    constexpr int KP = NT * 64, ldK = KP + 4;
    float *sO = lds, *sW = sO + rows * ldV, *sV = sW + rows * ldV;      // dO, dV', V'
    float *sK = sV + rows * ldV, *sQ = sK + rows * ldK;
    float *x = sQ + rows * ldK, *y = x + rows * ldX;                    // [i][j] of dP e and dL e
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int tiles = (len + 15) / 16;
    const Chunk c{seq, span.begin, len, len, true};
    constexpr int PER = VEC ? 4 : 1;                    // VEC: dk, dv and strides multiples of 4, rows on that
    {
        const __amdgpu_buffer_rsrc_t pk = rsrc_of(static_cast<const T *>(a.k) + (int64_t)c.begin * a.ks + hk * a.dk);
        const __amdgpu_buffer_rsrc_t pq = rsrc_of(static_cast<const T *>(a.q) + (int64_t)c.begin * a.qs + hk * a.dk);
        constexpr int TP = kWaves * 64 * 4 / KP;        // tokens a pass
        const int d = threadIdx.x % (KP / 4) * 4;
#pragma unroll
        for (int t0 = 0; t0 < rows; t0 += TP) {
            const int t = t0 + threadIdx.x / (KP / 4);
            f32x4 k, q;
#pragma unroll
            for (int e = 0; e < 4; e += PER) {
                const bool in = t < len && d + e < a.dk;
                const auto fk = load_if<Pack<T, PER>>(in, pk, sizeof(T) * (t * (uint32_t)a.ks + d + e));
                const auto fq = load_if<Pack<T, PER>>(in, pq, sizeof(T) * (t * (uint32_t)a.qs + d + e));
#pragma unroll
                for (int j = 0; j < PER; ++j) k[e + j] = to_float(fk.v[j]), q[e + j] = to_float(fq.v[j]);
            }
            *reinterpret_cast<f32x4 *>(sK + t * ldK + d) = k;
            *reinterpret_cast<f32x4 *>(sQ + t * ldK + d) = q;
        }
    }
    const auto mfma = [](float u, float v, f32x4 &acc) { acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u, v, acc, 0, 0, 0); };
    f32x4 tq[TT][NT], tk[TT][NT];                         // over the value heads
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) tq[t][n] = tk[t][n] = f32x4{};
    for (int h = hk * group; h < (hk + 1) * group; ++h) {
        const int64_t mem = (int64_t)a.dk * a.dv, row0 = ((int64_t)c.begin * a.hv + h) * a.dv;
        const __amdgpu_buffer_rsrc_t pS = rsrc_of(a.before + ((int64_t)kept_slot_of(span.begin, seq) * a.hv + h) * mem);
        const __amdgpu_buffer_rsrc_t pD = rsrc_of(a.dfinal ? a.dfinal + ((int64_t)seq * a.hv + h) * mem : a.before);
        struct Step {                                   // 32 columns of S and of dS'
            Pack<float, PER> s[NT][2][4 / PER], d[NT][2][4 / PER];
        } next;
        const auto fetch = [&](int v0) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int o = 0; o < 2; ++o)
#pragma unroll
                    for (int e = 0; e < 4; e += PER) {
                        const int d = (wave + 4 * n) * 16 + r, v = v0 + o * 16 + g * 4 + e;
                        const bool in = d < a.dk && v < a.dv;
                        next.s[n][o][e / PER] = load_if<Pack<float, PER>>(in, pS, 4 * (d * a.dv + v));
                        next.d[n][o][e / PER] = load_if<Pack<float, PER>>(in && a.dfinal, pD, 4 * (d * a.dv + v));
                    }
        };
        fetch(0);
        __syncthreads();                                // the last head's rows have been read
        if (wave == 0) {
            cs[lane] = decay_sums(a, c, h);
            beta[lane] = lane < len ? a.beta[(int64_t)(c.begin + lane) * a.hv + h] : 0.f;
        }
        // Eight threads a token: the rows, dv and dbeta.
        const int token = threadIdx.x >> 3;
        if (token < rows) {
            const __amdgpu_buffer_rsrc_t pO = rsrc_of(static_cast<const T *>(a.dout) + row0), pW = rsrc_of(a.dwrite + row0);
            const __amdgpu_buffer_rsrc_t pE = rsrc_of(a.err + row0), pV = rsrc_of(static_cast<T *>(a.dval) + row0);
            const uint32_t row = token * (uint32_t)(a.hv * a.dv);
            const float b = token < len ? a.beta[(int64_t)(c.begin + token) * a.hv + h] : 0.f;
            float db = 0.f;
            for (int v0 = (threadIdx.x & 7) * 4; v0 < dvp; v0 += 64) {
                Pack<T, PER> to[2][4 / PER];
                Pack<float, PER> tw[2][4 / PER], te[2][4 / PER];
#pragma unroll
                for (int u = 0; u < 2; ++u)             // all on their way before the first is used
#pragma unroll
                    for (int i = 0; i < 4; i += PER) {
                        const int v = v0 + 32 * u + i;
                        const bool in = token < len && v < a.dv;
                        to[u][i / PER] = load_if<Pack<T, PER>>(in, pO, sizeof(T) * (row + v));
                        tw[u][i / PER] = load_if<Pack<float, PER>>(in, pW, 4 * (row + v));
                        te[u][i / PER] = load_if<Pack<float, PER>>(in, pE, 4 * (row + v));
                    }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    f32x4 o, w, e;
#pragma unroll
                    for (int i = 0; i < 4; i += PER) {
                        const int v = v0 + 32 * u + i;
                        Pack<T, PER> dv;
#pragma unroll
                        for (int j = 0; j < PER; ++j) {
                            o[i + j] = to_float(to[u][i / PER].v[j]), w[i + j] = tw[u][i / PER].v[j], e[i + j] = te[u][i / PER].v[j];
                            db = fmaf(w[i + j], e[i + j], db);
                            e[i + j] *= b;
                            dv.v[j] = from_float<T>(w[i + j] * b);
                        }
                        store_if(token < len && v < a.dv, pV, sizeof(T) * (row + v), dv);
                    }
                    if (v0 + 32 * u < dvp) {
                        const int at = token * ldV + v0 + 32 * u;
                        *reinterpret_cast<f32x4 *>(sO + at) = o;
                        *reinterpret_cast<f32x4 *>(sW + at) = w;
                        *reinterpret_cast<f32x4 *>(sV + at) = e;
                    }
                }
            }
#pragma unroll
            for (int s = 1; s < 8; s <<= 1) db += __shfl_xor(db, s);
            if ((threadIdx.x & 7) == 0 && token < len) a.dbeta[(int64_t)(c.begin + token) * a.hv + h] = db;
        }
        __syncthreads();
        f32x4 gq[TT][NT], gr[TT][NT], gw[TT][NT];
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int n = 0; n < NT; ++n) gq[t][n] = gr[t][n] = gw[t][n] = f32x4{};
        float dot = 0.f;
        for (int v0 = 0; v0 < dvp; v0 += 32) {
            const Step now = next;
            fetch(v0 + 32);                             // nothing past the last column
#pragma unroll
            for (int o = 0; o < 2; ++o)
#pragma unroll
                for (int t = 0; t < TT; ++t)
                    if (t < tiles) {
                        const int at = (t * 16 + r) * ldV + v0 + o * 16 + g * 4;
                        const f32x4 fo = *reinterpret_cast<const f32x4 *>(sO + at), fw = *reinterpret_cast<const f32x4 *>(sW + at);
                        const f32x4 fv = *reinterpret_cast<const f32x4 *>(sV + at);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float s = now.s[n][o][e / PER].v[e % PER], d = now.d[n][o][e / PER].v[e % PER];
                                mfma(fo[e], s, gq[t][n]);
                                mfma(fw[e], s, gr[t][n]);
                                mfma(fv[e], d, gw[t][n]);
                                if (t == 0) dot = fmaf(s, d, dot);
                            }
                    }
        }
        // The pairs of tokens: a tile of dP or of dL a job.
        for (int job = wave; job < (tiles == 1 ? 2 : 6); job += kWaves) {
            const bool write = job & 1;
            const int ti = job > 1, tj = job > 3;
            const float *p = (write ? sW : sO) + (ti * 16 + r) * ldV + g * 4, *q = sV + (tj * 16 + r) * ldV + g * 4;
            f32x4 acc{};
            for (int v = 0; v < dvp; v += 16) {
                const f32x4 u = *reinterpret_cast<const f32x4 *>(p + v), w = *reinterpret_cast<const f32x4 *>(q + v);
#pragma unroll
                for (int e = 0; e < 4; ++e) mfma(u[e], w[e], acc);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = ti * 16 + g * 4 + j, u = tj * 16 + r;
                const float d = u <= t ? decay(cs[t] - cs[u]) : 0.f;
                if (write) y[t * ldX + u] = u < t ? -beta[t] * acc[j] * d : 0.f;
                else x[t * ldX + u] = u <= t ? acc[j] * d * a.scale : 0.f;
            }
        }
        // The memory's part of the sums, before the pairs' is added.
        const double last = cs[len - 1];
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < TT; ++t)
            if (t < tiles)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = t * 16 + g * 4 + j;
                    const float grown = decay(cs[i]), left = decay(last - cs[i]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        gq[t][n][j] *= grown * a.scale;
                        gr[t][n][j] *= -beta[i] * grown;
                        gw[t][n][j] *= left;
                        sum = fmaf(gw[t][n][j], sK[i * ldK + (wave + 4 * n) * 16 + r], sum);
                    }
                }
        sum = fmaf(dot, decay(last), sum);
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
        if (lane == 0) extra[wave] = sum;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int kt = 0; kt < TT; ++kt)
                if (t < tiles && kt < tiles)
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const int k = kt * 16 + e + g;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const int d = (wave + 4 * n) * 16 + r;
                            const float fk = sK[k * ldK + d];
                            if (kt <= t) {              // rows i: reads
                                mfma(x[(t * 16 + r) * ldX + k], fk, gq[t][n]);
                                mfma(y[(t * 16 + r) * ldX + k], fk, gr[t][n]);
                            }
                            if (kt >= t) {              // columns j: writes
                                mfma(x[k * ldX + t * 16 + r], sQ[k * ldK + d], gw[t][n]);
                                mfma(y[k * ldX + t * 16 + r], fk, gw[t][n]);
                            }
                        }
                    }
#pragma unroll
        for (int t = 0; t < TT; ++t)
            if (t < tiles)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = t * 16 + g * 4 + j;
                    float s = 0.f;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const int at = i * ldK + (wave + 4 * n) * 16 + r;
                        s = fmaf(gq[t][n][j], sQ[at], s);
                        s = fmaf(gr[t][n][j] - gw[t][n][j], sK[at], s);
                        tq[t][n][j] += gq[t][n][j];
                        tk[t][n][j] += gr[t][n][j] + gw[t][n][j];
                    }
#pragma unroll
                    for (int o = 1; o < 16; o <<= 1) s += __shfl_xor(s, o);
                    if (r == 0) dc[wave][i] = s;
                }
        __syncthreads();
        if (wave == 0) {
            double s = 0.;
            if (lane < len)
#pragma unroll
                for (int w = 0; w < kWaves; ++w) s += dc[w][lane] + (lane == len - 1 ? extra[w] : 0.f);
#pragma unroll
            for (int d = 1; d < kShort; d <<= 1) {
                const double u = __shfl_down(s, d);
                if (lane + d < kShort) s += u;
            }
            if (lane < len) a.dg[(int64_t)(c.begin + lane) * a.hv + h] = (float)s;
        }
    }
    const __amdgpu_buffer_rsrc_t rq = rsrc_of(static_cast<T *>(a.dq) + ((int64_t)c.begin * a.hk + hk) * a.dk);
    const __amdgpu_buffer_rsrc_t rk = rsrc_of(static_cast<T *>(a.dkey) + ((int64_t)c.begin * a.hk + hk) * a.dk);
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int i = t * 16 + g * 4 + j, d = (wave + 4 * n) * 16 + r;
                const uint32_t at = i * (uint32_t)(a.hk * a.dk) + d;
                store_if(i < len && d < a.dk, rq, sizeof(T) * at, from_float<T>(tq[t][n][j]));
                store_if(i < len && d < a.dk, rk, sizeof(T) * at, from_float<T>(tk[t][n][j]));
            }
}

template <class T, class F>
hipError_t by_rows(const DeltaArgs &a, const void *v, int64_t vs, F &&go) {
    if (a.n == 0) return hipSuccess;
    const dim3 grid = walk_grid(a, kWaves * 16);
    const auto even = [](const void *p, int64_t stride) {
        return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0 && stride % 4 == 0;
    };
    const bool vec = a.dk % 4 == 0 && a.dv % 4 == 0 && even(a.k, a.ks) && even(a.q, a.qs) && even(v, vs);
    const auto rows = [&](auto vec_) {
        if (a.dk <= 32) go(std::integral_constant<int, 8>{}, vec_, grid);
        else if (a.dk <= 64) go(std::integral_constant<int, 16>{}, vec_, grid);
        else go(std::integral_constant<int, 32>{}, vec_, grid);
    };
    if (vec) rows(std::true_type{});
    else rows(std::false_type{});
    return hipGetLastError();
}

template <class T>
hipError_t forward(const DeltaArgs &a, hipStream_t s) {
    return by_rows<T>(a, a.v, a.vs, [&](auto r, auto vec, dim3 grid) {
        constexpr int R = decltype(r)::value;
        constexpr bool VEC = decltype(vec)::value;
        if (a.before) k_delta_short<T, R, true, VEC><<<grid, kWaves * 64, 0, s>>>(a);
        else k_delta_short<T, R, false, VEC><<<grid, kWaves * 64, 0, s>>>(a);
    });
}

template <class T>
hipError_t backward(const DeltaArgs &a, hipStream_t s) {
    const hipError_t walk = by_rows<T>(a, a.dout, (int64_t)a.hv * a.dv, [&](auto r, auto vec, dim3 grid) {
        k_delta_short_bwd<T, decltype(r)::value, decltype(vec)::value><<<grid, kWaves * 64, 0, s>>>(a);
    });
    if (walk != hipSuccess || a.n == 0) return walk;
    const auto even = [](const void *p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 4 == 0; };
    const bool vec = a.dk % 4 == 0 && even(a.k, a.ks) && even(a.q, a.qs) && even(a.dout, a.dv) && even(a.dval, 0) && even(a.dfinal, 0);
    const auto grad = [&](auto nt_, auto tt_, auto vec_) -> hipError_t {
        constexpr int NT = decltype(nt_)::value, TT = decltype(tt_)::value, rows = 16 * TT;
        const int dvp = (a.dv + 31) / 32 * 32;
        const size_t bytes = sizeof(float) * rows * (3 * (dvp + 4) + 2 * (NT * 64 + 4) + 2 * (rows + 4));
        auto *kernel = k_delta_short_grad<T, NT, TT, decltype(vec_)::value>;
        if (hipError_t e = allow_lds(kernel, bytes)) return e;
        kernel<<<dim3(a.hk, a.n), kWaves * 64, bytes, s>>>(a);
        return hipGetLastError();
    };
    const auto by_vec = [&](auto nt, auto tt) { return vec ? grad(nt, tt, std::true_type{}) : grad(nt, tt, std::false_type{}); };
    // Even sequences of up to 16 tokens need room for one tile of tokens.
    const auto by_tokens = [&](auto nt) {
        return !a.off && a.tokens <= (int64_t)16 * a.n ? by_vec(nt, std::integral_constant<int, 1>{})
                                                       : by_vec(nt, std::integral_constant<int, 2>{});
    };
    return a.dk <= 64 ? by_tokens(std::integral_constant<int, 1>{}) : by_tokens(std::integral_constant<int, 2>{});
}

}  // namespace

hipError_t launch_delta_short_forward(const DeltaArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}
hipError_t launch_delta_short_backward(const DeltaArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? backward<bf16_t>(a, s) : backward<float>(a, s);
}

}  // namespace rn
