// The gated delta rule over short sequences, token by token.
//
// Forward, with S the memory and a = e^g:
//   err = v - a S^T k,  S <- a S + k (beta err)^T,  out = scale S^T q.
// Backward, with D the gradient of the memory, from the last token on:
//   D <- D + scale q dout^T,  x = D^T k (the gradient of beta err),
//   D <- a (D - k (beta x)^T).
// The chunks' gradients (k_delta_bwd_chunk) follow from err, x and the first
// memory, however those were made.
//
// A wave owns 16 columns: lane l column l % 16, rows R (l / 16) .. + R - 1, in its
// registers from the first token to the last.  Sums over the rows are R
// multiply-adds and two swaps of lanes; nothing passes between waves but k and q,
// which the block stages in LDS, all tokens at once.  Bound by those
// multiply-adds (4 R a token and wave; 256 episodes of 16 tokens and 4 heads of
// 64 x 64 take 9 us of them) and by the memories' bytes.
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

// A sequence's tokens: k, scale q, the values (forward) or
// their gradients, e^g and beta.  Rows past dk and columns past dv are 0.
template <class T, int R>
__device__ inline void fill(const DeltaArgs &a, Stage<R> &s, const void *v, int64_t vs, int h, int hk, int v0, Span span) {
    const int at = span.begin, count = span.len;
    for (int i = threadIdx.x; i < count * Stage<R>::K; i += kWaves * 64) {
        const int t = i / Stage<R>::K, d = i % Stage<R>::K;
        const bool in = d < a.dk;
        s.k[t][d] = in ? load<T>(a.k, (int64_t)(at + t) * a.ks + hk * a.dk + d) : 0.f;
        s.q[t][d] = in ? load<T>(a.q, (int64_t)(at + t) * a.qs + hk * a.dk + d) * a.scale : 0.f;
    }
    for (int i = threadIdx.x; i < count * kWaves * 16; i += kWaves * 64) {
        const int t = i / (kWaves * 16), c = i % (kWaves * 16);
        s.v[t][c] = v0 + c < a.dv ? load<T>(v, (int64_t)(at + t) * vs + h * a.dv + v0 + c) : 0.f;
    }
    if ((int)threadIdx.x < count) {
        const int64_t i = (int64_t)(at + threadIdx.x) * a.hv + h;
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

// A head's memory [dk][dv] at column v0 + r, this lane's R rows.
template <int R>
__device__ inline void load_memory(const DeltaArgs &a, const float *m, int row0, int col, float (&S)[R]) {
#pragma unroll
    for (int i = 0; i < R; ++i) S[i] = m && row0 + i < a.dk && col < a.dv ? m[(row0 + i) * a.dv + col] : 0.f;
}
template <int R>
__device__ inline void store_memory(const DeltaArgs &a, float *m, int row0, int col, const float (&S)[R]) {
    if (col < a.dv)
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (row0 + i < a.dk) m[(row0 + i) * a.dv + col] = S[i];
}

template <class T, int R, bool SAVE>
__global__ __launch_bounds__(kWaves * 64) void k_delta_short(DeltaArgs a) {
    __shared__ __align__(16) Stage<R> st;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int seq = blockIdx.x / a.hv, h = blockIdx.x % a.hv, hk = h / (a.hv / a.hk);
    const Span span = span_of(a, seq);
    if (span.len > a.short_len) return;
    const int v0 = blockIdx.y * kWaves * 16, vc = wave * 16 + r, col = v0 + vc, row0 = g * R;
    const int64_t mem = ((int64_t)seq * a.hv + h) * a.dk * a.dv;
    float S[R];
    load_memory<R>(a, a.state ? a.state + mem : nullptr, row0, col, S);
    if constexpr (SAVE)
        if (span.len > 0)
            store_memory<R>(a, a.before + ((int64_t)slot_of(span, seq, 0) * a.hv + h) * a.dk * a.dv, row0, col, S);
    fill<T, R>(a, st, a.v, a.vs, h, hk, v0, span);
    __syncthreads();
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

template <class T, int R>
__global__ __launch_bounds__(kWaves * 64) void k_delta_short_bwd(DeltaArgs a) {
    __shared__ __align__(16) Stage<R> st;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int seq = blockIdx.x / a.hv, h = blockIdx.x % a.hv, hk = h / (a.hv / a.hk);
    const Span span = span_of(a, seq);
    if (span.len > a.short_len) return;
    const int v0 = blockIdx.y * kWaves * 16, vc = wave * 16 + r, col = v0 + vc, row0 = g * R;
    const int64_t mem = ((int64_t)seq * a.hv + h) * a.dk * a.dv;
    float D[R];
    load_memory<R>(a, a.dfinal ? a.dfinal + mem : nullptr, row0, col, D);
    fill<T, R>(a, st, a.dout, (int64_t)a.hv * a.dv, h, hk, v0, span);
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

template <class T, class F>
hipError_t by_rows(const DeltaArgs &a, F &&go) {
    if (a.n == 0) return hipSuccess;
    const dim3 grid(a.n * a.hv, (a.dv + kWaves * 16 - 1) / (kWaves * 16));
    if (a.dk <= 32) go(std::integral_constant<int, 8>{}, grid);
    else if (a.dk <= 64) go(std::integral_constant<int, 16>{}, grid);
    else go(std::integral_constant<int, 32>{}, grid);
    return hipGetLastError();
}

template <class T>
hipError_t forward(const DeltaArgs &a, hipStream_t s) {
    return by_rows<T>(a, [&](auto r, dim3 grid) {
        constexpr int R = decltype(r)::value;
        if (a.before) k_delta_short<T, R, true><<<grid, kWaves * 64, 0, s>>>(a);
        else k_delta_short<T, R, false><<<grid, kWaves * 64, 0, s>>>(a);
    });
}

template <class T>
hipError_t backward(const DeltaArgs &a, hipStream_t s) {
    return by_rows<T>(a, [&](auto r, dim3 grid) {
        k_delta_short_bwd<T, decltype(r)::value><<<grid, kWaves * 64, 0, s>>>(a);
    });
}

}  // namespace

hipError_t launch_delta_short_forward(const DeltaArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}
hipError_t launch_delta_short_backward(const DeltaArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? backward<bf16_t>(a, s) : backward<float>(a, s);
}

}  // namespace rn
