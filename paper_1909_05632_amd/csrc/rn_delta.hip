// The gated delta rule: one token a stream (the step), and whole sequences.
//
//   S <- e^g S;  S <- S + beta k (v - S^T k)^T;  out = scale S^T q.
//
// Sequences are taken in chunks of 64 tokens.  With c the sums of g within the
// chunk, S the memory before it and V' the values as written, beta (v - S_t^T k),
//   (I + A) V' = beta (V - e^c K S),   A_ij = beta_i e^(ci - cj) k_i . k_j  (j < i),
//   O  = scale (e^c Q S + P V'),       P_ij = e^(ci - cj) q_i . k_j          (j <= i),
//   S' = e^(c64) S + (e^(c64 - c) K)^T V'.
// (I + A)^-1 and P do not depend on S: k_delta_prepare makes them for all chunks
// at once.  k_delta_walk then goes through a sequence's chunks in order; columns
// of S do not meet, so each block takes a head's 16 of them.
#include "rn_delta.hpp"

namespace rn {
namespace {

using namespace ops;

// ------------------------------------------------------------------ one token

// A block owns one stream's head.  Its memory is read once into registers and
// written once: VEC columns a thread, `lanes` threads across the columns, the
// 256 / lanes groups each with every such row.  Bound by HBM (the memory's
// 2 dk dv float32 outweigh all else).
template <class T, int VEC, int ROWS>
__global__ __launch_bounds__(256) void k_delta_step(DeltaArgs a, int lanes) {
    __shared__ float sq[RN_DELTA_MAX_DIM], sk[RN_DELTA_MAX_DIM];
    __shared__ float red[256 * VEC];
    const int head = blockIdx.x % a.hv, i = blockIdx.x / a.hv;
    const int slot = a.ids ? a.ids[i] : i;
    const int hk = head / (a.hv / a.hk);
    const int col = threadIdx.x % lanes, grp = threadIdx.x / lanes, groups = 256 / lanes;
    const bool mine = col * VEC < a.dv;
    T *out = static_cast<T *>(a.out) + ((int64_t)i * a.hv + head) * a.dv;
    if (slot < 0 || slot >= a.slots) {
        for (int c = threadIdx.x; c < a.dv; c += 256) out[c] = from_float<T>(0.f);
        return;
    }
    for (int c = threadIdx.x; c < a.dk; c += 256) {
        sq[c] = load<T>(a.q, i * a.qs + hk * a.dk + c) * a.scale;
        sk[c] = load<T>(a.k, i * a.ks + hk * a.dk + c);
    }
    float *S = a.final_state + ((int64_t)slot * a.hv + head) * a.dk * a.dv + col * VEC;
    Pack<float, VEC> s[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (mine && grp + groups * r < a.dk)
            s[r] = *reinterpret_cast<const Pack<float, VEC> *>(S + (grp + groups * r) * a.dv);
    const float decay = expf(a.g[(int64_t)i * a.hv + head]), beta = a.beta[(int64_t)i * a.hv + head];
    __syncthreads();
    float part[VEC];
    const auto sum_groups = [&](float (&v)[VEC]) {      // over the groups, for every thread
        __syncthreads();
#pragma unroll
        for (int j = 0; j < VEC; ++j) red[threadIdx.x * VEC + j] = v[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = 0.f;
        for (int g = 0; g < groups; ++g)
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] += red[(g * lanes + col) * VEC + j];
    };
#pragma unroll
    for (int j = 0; j < VEC; ++j) part[j] = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (mine && grp + groups * r < a.dk)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                s[r].v[j] *= decay;
                part[j] = fmaf(sk[grp + groups * r], s[r].v[j], part[j]);
            }
    sum_groups(part);
    float write[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const float v = mine ? load<T>(a.v, i * a.vs + (int64_t)head * a.dv + col * VEC + j) : 0.f;
        write[j] = beta * (v - part[j]);
        part[j] = 0.f;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (mine && grp + groups * r < a.dk) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                s[r].v[j] = fmaf(sk[grp + groups * r], write[j], s[r].v[j]);
                part[j] = fmaf(sq[grp + groups * r], s[r].v[j], part[j]);
            }
            *reinterpret_cast<Pack<float, VEC> *>(S + (grp + groups * r) * a.dv) = s[r];
        }
    sum_groups(part);
    if (grp == 0 && mine)
#pragma unroll
        for (int j = 0; j < VEC; ++j) out[col * VEC + j] = from_float<T>(part[j]);
}

template <class T, int VEC>
void step(const DeltaArgs &a, hipStream_t s) {
    int lanes = 1;
    while (lanes * VEC < a.dv) lanes *= 2;              // at most 32 (VEC 4) or 128 (VEC 1)
    const int rows = (a.dk * lanes + 255) / 256;
    const int blocks = a.n * a.hv;
    if (rows <= 4) k_delta_step<T, VEC, 4><<<blocks, 256, 0, s>>>(a, lanes);
    else if (rows <= 16) k_delta_step<T, VEC, 16><<<blocks, 256, 0, s>>>(a, lanes);
    else if constexpr (VEC == 1) k_delta_step<T, VEC, 64><<<blocks, 256, 0, s>>>(a, lanes);
}

// ------------------------------------------------------------------ chunks

constexpr int kLd = kC + 4;       // row length of a 64-wide LDS tile, off the banks' stride

// (I + A)^-1 and P of every chunk: a block takes a chunk slot and a key head,
// whose K K^T and Q K^T serve the value heads that share it.
template <class T>
__global__ __launch_bounds__(256) void k_delta_prepare(DeltaArgs a) {
    extern __shared__ float lds[];
    const int ld = a.dk + 4 + (a.dk & 3 ? 4 - (a.dk & 3) : 0);
    float *sk = lds, *sq = sk + kC * ld, *kk = sq + kC * ld, *qk = kk + kC * kLd, *x = qk + kC * kLd;
    __shared__ double cs[kC];
    __shared__ float beta[kC];
    const int slot = blockIdx.x, hk = blockIdx.y, group = a.hv / a.hk;
    const Chunk c = chunk_of(a, slot);
    if (c.len == 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int kp = (a.dk + 3) / 4 * 4;
    for (int i = threadIdx.x; i < kC * kp; i += 256) {
        const int t = i / kp, d = i % kp;
        const bool in = t < c.len && d < a.dk;
        sk[t * ld + d] = in ? load<T>(a.k, (c.begin + t) * a.ks + hk * a.dk + d) : 0.f;
        sq[t * ld + d] = in ? load<T>(a.q, (c.begin + t) * a.qs + hk * a.dk + d) * a.scale : 0.f;
    }
    __syncthreads();
    const int r0 = wave * 16;
    for (int n = 0; n < 4; ++n) {
        const auto kt = [&](int k, int j) { return sk[(n * 16 + j) * ld + k]; };
        const f32x4 u = tile_mm(kp, [&](int i, int k) { return sk[(r0 + i) * ld + k]; }, kt, f32x4{});
        const f32x4 w = tile_mm(kp, [&](int i, int k) { return sq[(r0 + i) * ld + k]; }, kt, f32x4{});
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = r0 + (lane >> 4) * 4 + j, colm = n * 16 + (lane & 15);
            kk[row * kLd + colm] = u[j];
            qk[row * kLd + colm] = w[j];
        }
    }
    for (int h = hk * group; h < (hk + 1) * group; ++h) {
        __syncthreads();
        if (wave == 0) {
            cs[lane] = decay_sums(a, c, h);
            beta[lane] = lane < c.len ? a.beta[(int64_t)(c.begin + lane) * a.hv + h] : 0.f;
        }
        __syncthreads();
        const int64_t at = ((int64_t)slot * a.hv + h) * kC * kC;
        for (int i = threadIdx.x; i < kC * kC; i += 256) {
            const int row = i / kC, colm = i % kC;
            const float d = colm <= row ? expf((float)(cs[row] - cs[colm])) : 0.f;
            a.score[at + i] = colm <= row ? d * qk[row * kLd + colm] : 0.f;
            x[row * kLd + colm] = colm < row ? beta[row] * d * kk[row * kLd + colm] : 0.f;   // A
        }
        __syncthreads();
        // Forward substitution, a column of the inverse a lane of one wave:
        // X_ij = [i == j] - sum_(l < i) A_il X_lj, kept in registers.
        if (wave == 0) {
            float col[kC];
#pragma unroll
            for (int i = 0; i < kC; ++i) {
                float s = i == lane ? 1.f : 0.f;
#pragma unroll
                for (int l = 0; l < i; ++l) s = fmaf(-x[i * kLd + l], col[l], s);
                col[i] = s;
            }
#pragma unroll
            for (int i = 0; i < kC; ++i) a.inv[at + i * kC + lane] = col[i];
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void k_delta_walk(DeltaArgs a) {
    extern __shared__ float lds[];
    const int kp = (a.dk + 15) / 16 * 16, ld = kp + 4;
    constexpr int ldv = kVT + 1;
    float *sk = lds, *sq = sk + kC * ld, *m = sq + kC * ld, *p = m + kC * kLd;
    float *S = p + kC * kLd, *w = S + kp * ldv;
    __shared__ double cs[kC];
    __shared__ float beta[kC];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int seq = blockIdx.x / a.hv, h = blockIdx.x % a.hv, hk = h / (a.hv / a.hk);
    const int v0 = blockIdx.y * kVT;
    const Span span = span_of(a, seq);
    const int64_t sbase = ((int64_t)seq * a.hv + h) * a.dk * a.dv;
    for (int i = threadIdx.x; i < kp * kVT; i += 256) {
        const int d = i / kVT, v = i % kVT;
        S[d * ldv + v] = a.state && d < a.dk && v0 + v < a.dv ? a.state[sbase + d * a.dv + v0 + v] : 0.f;
    }
    const int r0 = wave * 16, row4 = r0 + (lane >> 4) * 4, colv = lane & 15;
    for (int at = 0, chunk = 0; at < span.len; at += kC, ++chunk) {
        const Chunk c{seq, span.begin + at, min(kC, span.len - at)};
        const int64_t ch = (int64_t)slot_of(span, seq, chunk) * a.hv + h;
        __syncthreads();
        if (wave == 0) {
            cs[lane] = decay_sums(a, c, h);
            beta[lane] = lane < c.len ? a.beta[(int64_t)(c.begin + lane) * a.hv + h] : 0.f;
        }
        for (int i = threadIdx.x; i < kC * kp; i += 256) {
            const int t = i / kp, d = i % kp;
            const bool in = t < c.len && d < a.dk;
            sk[t * ld + d] = in ? load<T>(a.k, (c.begin + t) * a.ks + hk * a.dk + d) : 0.f;
            sq[t * ld + d] = in ? load<T>(a.q, (c.begin + t) * a.qs + hk * a.dk + d) * a.scale : 0.f;
        }
        for (int i = threadIdx.x; i < kC * kC; i += 256) {
            m[i / kC * kLd + i % kC] = a.inv[ch * kC * kC + i];
            p[i / kC * kLd + i % kC] = a.score[ch * kC * kC + i];
        }
        if (a.before)
            for (int i = threadIdx.x; i < a.dk * kVT; i += 256) {
                const int d = i / kVT, v = i % kVT;
                if (v0 + v < a.dv) a.before[(ch * a.dk + d) * a.dv + v0 + v] = S[d * ldv + v];
            }
        __syncthreads();
        // beta (V - e^c K S), then V', then out: the wave's 16 tokens each.
        const auto sb = [&](int k, int j) { return S[k * ldv + j]; };
        const f32x4 held = tile_mm(kp, [&](int i, int k) { return sk[(r0 + i) * ld + k]; }, sb, f32x4{});
        f32x4 o = tile_mm(kp, [&](int i, int k) { return sq[(r0 + i) * ld + k]; }, sb, f32x4{});
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = row4 + j;
            const bool in = t < c.len && v0 + colv < a.dv;
            const float v = in ? load<T>(a.v, (c.begin + t) * a.vs + (int64_t)h * a.dv + v0 + colv) : 0.f;
            const float grown = expf((float)cs[t]);
            w[t * ldv + colv] = beta[t] * (v - grown * held[j]);
            o[j] *= grown;
        }
        __syncthreads();
        const auto wb = [&](int k, int j) { return w[k * ldv + j]; };
        const f32x4 nv = tile_mm(r0 + 16, [&](int i, int k) { return m[(r0 + i) * kLd + k]; }, wb, f32x4{});
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) w[(row4 + j) * ldv + colv] = nv[j];
        __syncthreads();
        o = tile_mm(r0 + 16, [&](int i, int k) { return p[(r0 + i) * kLd + k]; }, wb, o);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = row4 + j;
            if (t < c.len && v0 + colv < a.dv)
                static_cast<T *>(a.out)[((int64_t)(c.begin + t) * a.hv + h) * a.dv + v0 + colv] = from_float<T>(o[j]);
        }
        // the memory after the chunk: rows of S, a wave every fourth 16
        __syncthreads();
        const double last = cs[kC - 1];
        const float whole = expf((float)last);
        for (int d0 = wave * 16; d0 < kp; d0 += 64) {
            const f32x4 add = tile_mm(
                kC, [&](int i, int k) { return sk[k * ld + d0 + i] * expf((float)(last - cs[k])); }, wb, f32x4{});
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float &s = S[(d0 + (lane >> 4) * 4 + j) * ldv + colv];
                s = fmaf(whole, s, add[j]);
            }
        }
    }
    __syncthreads();
    if (a.final_state)
        for (int i = threadIdx.x; i < a.dk * kVT; i += 256) {
            const int d = i / kVT, v = i % kVT;
            if (v0 + v < a.dv) a.final_state[sbase + d * a.dv + v0 + v] = S[d * ldv + v];
        }
}

template <class T>
hipError_t forward(const DeltaArgs &a, hipStream_t s) {
    const int slots = (int)delta_chunk_slots(a.tokens, a.n);
    if (a.tokens > 0) {
        const int ld = (a.dk + 3) / 4 * 4 + 4;
        const size_t bytes = sizeof(float) * (2 * kC * ld + 3 * kC * kLd);
        if (hipError_t e = allow_lds(k_delta_prepare<T>, bytes)) return e;
        k_delta_prepare<T><<<dim3(slots, a.hk), 256, bytes, s>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    const int kp = (a.dk + 15) / 16 * 16;
    const size_t bytes = sizeof(float) * (2 * kC * (kp + 4) + 2 * kC * kLd + (kp + kC) * (kVT + 1));
    if (hipError_t e = allow_lds(k_delta_walk<T>, bytes)) return e;
    k_delta_walk<T><<<dim3(a.n * a.hv, (a.dv + kVT - 1) / kVT), 256, bytes, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_step(const DeltaArgs &a, bool bf16, hipStream_t s) {
    const bool vec = a.dv % 4 == 0 && reinterpret_cast<uintptr_t>(a.final_state) % 16 == 0;
    if (bf16) vec ? step<bf16_t, 4>(a, s) : step<bf16_t, 1>(a, s);
    else vec ? step<float, 4>(a, s) : step<float, 1>(a, s);
    return hipGetLastError();
}

hipError_t launch_delta_forward(const DeltaArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}

}  // namespace rn
