// Gradients of the gated delta rule over whole sequences.
//
// With the chunk quantities of rn_delta.hip (S and S' the memories before and
// after a chunk, M = I + A, P, c) and dS' = dJ/dS':
//   dV' = P^T dO + (e^(c64 - c) K) dS',      dR = M^-T dV'    (R = beta (V - e^c K S)),
//   dS  = e^(c64) dS' + (scale e^c Q)^T dO - (beta e^c K)^T dR:
// k_delta_bwd_walk takes the chunks of a sequence from the last to the first,
// 16 columns of S a block, and leaves dS' and dR.  Then every chunk by itself
// (k_delta_bwd_chunk), with dP = dO V'^T, dA = -dR V'^T and e = c_i - c_j:
//   dv = beta dR,
//   dq = scale (e^c dO S^T + (dP e^e) K),
//   dk = [-beta e^c dR S^T + (beta dA e^e) K]  (k as the row: reads)
//      + [e^(c64 - c) V' dS'^T + (dP e^e)^T scale Q + (beta dA e^e)^T K]  (as the column: writes),
//   dbeta_i = sum dR (V - e^c K S) + sum_j dA_ij A_ij / beta_i,
//   dc_i = q_i . dq_i + k_i . dk_i(reads) - k_i . dk_i(writes): every term of
//     these products holds e^(c_i) or e^(-c_i) once,
//   dc_64 also has sum_i e^(c64 - ci) k_i . (V' dS'^T)_i + e^(c64) <S, dS'>,
//   dg_t = sum over s >= t in the chunk of dc_s.
#include "rn_delta.hpp"

namespace rn {
namespace {

using namespace ops;

constexpr int kLd = kC + 4;
constexpr int kLdV = kVT + 1;

template <class T>
__global__ __launch_bounds__(256) void k_delta_bwd_walk(DeltaArgs a) {
    extern __shared__ float lds[];
    const int kp = (a.dk + 15) / 16 * 16, ld = kp + 4;
    float *sk = lds, *sq = sk + kC * ld, *m = sq + kC * ld, *p = m + kC * kLd;
    float *dS = p + kC * kLd, *w = dS + kp * kLdV, *od = w + kC * kLdV;
    __shared__ double cs[kC];
    __shared__ float beta[kC];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int seq = blockIdx.x / a.hv, h = blockIdx.x % a.hv, hk = h / (a.hv / a.hk);
    const int v0 = blockIdx.y * kVT;
    const Span span = span_of(a, seq);
    const int64_t sbase = ((int64_t)seq * a.hv + h) * a.dk * a.dv;
    for (int i = threadIdx.x; i < kp * kVT; i += 256) {
        const int d = i / kVT, v = i % kVT;
        dS[d * kLdV + v] = a.dfinal && d < a.dk && v0 + v < a.dv ? a.dfinal[sbase + d * a.dv + v0 + v] : 0.f;
    }
    const int r0 = wave * 16, row4 = r0 + (lane >> 4) * 4, colv = lane & 15;
    for (int chunk = (span.len + kC - 1) / kC - 1; chunk >= 0; --chunk) {
        const int at = chunk * kC;
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
        for (int i = threadIdx.x; i < kC * kVT; i += 256) {
            const int t = i / kVT, v = i % kVT;
            const bool in = t < c.len && v0 + v < a.dv;
            od[t * kLdV + v] = in ? load<T>(a.dout, ((int64_t)(c.begin + t) * a.hv + h) * a.dv + v0 + v) : 0.f;
        }
        for (int i = threadIdx.x; i < a.dk * kVT; i += 256) {
            const int d = i / kVT, v = i % kVT;
            if (v0 + v < a.dv) a.after[(ch * a.dk + d) * a.dv + v0 + v] = dS[d * kLdV + v];
        }
        __syncthreads();
        const double last = cs[kC - 1];
        const auto ob = [&](int k, int j) { return od[k * kLdV + j]; };
        const auto wb = [&](int k, int j) { return w[k * kLdV + j]; };
        f32x4 x = tile_mm(kp, [&](int i, int k) { return sk[(r0 + i) * ld + k]; },
                          [&](int k, int j) { return dS[k * kLdV + j]; }, f32x4{});
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] *= expf((float)(last - cs[row4 + j]));
        x = tile_mm(kC, [&](int i, int k) { return p[k * kLd + r0 + i]; }, ob, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[(row4 + j) * kLdV + colv] = x[j];
        __syncthreads();
        x = tile_mm(kC, [&](int i, int k) { return m[k * kLd + r0 + i]; }, wb, f32x4{});
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = row4 + j;
            w[t * kLdV + colv] = x[j];
            if (t < c.len && v0 + colv < a.dv)
                a.dwrite[((int64_t)(c.begin + t) * a.hv + h) * a.dv + v0 + colv] = x[j];
        }
        __syncthreads();
        const float whole = expf((float)last);
        for (int d0 = wave * 16; d0 < kp; d0 += 64) {
            f32x4 y = tile_mm(kC, [&](int i, int k) { return sq[k * ld + d0 + i] * expf((float)cs[k]); }, ob, f32x4{});
            y = tile_mm(kC, [&](int i, int k) { return -beta[k] * expf((float)cs[k]) * sk[k * ld + d0 + i]; }, wb, y);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float &s = dS[(d0 + (lane >> 4) * 4 + j) * kLdV + colv];
                s = fmaf(whole, s, y[j]);
            }
        }
    }
    __syncthreads();
    if (a.dstate)
        for (int i = threadIdx.x; i < a.dk * kVT; i += 256) {
            const int d = i / kVT, v = i % kVT;
            if (v0 + v < a.dv) a.dstate[sbase + d * a.dv + v0 + v] = dS[d * kLdV + v];
        }
}

// A block takes a chunk slot and a key head and adds the value heads that share
// it; a wave owns 16 tokens.  KT: 16-wide tiles of dk that a wave's registers hold.
template <class T, int KT>
__global__ __launch_bounds__(256) void k_delta_bwd_chunk(DeltaArgs a) {
    extern __shared__ float lds[];
    constexpr int kp = KT * 16, ld = kp + 4;
    float *sk = lds, *sq = sk + kC * ld, *m = sq + kC * ld, *x = m + kC * kLd, *y = x + kC * kLd;
    float *S = y + kC * kLd, *dS = S + kp * kLdV, *od = dS + kp * kLdV, *dr = od + kC * kLdV, *w = dr + kC * kLdV;
    __shared__ double cs[kC];
    __shared__ float beta[kC], dc[kC], extra[4];
    const int slot = blockIdx.x, hk = blockIdx.y, group = a.hv / a.hk;
    const Chunk c = chunk_of(a, slot);
    if (c.len == 0) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int r0 = wave * 16, row4 = r0 + (lane >> 4) * 4, col = lane & 15;
    for (int i = threadIdx.x; i < kC * kp; i += 256) {
        const int t = i / kp, d = i % kp;
        const bool in = t < c.len && d < a.dk;
        sk[t * ld + d] = in ? load<T>(a.k, (c.begin + t) * a.ks + hk * a.dk + d) : 0.f;
        sq[t * ld + d] = in ? load<T>(a.q, (c.begin + t) * a.qs + hk * a.dk + d) * a.scale : 0.f;
    }
    // Sum over the 16 lanes that hold a row's columns.
    const auto across = [&](float v) {
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) v += __shfl_xor(v, s);
        return v;
    };
    f32x4 tq[KT], tk[KT];
#pragma unroll
    for (int n = 0; n < KT; ++n) tq[n] = tk[n] = f32x4{};
    for (int h = hk * group; h < (hk + 1) * group; ++h) {
        const int64_t ch = (int64_t)slot * a.hv + h;
        __syncthreads();
        if (wave == 0) {
            cs[lane] = decay_sums(a, c, h);
            beta[lane] = lane < c.len ? a.beta[(int64_t)(c.begin + lane) * a.hv + h] : 0.f;
        }
        for (int i = threadIdx.x; i < kC * kC; i += 256) m[i / kC * kLd + i % kC] = a.inv[ch * kC * kC + i];
        f32x4 gq[KT], gr[KT], gw[KT], dp[4], da[4];
#pragma unroll
        for (int n = 0; n < KT; ++n) gq[n] = gr[n] = gw[n] = f32x4{};
#pragma unroll
        for (int n = 0; n < 4; ++n) dp[n] = da[n] = f32x4{};
        float db[4] = {0.f, 0.f, 0.f, 0.f}, dot = 0.f;
        for (int v0 = 0; v0 < a.dv; v0 += kVT) {
            __syncthreads();
            for (int i = threadIdx.x; i < kp * kVT; i += 256) {
                const int d = i / kVT, v = i % kVT;
                const bool in = d < a.dk && v0 + v < a.dv;
                const int64_t at = (ch * a.dk + d) * a.dv + v0 + v;
                const float s = in ? a.before[at] : 0.f, t = in ? a.after[at] : 0.f;
                S[d * kLdV + v] = s;
                dS[d * kLdV + v] = t;
                dot = fmaf(s, t, dot);
            }
            for (int i = threadIdx.x; i < kC * kVT; i += 256) {
                const int t = i / kVT, v = i % kVT;
                const bool in = t < c.len && v0 + v < a.dv;
                const int64_t at = ((int64_t)(c.begin + t) * a.hv + h) * a.dv + v0 + v;
                od[t * kLdV + v] = in ? load<T>(a.dout, at) : 0.f;
                dr[t * kLdV + v] = in ? a.dwrite[at] : 0.f;
            }
            __syncthreads();
            const f32x4 held = tile_mm(kp, [&](int i, int k) { return sk[(r0 + i) * ld + k]; },
                                       [&](int k, int j) { return S[k * kLdV + j]; }, f32x4{});
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = row4 + j;
                const bool in = t < c.len && v0 + col < a.dv;
                const float v = in ? load<T>(a.v, (c.begin + t) * a.vs + (int64_t)h * a.dv + v0 + col) : 0.f;
                const float gap = v - expf((float)cs[t]) * held[j], g = dr[t * kLdV + col];
                db[j] += across(g * gap);
                w[t * kLdV + col] = beta[t] * gap;
                if (in)
                    static_cast<T *>(a.dval)[((int64_t)(c.begin + t) * a.hv + h) * a.dv + v0 + col] =
                        from_float<T>(beta[t] * g);
            }
            __syncthreads();
            const f32x4 nv = tile_mm(r0 + 16, [&](int i, int k) { return m[(r0 + i) * kLd + k]; },
                                     [&](int k, int j) { return w[k * kLdV + j]; }, f32x4{});
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 4; ++j) w[(row4 + j) * kLdV + col] = nv[j];
            __syncthreads();
            const auto oa = [&](int i, int k) { return od[(r0 + i) * kLdV + k]; };
            const auto ra = [&](int i, int k) { return dr[(r0 + i) * kLdV + k]; };
            const auto wa = [&](int i, int k) { return w[(r0 + i) * kLdV + k]; };
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const auto wt = [&](int k, int j) { return w[(n * 16 + j) * kLdV + k]; };
                dp[n] = tile_mm(kVT, oa, wt, dp[n]);
                da[n] = tile_mm(kVT, ra, wt, da[n]);
            }
#pragma unroll
            for (int n = 0; n < KT; ++n) {
                const auto st = [&](int k, int j) { return S[(n * 16 + j) * kLdV + k]; };
                const auto dt = [&](int k, int j) { return dS[(n * 16 + j) * kLdV + k]; };
                gq[n] = tile_mm(kVT, oa, st, gq[n]);
                gr[n] = tile_mm(kVT, ra, st, gr[n]);
                gw[n] = tile_mm(kVT, wa, dt, gw[n]);
            }
        }
        const double last = cs[kC - 1];
        // k_i . k_j and the pairs' weights; dbeta's share of A.
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const f32x4 kk = tile_mm(kp, [&](int i, int k) { return sk[(r0 + i) * ld + k]; },
                                     [&](int k, int j) { return sk[(n * 16 + j) * ld + k]; }, f32x4{});
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = row4 + j, u = n * 16 + col;
                const float d = u <= t ? expf((float)(cs[t] - cs[u])) : 0.f;
                const float pa = u < t ? -da[n][j] * d : 0.f;
                x[t * kLd + u] = u <= t ? dp[n][j] * d : 0.f;
                y[t * kLd + u] = beta[t] * pa;
                db[j] += across(u < t ? pa * kk[j] : 0.f);
            }
        }
        // the memory's part of the sums, before the pairs' is added
        float wsum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = row4 + j;
            const float grown = expf((float)cs[t]), left = expf((float)(last - cs[t]));
            float s = 0.f;
#pragma unroll
            for (int n = 0; n < KT; ++n) {
                gq[n][j] *= grown;
                gr[n][j] *= -beta[t] * grown;
                gw[n][j] *= left;
                s = fmaf(gw[n][j], sk[t * ld + n * 16 + col], s);
            }
            wsum += across(s);
        }
        wsum += __shfl_xor(wsum, 16);
        wsum += __shfl_xor(wsum, 32);
        float all = dot * expf((float)last);
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) all += __shfl_xor(all, s);
        if (lane == 0) extra[wave] = all + wsum;
        __syncthreads();
#pragma unroll
        for (int n = 0; n < KT; ++n) {
            const auto kb = [&](int k, int j) { return sk[k * ld + n * 16 + j]; };
            const auto qb = [&](int k, int j) { return sq[k * ld + n * 16 + j]; };
            gq[n] = tile_mm(r0 + 16, [&](int i, int k) { return x[(r0 + i) * kLd + k]; }, kb, gq[n]);
            gr[n] = tile_mm(r0 + 16, [&](int i, int k) { return y[(r0 + i) * kLd + k]; }, kb, gr[n]);
            gw[n] = tile_mm(kC, [&](int i, int k) { return x[k * kLd + r0 + i]; }, qb, gw[n]);
            gw[n] = tile_mm(kC, [&](int i, int k) { return y[k * kLd + r0 + i]; }, kb, gw[n]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = row4 + j;
            float s = 0.f;
#pragma unroll
            for (int n = 0; n < KT; ++n) {
                s = fmaf(gq[n][j], sq[t * ld + n * 16 + col], s);
                s = fmaf(gr[n][j] - gw[n][j], sk[t * ld + n * 16 + col], s);
                tq[n][j] += gq[n][j];
                tk[n][j] += gr[n][j] + gw[n][j];
            }
            s = across(s);
            if (col == 0) {
                dc[t] = s;
                if (t < c.len) a.dbeta[(int64_t)(c.begin + t) * a.hv + h] = db[j];
            }
        }
        __syncthreads();
        if (wave == 0) {
            double s = dc[lane];
            if (lane == kC - 1) s += ((double)extra[0] + extra[1]) + ((double)extra[2] + extra[3]);
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const double u = __shfl_down(s, d);
                if (lane + d < 64) s += u;
            }
            if (lane < c.len) a.dg[(int64_t)(c.begin + lane) * a.hv + h] = (float)s;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int t = row4 + j;
        if (t >= c.len) continue;
        const int64_t at = ((int64_t)(c.begin + t) * a.hk + hk) * a.dk;
#pragma unroll
        for (int n = 0; n < KT; ++n)
            if (n * 16 + col < a.dk) {
                static_cast<T *>(a.dq)[at + n * 16 + col] = from_float<T>(tq[n][j] * a.scale);
                static_cast<T *>(a.dkey)[at + n * 16 + col] = from_float<T>(tk[n][j]);
            }
    }
}

template <class T, int KT>
hipError_t chunks(const DeltaArgs &a, hipStream_t s) {
    constexpr int kp = KT * 16;
    const size_t bytes = sizeof(float) * (2 * kC * (kp + 4) + 3 * kC * kLd + (2 * kp + 3 * kC) * kLdV);
    if (hipError_t e = allow_lds(k_delta_bwd_chunk<T, KT>, bytes)) return e;
    k_delta_bwd_chunk<T, KT><<<dim3((int)delta_chunk_slots(a.tokens, a.n), a.hk), 256, bytes, s>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t backward(const DeltaArgs &a, hipStream_t s) {
    const int kp = (a.dk + 15) / 16 * 16;
    const size_t bytes = sizeof(float) * (2 * kC * (kp + 4) + 2 * kC * kLd + (kp + 2 * kC) * kLdV);
    if (hipError_t e = allow_lds(k_delta_bwd_walk<T>, bytes)) return e;
    k_delta_bwd_walk<T><<<dim3(a.n * a.hv, (a.dv + kVT - 1) / kVT), 256, bytes, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.tokens == 0) return hipSuccess;
    if (a.dk <= 32) return chunks<T, 2>(a, s);
    if (a.dk <= 64) return chunks<T, 4>(a, s);
    return chunks<T, 8>(a, s);
}

}  // namespace

hipError_t launch_delta_backward(const DeltaArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? backward<bf16_t>(a, s) : backward<float>(a, s);
}

}  // namespace rn
