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

// The chunk operands of k_delta_walk, in fragment order: (I + A)^-1, P and the
// decays of a chunk and value head, and with the first of the value heads that
// share a key head its K, Q and K^T.  A block takes a chunk slot and a value
// head, a wave 16 of its tokens; what lies past the chunk's last 16 is not made.
//
// The inverse by blocks of 16: the four on the diagonal by forward substitution,
// a column a lane; then the 32s and the 64 from
//   [L11 0; L21 L22]^-1 = [X11 0; -X22 L21 X11  X22]
// on the float32 matrix cores.  Substitution of the blocks alone keeps this as
// stable as that of the whole, with a chain of 16 rows in place of 64.  (A power
// series of the nilpotent A would be shorter, and loses all its bits where keys
// are nearly parallel, as those of neighbouring frames are.)
//
// A chain of small steps with barriers between them: bound by their latency, so
// the LDS is kept small (four blocks a CU in bfloat16) and the blocks many.
template <class T, int KS, bool VEC>
__global__ __launch_bounds__(256) void k_delta_operands(DeltaArgs a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3, NPP = sizeof(T) == 2 ? 2 : 3;
    constexpr int kKeys = 4 * KS * NP * kFrag;          // bf16 of one of kf, qf, kt
    extern __shared__ __align__(16) float lds[];
    float *x = lds, *y = x + kC * kLd;                  // A, then its inverse; P, over K's fragments
    uint16_t *skf = reinterpret_cast<uint16_t *>(y);
    __shared__ double cs[kC];
    __shared__ float beta[kC];
    const int slot = blockIdx.x, h = blockIdx.y, group = a.hv / a.hk, hk = h / group;
    const Chunk c = chunk_of(a, slot);
    if (c.len == 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int blocks = (c.len + 15) / 16;               // 16s of tokens
    const bool first = h % group == 0, busy = wave < blocks;
    const int64_t keys = ((int64_t)slot * a.hk + hk) * kKeys, ch = (int64_t)slot * a.hv + h;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    // K and Q as rows: the wave's 16 tokens.
    const int token = wave * 16 + r;
    bf16x8 ka[KS][NP], qa[KS][NP];
    const auto row = [&](const void *p, int64_t stride, int ks, bf16x8 (&f)[NP]) {
        const int64_t at = (int64_t)(c.begin + token) * stride + hk * a.dk;
        const int d0 = ks * 32 + g * 8;
        float v[8];
        if constexpr (VEC) {                            // rows on 16 bytes, dk a multiple of 8
            constexpr int PER = 16 / sizeof(T);
#pragma unroll
            for (int e = 0; e < 8; e += PER) {
                Pack<T, PER> q{};
                if (token < c.len && d0 < a.dk) q = *reinterpret_cast<const Pack<T, PER> *>(static_cast<const T *>(p) + at + d0 + e);
#pragma unroll
                for (int o = 0; o < PER; ++o) v[e + o] = to_float(q.v[o]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = token < c.len && d0 + e < a.dk ? load<T>(p, at + d0 + e) : 0.f;
        }
        uint32_t w[4][NP];
#pragma unroll
        for (int e = 0; e < 4; ++e) split_pair<NP>(v[2 * e], v[2 * e + 1], w[e]);
#pragma unroll
        for (int i = 0; i < NP; ++i) f[i] = __builtin_bit_cast(bf16x8, u32x4{w[0][i], w[1][i], w[2][i], w[3][i]});
    };
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        row(a.k, a.ks, ks, ka[ks]);
        row(a.q, a.qs, ks, qa[ks]);
    }
    if (wave == 0) {
        const double s = decay_sums(a, c, h), last = __shfl(s, 63);
        const float b = lane < c.len ? a.beta[(int64_t)(c.begin + lane) * a.hv + h] : 0.f;
        cs[lane] = s;
        beta[lane] = b;
        a.dec[ch * 3 * kC + lane] = expf((float)s);
        a.dec[ch * 3 * kC + kC + lane] = expf((float)(last - s));
        a.dec[ch * 3 * kC + 2 * kC + lane] = b;
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = ((wave * KS + ks) * NP + i) * kFrag + lane * 8;
            *reinterpret_cast<bf16x8 *>(skf + at) = ka[ks][i];
            if (first && busy) {
                *reinterpret_cast<bf16x8 *>(a.kf + keys + at) = ka[ks][i];
                *reinterpret_cast<bf16x8 *>(a.qf + keys + at) = qa[ks][i];
            }
        }
    __syncthreads();
    // K K^T and Q K^T, the wave's rows of them.
    f32x4 u[4] = {}, w[4] = {};
#pragma unroll
    for (int n = 0; n < 4; ++n)
        if (busy && n <= wave)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                bf16x8 kb[NP];
                load_frags<NP>(skf + ((n * KS + ks) * NP) * kFrag + lane * 8, kb);
                u[n] = mm<NP, NP>(ka[ks], kb, u[n]);
                w[n] = mm<NP, NP>(qa[ks], kb, w[n]);
            }
    // K^T as rows: element (d, token) from K's fragments.
    if (first)
        for (int i = wave; i < 2 * KS * 2; i += 4) {
            const int rt = i / 2, ks = i % 2, d = rt * 16 + r;
            if (ks * 32 >= c.len) continue;
            const int from = ((d / 32) * NP) * kFrag + (d % 32 / 8) * 16 * 8 + d % 8;    // of row block 0, token 0
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
                u16x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = ks * 32 + g * 8 + e;
                    v[e] = skf[from + (t / 16) * KS * NP * kFrag + p * kFrag + (t % 16) * 8];
                }
                *reinterpret_cast<u16x8 *>(a.kt + keys + (i * NP + p) * kFrag + lane * 8) = v;
            }
        }
    __syncthreads();                                    // K's fragments have been read
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int col = n * 16 + r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = wave * 16 + g * 4 + j;
            const float d = busy && n <= wave && col <= t ? expf((float)(cs[t] - cs[col])) : 0.f;
            y[t * kLd + col] = col <= t ? d * w[n][j] * a.scale : 0.f;
            x[t * kLd + col] = col < t ? beta[t] * d * u[n][j] : 0.f;
        }
    }
    __syncthreads();
    if (wave == 0) {                                    // the diagonal blocks, one a quarter wave
        const float *d = x + g * 16 * kLd + g * 16;
        float col[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i == r ? 1.f : 0.f;
#pragma unroll
            for (int l = 0; l < i; l += 4) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(d + i * kLd + l);
#pragma unroll
                for (int o = 0; o < 4; ++o)
                    if (l + o < i) s = fmaf(-v[o], col[l + o], s);
            }
            col[i] = s;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[(g * 16 + i) * kLd + g * 16 + r] = col[i];
    } else {
        // P into fragments meanwhile: a lane's eight columns of a row.
        for (int i = wave - 1; i < kTri; i += 3) {
            const int rb = i < 2 ? i : i / 2 + 1, ks = i < 2 ? 0 : i & 1;
            if (rb >= blocks) continue;
            const float *p = y + (rb * 16 + r) * kLd + ks * 32 + g * 8;
            uint32_t q[4][NPP];
#pragma unroll
            for (int e = 0; e < 4; ++e) split_pair<NPP>(p[2 * e], p[2 * e + 1], q[e]);
#pragma unroll
            for (int o = 0; o < NPP; ++o)
                *reinterpret_cast<u32x4 *>(a.pf + (ch * kTri + i) * NPP * kFrag + o * kFrag + lane * 8) =
                    u32x4{q[0][o], q[1][o], q[2][o], q[3][o]};
        }
    }
    __syncthreads();
    const auto put = [&](float *to, f32x4 v, float sign) {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[(g * 4 + j) * kLd + r] = sign * v[j];
    };
    // The 32s: -X11 (A10 X00) for the pairs (0, 1) and (2, 3), a wave each.
    if (blocks > 1) {
        if (wave < 2) {
            float *b = x + wave * 32 * kLd + wave * 32, *l = b + 16 * kLd;
            const f32x4 t = tile_mm(16, [&](int i, int k) { return l[i * kLd + k]; },
                                    [&](int k, int j) { return b[k * kLd + j]; }, f32x4{});
            put(y + wave * 16 * kLd, t, 1.f);           // y's first rows: P is out of them
            const f32x4 v = tile_mm(16, [&](int i, int k) { return l[i * kLd + 16 + k]; },
                                    [&](int k, int j) { return y[(wave * 16 + k) * kLd + j]; }, f32x4{});
            put(l, v, -1.f);
        }
        __syncthreads();
    }
    // The 64: -X22 (A21 X11), a 16 x 16 tile a wave.
    if (blocks > 2) {
        const int ti = wave / 2 * 16, tj = wave % 2 * 16;
        float *l = x + 32 * kLd;
        const f32x4 t = tile_mm(32, [&](int i, int k) { return l[(ti + i) * kLd + k]; },
                                [&](int k, int j) { return x[k * kLd + tj + j]; }, f32x4{});
        put(y + ti * kLd + tj, t, 1.f);
        __syncthreads();
        const f32x4 v = tile_mm(32, [&](int i, int k) { return l[(ti + i) * kLd + 32 + k]; },
                                [&](int k, int j) { return y[k * kLd + tj + j]; }, f32x4{});
        put(l + ti * kLd + tj, v, -1.f);
        __syncthreads();
    }
    for (int i = wave; i < kTri; i += 4) {
        const int rb = i < 2 ? i : i / 2 + 1, ks = i < 2 ? 0 : i & 1;
        if (rb >= blocks) continue;
        const float *p = x + (rb * 16 + r) * kLd + ks * 32 + g * 8;
        uint32_t q[4][3];
#pragma unroll
        for (int e = 0; e < 4; ++e) split_pair<3>(p[2 * e], p[2 * e + 1], q[e]);
#pragma unroll
        for (int o = 0; o < 3; ++o)
            *reinterpret_cast<u32x4 *>(a.mf + (ch * kTri + i) * 3 * kFrag + o * kFrag + lane * 8) =
                u32x4{q[0][o], q[1][o], q[2][o], q[3][o]};
    }
}

// A sequence's chunks in order.  A block takes 16 CT columns of a head's memory,
// wave w the tokens 16 w .. + 15 of a chunk and the memory's row tiles w, w + 4;
// the memory stays in its owners' registers in float32, and goes through LDS as
// bf16 planes to the waves that multiply by it, as do beta (V - e^c K S) and V'.
// The left operands are read from memory in fragment order, straight into
// registers, each for the next chunk as soon as this one's use of it is over.
template <class T, int KS, int CT, bool SAVE>
__global__ __launch_bounds__(256, sizeof(T) == 4 && KS == 4 ? 1 : 2) void k_delta_walk(DeltaArgs a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3, NPP = sizeof(T) == 2 ? 2 : 3;
    constexpr int KP = KS * 32, RT = KP > 64 ? KP / 64 : 1;        // row tiles of the memory a wave owns
    constexpr int VT = 16 * CT, ldS = KP + 8, ldT = kC + 8;
    constexpr int kKeys = 4 * KS * NP * kFrag;
    __shared__ __align__(16) uint16_t sS[3 * VT * ldS], sR[3 * VT * ldT], sV[NPP * VT * ldT], sL[3 * VT * ldT];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int seq = blockIdx.x / a.hv, h = blockIdx.x % a.hv, hk = h / (a.hv / a.hk);
    const int v0 = blockIdx.y * VT;
    const Span span = span_of(a, seq);
    const int chunks = (span.len + kC - 1) / kC;
    const int64_t slot0 = slot_of(span, seq, 0);
    const int64_t sbase = ((int64_t)seq * a.hv + h) * a.dk * a.dv + v0;
    const bool owner = KP >= 64 || wave * 16 < KP;
    bool col_in[CT];
#pragma unroll
    for (int n = 0; n < CT; ++n) col_in[n] = v0 + n * 16 + (int)r < a.dv;

    f32x4 S[RT][CT];
    const auto put_state = [&] {
        if (owner)
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int n = 0; n < CT; ++n)
                    put4<3>(sS, VT * ldS, (n * 16 + r) * ldS + (wave + 4 * i) * 16 + g * 4, S[i][n]);
    };
    const auto write_state = [&](float *to) {                       // to: [dk][dv] from column v0
        if (!owner) return;
        const __amdgpu_buffer_rsrc_t rs = rsrc_of(to);
        const uint32_t at = (wave * 16 + g * 4) * a.dv + r;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int n = 0; n < CT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    store_if(col_in[n] && (wave + 4 * i) * 16 + (int)g * 4 + j < a.dk, rs,
                             4 * (at + (64 * i + j) * a.dv + n * 16), (float)S[i][n][j]);
    };
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int n = 0; n < CT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = (wave + 4 * i) * 16 + g * 4 + j;
                const bool in = a.state && owner && d < a.dk && col_in[n];
                S[i][n][j] = in ? a.state[sbase + (int64_t)d * a.dv + n * 16 + r] : 0.f;
            }

    // Loads are unconditional, from places clamped into the arrays, so that the
    // compiler can count them and wait for each only where it is used.
    bf16x8 kf[KS][NP], qf[KS][NP], kt[RT][2][NP], mf[2][3], pf[2][NPP];
    T vv[CT][4];
    const auto load_rows = [&](int64_t slot) {
        const int64_t at = (slot * a.hk + hk) * kKeys + wave * KS * NP * kFrag;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            load_frags<NP>(a.kf + at + (lane * 8 + ks * NP * kFrag), kf[ks]);
            load_frags<NP>(a.qf + at + (lane * 8 + ks * NP * kFrag), qf[ks]);
        }
    };
    const auto load_kt = [&](int64_t slot) {
        const int64_t at = (slot * a.hk + hk) * kKeys + (wave % (2 * KS)) * 2 * NP * kFrag;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) load_frags<NP>(a.kt + at + (lane * 8 + (8 * i + ks) * NP * kFrag), kt[i][ks]);
    };
    const auto load_inv = [&](int64_t slot) {
        const int64_t at = (slot * a.hv + h) * kTri * 3 * kFrag;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) load_frags<3>(a.mf + (at + tri(wave, min(ks, wave / 2)) * 3 * kFrag) + lane * 8, mf[ks]);
    };
    const auto load_score = [&](int64_t slot) {
        const int64_t at = (slot * a.hv + h) * kTri * NPP * kFrag;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            load_frags<NPP>(a.pf + (at + tri(wave, min(ks, wave / 2)) * NPP * kFrag) + lane * 8, pf[ks]);
    };
    f32x4 grown{}, left{}, beta{}, next_grown{}, next_left{}, next_beta{};
    float whole = 0.f, next_whole = 0.f;
    const auto load_decays = [&](int64_t slot) {
        const float *d = a.dec + (slot * a.hv + h) * 3 * kC + wave * 16;
        next_grown = *reinterpret_cast<const f32x4 *>(d + g * 4);
        next_left = *reinterpret_cast<const f32x4 *>(d + (kC + g * 4));
        next_beta = *reinterpret_cast<const f32x4 *>(d + (2 * kC + g * 4));
        next_whole = a.dec[(slot * a.hv + h) * 3 * kC + kC - 1];
    };
    // Tokens past the end have beta 0; columns past dv are not written.  Offsets
    // within a chunk fit 32 bits (token strides are below 2^23).
    uint32_t col[CT], voff[4];
#pragma unroll
    for (int n = 0; n < CT; ++n) col[n] = min(n * 16 + (int)r, a.dv - 1 - v0);
    const auto load_v = [&](int chunk) {
        const T *base = static_cast<const T *>(a.v) + (int64_t)(span.begin + chunk * kC) * a.vs + (h * a.dv + v0);
        const int last = span.len - chunk * kC - 1;
#pragma unroll
        for (int j = 0; j < 4; ++j) voff[j] = min(wave * 16 + (int)g * 4 + j, last) * (uint32_t)a.vs;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < CT; ++n) vv[n][j] = base[voff[j] + col[n]];
    };
    const uint32_t ooff = (wave * 16 + g * 4) * (uint32_t)(a.hv * a.dv) + r;
    if (chunks > 0)
        load_decays(slot0), load_rows(slot0), load_v(0), load_inv(slot0), load_kt(slot0), load_score(slot0);
    put_state();

    const auto step = [&](int chunk, auto more_) {
        constexpr bool more = decltype(more_)::value;   // every chunk but the last: 64 tokens, and one follows
        const int64_t next = slot0 + chunk + 1, ch = (slot0 + chunk) * a.hv + h;
        const int len = more ? kC : span.len - chunk * kC;
        const bool busy = more || wave * 16 < len;      // any token of this wave
        const bool half2 = more || len > 32;            // tokens in the second 32
        grown = next_grown, left = next_left, beta = next_beta, whole = next_whole;
        if constexpr (SAVE) write_state(a.before + ch * a.dk * a.dv + v0);
        dev::lds_barrier();                             // the memory's planes are there
        f32x4 o[CT];
#pragma unroll
        for (int n = 0; n < CT; ++n) {
            f32x4 held{};
            o[n] = f32x4{};
            if (busy)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    bf16x8 s[3], s2[NPP];
                    get8<3>(sS, VT * ldS, (n * 16 + r) * ldS + ks * 32 + g * 8, s);
#pragma unroll
                    for (int i = 0; i < NPP; ++i) s2[i] = s[i];
                    held = mm<NP, 3>(kf[ks], s, held);
                    o[n] = mm<NP, NPP>(qf[ks], s2, o[n]);
                }
            f32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float gap = to_float(vv[n][j]) - grown[j] * held[j];
                w[j] = beta[j] * (more || beta[j] != 0.f ? gap : 0.f);
                o[n][j] *= grown[j] * a.scale;
            }
            put4<3>(sR, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, w);
        }
        if constexpr (more) load_decays(next), load_rows(next), load_v(chunk + 1);
        dev::lds_barrier();
#pragma unroll
        for (int n = 0; n < CT; ++n) {
            f32x4 w{};
            if (busy)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    if (ks <= wave / 2) {
                        bf16x8 b[3];
                        get8<3>(sR, VT * ldT, (n * 16 + r) * ldT + ks * 32 + g * 8, b);
                        w = mm<3, 3>(mf[ks], b, w);
                    }
            put4<NPP>(sV, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] *= left[j];
            put4<3>(sL, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, w);
        }
        if constexpr (more) load_inv(next);
        dev::lds_barrier();
        if (owner)
#pragma unroll
            for (int n = 0; n < CT; ++n) {
                bf16x8 b[2][3];
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    get8<3>(sL, VT * ldT, (n * 16 + r) * ldT + ks * 32 + g * 8, b[ks]);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) S[i][n][j] *= whole;
                    S[i][n] = mm<NP, 3>(kt[i][0], b[0], S[i][n]);
                    if (half2) S[i][n] = mm<NP, 3>(kt[i][1], b[1], S[i][n]);
                }
            }
        if constexpr (more) {
            put_state();                                // every wave is past its reads of the planes
            load_kt(next);
        }
        if (busy) {
            T *out = static_cast<T *>(a.out) + ((int64_t)(span.begin + chunk * kC) * a.hv + h) * a.dv + v0;
#pragma unroll
            for (int n = 0; n < CT; ++n) {
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    if (ks <= wave / 2) {
                        bf16x8 b[NPP];
                        get8<NPP>(sV, VT * ldT, (n * 16 + r) * ldT + ks * 32 + g * 8, b);
                        o[n] = mm<NPP, NPP>(pf[ks], b, o[n]);
                    }
            }
            const __amdgpu_buffer_rsrc_t rs = rsrc_of(out);
#pragma unroll
            for (int n = 0; n < CT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    store_if(col_in[n] && (more || wave * 16 + (int)g * 4 + j < len), rs,
                             sizeof(T) * (ooff + j * a.hv * a.dv + n * 16), from_float<T>(o[n][j]));
        }
        if constexpr (more) load_score(next);
    };
    for (int chunk = 0; chunk + 1 < chunks; ++chunk) step(chunk, std::true_type{});
    if (chunks > 0) step(chunks - 1, std::false_type{});
    if (a.final_state) write_state(a.final_state + sbase);
}

template <class T, int KS>
hipError_t forward_ks(const DeltaArgs &a, hipStream_t s) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3;
    const int slots = (int)delta_chunk_slots(a.tokens, a.n);
    if (a.tokens > 0) {
        if (a.before) {
            const int ld = (a.dk + 3) / 4 * 4 + 4;
            const size_t bytes = sizeof(float) * (2 * kC * ld + 3 * kC * kLd);
            if (hipError_t e = allow_lds(k_delta_prepare<T>, bytes)) return e;
            k_delta_prepare<T><<<dim3(slots, a.hk), 256, bytes, s>>>(a);
            if (hipError_t e = hipGetLastError()) return e;
        }
        constexpr size_t tile = sizeof(float) * kC * kLd, frags = 2 * 4 * KS * NP * kFrag;
        constexpr size_t bytes = tile + (frags > tile ? frags : tile);
        const auto even = [&](const void *p, int64_t stride) {
            return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * sizeof(T) % 16 == 0;
        };
        const bool vec = a.dk % 8 == 0 && even(a.q, a.qs) && even(a.k, a.ks);
        auto *kernel = vec ? k_delta_operands<T, KS, true> : k_delta_operands<T, KS, false>;
        if (hipError_t e = allow_lds(kernel, bytes)) return e;
        kernel<<<dim3(slots, a.hv), 256, bytes, s>>>(a);
        if (hipError_t e = hipGetLastError()) return e;
    }
    const auto walk = [&](auto ct) {
        constexpr int CT = decltype(ct)::value;
        const dim3 grid(a.n * a.hv, (a.dv + 16 * CT - 1) / (16 * CT));
        if (a.before) k_delta_walk<T, KS, CT, true><<<grid, 256, 0, s>>>(a);
        else k_delta_walk<T, KS, CT, false><<<grid, 256, 0, s>>>(a);
    };
    // Two column tiles a block share the left operands' loads; with too few
    // blocks for the CUs one tile's shorter chain counts more.  7 ragged sequences
    // of 8 heads (224 blocks of two tiles): 132 us with two, 105 with one; 256 of 4
    // heads: 41 us with two, 71 with one.
    if (a.dv <= 16 || a.n * a.hv * ((a.dv + 31) / 32) <= 256) walk(std::integral_constant<int, 1>{});
    else walk(std::integral_constant<int, 2>{});
    return hipGetLastError();
}

template <class T>
hipError_t forward(const DeltaArgs &a, hipStream_t s) {
    const int ks = delta_ksteps(a.dk);
    return ks == 1 ? forward_ks<T, 1>(a, s) : ks == 2 ? forward_ks<T, 2>(a, s) : forward_ks<T, 4>(a, s);
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
