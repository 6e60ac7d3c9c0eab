// Gradients of the gated delta rule over whole sequences.
//
// With the chunk quantities of rn_delta.hip (S and S' the memories before and
// after a chunk, E the errors, V' = beta E, P, c), M = I + A for
// A_ij = beta_i e^(ci - cj) k_i . k_j, and dS' = dJ/dS':
//   dV' = M^-T (P^T dO + (e^(c64 - c) K) dS'),
//   dS  = e^(c64) dS' + (scale e^c Q)^T dO - (beta e^c K)^T dV':
// k_delta_bwd_walk takes the chunks of a sequence from the last to the first and
// leaves dS' and dV'.  Then every chunk by itself (k_delta_bwd_chunk; short sequences:
// k_delta_short_grad), with
// dP = dO V'^T, dL = -beta dV' V'^T and e = e^(ci - cj) for j <= i:
//   dv = beta dV',  dbeta_i = dV'_i . E_i,
//   dq = scale (e^c dO S^T + (dP e) K),
//   dk = [-beta e^c dV' S^T + (dL e) K]                        (reads: k_i as the row)
//      + [e^(c64 - c) V' dS'^T + scale (dP e)^T Q + (dL e)^T K]  (writes: k_j as the column),
//   dc_i = q_i . dq_i + k_i . dk_i(reads) - k_i . dk_i(writes): every term of
//     these products holds e^(c_i) or e^(-c_i) once,
//   dc_64 also has sum_i e^(c64 - ci) k_i . (V' dS'^T)_i + e^(c64) <S, dS'>,
//   dg_t = sum over s >= t in the chunk of dc_s.
#include "rn_delta.hpp"

namespace rn {
namespace {

using namespace ops;

// Laid out as the forward walk: 16 CT columns a block, wave w the tokens
// 16 w .. + 15 and the gradient's row tiles w, w + 4, which stay in registers in
// float32 and go through LDS as planes, as do dO, scale e^c dO, the right side of
// the triangular system and -beta e^c dV'.  Bound as that is, by a chunk's chain:
// 8192 ragged tokens of 7 sequences and 8 heads of 128 x 128 in 120 us, 2.7 us a
// chunk of the longest.
template <class T, int KS, int CT>
__global__ __launch_bounds__(256, sizeof(T) == 4 && KS == 4 ? 1 : 2) void k_delta_bwd_walk(DeltaArgs a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3;
    constexpr int KP = KS * 32, RT = KP > 64 ? KP / 64 : 1;        // row tiles of the gradient a wave owns
    constexpr int VT = 16 * CT, ldS = KP + 8, ldT = kC + 8;
    constexpr int kKeys = 4 * KS * NP * kFrag;
    __shared__ __align__(16) uint16_t sS[3 * VT * ldS], sO[NP * VT * ldT], sG[3 * VT * ldT], sX[3 * VT * ldT], sL[3 * VT * ldT];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const WalkBlock at = walk_block(a);
    const int seq = at.seq, h = at.head, hk = h / (a.hv / a.hk), v0 = at.tile * VT;
    const Span span = span_of(a, seq);
    if (span.len <= a.short_len) return;                // taken token by token
    const int chunks = (span.len + kC - 1) / kC;
    const int64_t slot0 = slot_of(a, span.begin, seq);
    const int64_t sbase = ((int64_t)seq * a.hv + h) * a.dk * a.dv + v0;
    const bool owner = KP >= 64 || wave * 16 < KP;
    bool col_in[CT];
#pragma unroll
    for (int n = 0; n < CT; ++n) col_in[n] = v0 + n * 16 + (int)r < a.dv;

    f32x4 S[RT][CT];                                    // the gradient of the memory
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
                const bool in = a.dfinal && owner && d < a.dk && col_in[n];
                S[i][n][j] = in ? a.dfinal[sbase + (int64_t)d * a.dv + n * 16 + r] : 0.f;
            }

    // Loads are unconditional, as in the forward walk.
    bf16x8 kf[KS][NP], kt[RT][2][NP], qt[RT][2][NP], mf[2][3], pf[2][3];
    T od[CT][4];
    const auto load_k = [&](int64_t slot) {
        const int64_t at = (slot * a.hk + hk) * kKeys + wave * KS * NP * kFrag;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) load_frags<NP>(a.kf + at + (lane * 8 + ks * NP * kFrag), kf[ks]);
    };
    const auto load_kq = [&](int64_t slot) {
        const int64_t at = (slot * a.hk + hk) * kKeys + (wave % (2 * KS)) * 2 * NP * kFrag;
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                load_frags<NP>(a.kt + at + (lane * 8 + (8 * i + ks) * NP * kFrag), kt[i][ks]);
                load_frags<NP>(a.qt + at + (lane * 8 + (8 * i + ks) * NP * kFrag), qt[i][ks]);
            }
    };
    const auto load_tri = [&](const uint16_t *p, int64_t slot, bf16x8 (&f)[2][3]) {
        const uint16_t *at = p + (slot * a.hv + h) * kTri * 3 * kFrag;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
            load_frags<3>(at + tri_t(wave, wave < 2 ? ks : 1) * 3 * kFrag + lane * 8, f[ks]);
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
    uint32_t col[CT];
#pragma unroll
    for (int n = 0; n < CT; ++n) col[n] = min(n * 16 + (int)r, a.dv - 1 - v0);
    const uint32_t ooff = (wave * 16 + g * 4) * (uint32_t)(a.hv * a.dv) + r;
    const auto load_o = [&](int chunk) {
        const T *base = static_cast<const T *>(a.dout) + ((int64_t)(span.begin + chunk * kC) * a.hv + h) * a.dv + v0;
        const int last = span.len - chunk * kC - 1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t t = min(wave * 16 + (int)g * 4 + j, last) * (uint32_t)(a.hv * a.dv);
#pragma unroll
            for (int n = 0; n < CT; ++n) od[n][j] = base[t + col[n]];
        }
    };
    if (chunks > 0) {
        const int64_t slot = slot0 + chunks - 1;
        load_decays(slot), load_o(chunks - 1), load_k(slot), load_tri(a.pf, slot, pf), load_tri(a.mf, slot, mf), load_kq(slot);
    }
    put_state();

    const auto step = [&](int chunk, auto more_) {
        constexpr bool more = decltype(more_)::value;   // a chunk comes before this one
        const int64_t next = slot0 + chunk - 1, ch = (slot0 + chunk) * a.hv + h;
        const int len = min(kC, span.len - chunk * kC);
        const bool busy = wave * 16 < len;              // any token of this wave
        const bool half2 = len > 32;                    // tokens in the second 32
        grown = next_grown, left = next_left, beta = next_beta, whole = next_whole;
        if (chunk + 1 < chunks) write_state(a.after + ch * a.dk * a.dv + v0);
        f32x4 o[CT];
#pragma unroll
        for (int n = 0; n < CT; ++n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][j] = wave * 16 + (int)g * 4 + j < len ? to_float(od[n][j]) : 0.f;
            put4<NP>(sO, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, o[n]);
        }
        dev::lds_barrier();                             // planes of dS' and dO are there
        f32x4 x[CT];
#pragma unroll
        for (int n = 0; n < CT; ++n) {
            x[n] = f32x4{};
            if (busy) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    bf16x8 s[3];
                    get8<3>(sS, VT * ldS, (n * 16 + r) * ldS + ks * 32 + g * 8, s);
                    x[n] = mm<NP, 3>(kf[ks], s, x[n]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) x[n][j] *= left[j];
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    if (wave < 2 ? ks == 0 || half2 : ks == 1) {
                        bf16x8 b[NP];
                        get8<NP>(sO, VT * ldT, (n * 16 + r) * ldT + ks * 32 + g * 8, b);
                        x[n] = mm<3, NP>(pf[ks], b, x[n]);
                    }
            }
            put4<3>(sX, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, x[n]);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][j] *= grown[j] * a.scale;
            put4<3>(sG, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, o[n]);
        }
        if constexpr (more) load_decays(next), load_o(chunk - 1), load_k(next), load_tri(a.pf, next, pf);
        dev::lds_barrier();
        const __amdgpu_buffer_rsrc_t rs = rsrc_of(a.dwrite + ((int64_t)(span.begin + chunk * kC) * a.hv + h) * a.dv + v0);
#pragma unroll
        for (int n = 0; n < CT; ++n) {
            f32x4 w{};
            if (busy)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    if (wave < 2 ? ks == 0 || half2 : ks == 1) {
                        bf16x8 b[3];
                        get8<3>(sX, VT * ldT, (n * 16 + r) * ldT + ks * 32 + g * 8, b);
                        w = mm<3, 3>(mf[ks], b, w);
                    }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                store_if(col_in[n] && wave * 16 + (int)g * 4 + j < len, rs, 4 * (ooff + j * a.hv * a.dv + n * 16), (float)w[j]);
                w[j] *= -beta[j] * grown[j];
            }
            put4<3>(sL, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, w);
        }
        if constexpr (more) load_tri(a.mf, next, mf);
        dev::lds_barrier();
        if (owner)
#pragma unroll
            for (int n = 0; n < CT; ++n) {
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) S[i][n][j] *= whole;
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
                    if (ks == 0 || half2) {
                        bf16x8 b[3], c[3];
                        get8<3>(sG, VT * ldT, (n * 16 + r) * ldT + ks * 32 + g * 8, b);
                        get8<3>(sL, VT * ldT, (n * 16 + r) * ldT + ks * 32 + g * 8, c);
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            S[i][n] = mm<NP, 3>(qt[i][ks], b, S[i][n]);
                            S[i][n] = mm<NP, 3>(kt[i][ks], c, S[i][n]);
                        }
                    }
            }
        if constexpr (more) {
            put_state();                                // every wave is past its reads of the planes
            load_kq(next);
        }
    };
    for (int chunk = chunks - 1; chunk > 0; --chunk) step(chunk, std::true_type{});
    if (chunks > 0) step(0, std::false_type{});
    if (a.dstate) write_state(a.dstate + sbase);
}

// ------------------------------------------------------------------ a chunk by itself

// Elements from .. + 3 and from + 16 .. + 19 of a row of `count`, zeros where there
// are none; as loaded, so that a later step's can be on their way while this one
// is computed.  (Which of 32 elements a lane holds is free as long as both
// operands of a product agree; four lanes read 64 bytes on end this way.)  `row`
// is the row's offset in bytes from a base that the wave shares; nothing branches,
// as in store_if, so that each wait is for no more than it needs.
template <class T, bool VEC>
struct Raw8 {
    static constexpr int PER = VEC ? 4 : 1;             // VEC: count a multiple of 8, rows on 16 bytes
    Pack<T, PER> v[8 / PER];
    __device__ void load(__amdgpu_buffer_rsrc_t p, bool in, uint32_t row, int from, int count) {
#pragma unroll
        for (int e = 0; e < 8; e += PER) {
            const int at = from + (e < 4 ? e : e + 12);
            v[e / PER] = load_if<Pack<T, PER>>(in && at < count, p, row + sizeof(T) * at);
        }
    }
    __device__ void store(__amdgpu_buffer_rsrc_t p, bool in, uint32_t row, int from, int count) const {
#pragma unroll
        for (int e = 0; e < 8; e += PER) {
            const int at = from + (e < 4 ? e : e + 12);
            store_if(in && at < count, p, row + sizeof(T) * at, v[e / PER]);
        }
    }
    __device__ void get(float (&f)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = to_float(v[e / PER].v[e % PER]);
    }
    __device__ void set(const float (&f)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e / PER].v[e % PER] = from_float<T>(f[e]);
    }
};
template <int N>
__device__ inline void planes8(const float (&v)[8], bf16x8 (&f)[N]) {
    uint32_t w[4][N];
#pragma unroll
    for (int e = 0; e < 4; ++e) split_pair<N>(v[2 * e], v[2 * e + 1], w[e]);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = __builtin_bit_cast(bf16x8, u32x4{w[0][i], w[1][i], w[2][i], w[3][i]});
}

// A block takes a chunk slot and a key head and adds the value heads that share
// it.  All big products sum over the values, 32 at a time: rows of dO, dV', E, S
// and dS' are operands as they lie in memory.  The waves split them into planes
// once for all, through LDS, while the next step's are on their way.  dk above 64
// takes eight waves: w and w + 4 own 16 tokens, half of dk's row tiles of dq,
// dk(reads) and dk(writes) in the registers of each (four waves that own all of
// dk fill the registers with these sums, and no second wave a SIMD covers the
// first one's waits: 274 us for 8192 ragged tokens of 8 heads, 182 with eight;
// 155 with loads that do not branch).
// Up to 64 four waves do: for a chunk of 16 tokens one of four works.
// SHARED keeps dq's and dk's sums over the heads in registers too, and from dk 33 on
// does not fit into the 256 there are: 2 and 3 of them spill for bfloat16 above 64, 31
// for float32, 22 to 71 for four waves of 33 to 64.
template <class T, int KS, bool VEC, bool SHARED>
__global__ __launch_bounds__(KS == 4 ? 512 : 256, 2) void k_delta_bwd_chunk(DeltaArgs a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3, KT = 2 * KS, PARTS = KS == 4 ? 2 : 1, HT = KT / PARTS;
    constexpr int kKeys = 4 * KS * NP * kFrag;
    constexpr int kStep = (2 * KT * 3 + 4 * (6 + NP)) * kFrag * 2, kPairs = 2 * kC * kLd * 4;   // bytes of the two uses
    __shared__ __align__(16) char lds[kStep > kPairs ? kStep : kPairs];
    uint16_t *fS = reinterpret_cast<uint16_t *>(lds), *fD = fS + KT * 3 * kFrag;
    uint16_t *fV = fD + KT * 3 * kFrag, *fR = fV + 4 * 3 * kFrag, *fO = fR + 4 * 3 * kFrag;     // V', dv, dO by 16 tokens
    float *x = reinterpret_cast<float *>(lds), *y = x + kC * kLd;   // [i][j] of dP e and dL e
    __shared__ double cs[kC];
    __shared__ float beta_s[kC], dc[PARTS][kC], extra[4 * PARTS];
    const int slot = blockIdx.x, hk = blockIdx.y, group = a.hv / a.hk;
    const Chunk c{a.map[4 * slot + 2], a.map[4 * slot], a.map[4 * slot + 1], 0, a.map[4 * slot + 3] != 0};
    if (c.len == 0) return;
    const int wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = wave8 & 3;
    const int part = PARTS > 1 ? wave8 >> 2 : 0;
    const uint32_t lane_ = threadIdx.x & 63;
    const int blocks = (c.len + 15) / 16, half = (c.len + 31) / 32;
    const bool busy = wave < blocks;
    const int64_t keys = ((int64_t)slot * a.hk + hk) * kKeys, kept = kept_slot_of(c.begin, c.seq);
    // Sum over the 16 lanes that hold a row's columns.
    const auto across = [&](float v) {
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) v += __shfl_xor(v, s);
        return v;
    };
    f32x4 tq[HT], tk[HT];                               // over the value heads (SHARED)
#pragma unroll
    for (int n = 0; n < HT; ++n) tq[n] = tk[n] = f32x4{};
    for (int h = hk * group;; ++h) {
        // The lane anew for each head: offsets from it are not kept from head to
        // head, which would cost more registers than there are.
        uint32_t lane = lane_, r = lane & 15, g = lane >> 4;
        asm volatile("" : "+v"(lane), "+v"(r), "+v"(g));
        const int token = wave * 16 + (int)r;           // as an operand's row
        const int row4 = wave * 16 + (int)g * 4;        // as a result's rows
        const int64_t ch = (int64_t)slot * a.hv + h;
        __syncthreads();
        if (wave8 == 0) {
            cs[lane] = decay_sums(a, c, h);
            beta_s[lane] = (int)lane < c.len ? a.beta[(int64_t)(c.begin + lane) * a.hv + h] : 0.f;
        }
        __syncthreads();
        // pr: dP and dL (with two parts, dP with the one and dL with the other)
        f32x4 gq[HT], gr[HT], gw[HT], pr[3 - PARTS][4];
#pragma unroll
        for (int n = 0; n < HT; ++n) gq[n] = gr[n] = gw[n] = f32x4{};
#pragma unroll
        for (int n = 0; n < 4; ++n) pr[0][n] = pr[2 - PARTS][n] = f32x4{};
        float db = 0.f, dot = 0.f;
        const float b = beta_s[token];
        const int64_t row0 = ((int64_t)c.begin * a.hv + h) * a.dv;
        const uint32_t row = token * (uint32_t)(a.hv * a.dv);
        const bool in = token < c.len;
        constexpr int W8 = 4 * PARTS, RT = KT > W8 ? KT / W8 : 1;       // row tiles of S and dS' a wave splits
        Raw8<float, VEC> rs[RT], rt[RT], rw, re;
        Raw8<T, VEC> ro, rv{};
        // the gradient of the memory after the chunk: dfinal after a sequence's last
        const int64_t mem = (int64_t)a.dk * a.dv;
        const bool no_after = c.last && !a.dfinal;
        const __amdgpu_buffer_rsrc_t pS = rsrc_of(a.before + (kept * a.hv + h) * mem), pE = rsrc_of(a.err + row0), pW = rsrc_of(a.dwrite + row0);
        const __amdgpu_buffer_rsrc_t pD = rsrc_of(c.last && a.dfinal ? a.dfinal + ((int64_t)c.seq * a.hv + h) * mem : a.after + ch * mem);
        const __amdgpu_buffer_rsrc_t pO = rsrc_of(static_cast<const T *>(a.dout) + row0);
        const __amdgpu_buffer_rsrc_t pV = rsrc_of(static_cast<T *>(a.dval) + row0);
        const auto fetch = [&](int v) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int d = (wave8 + W8 * i) * 16 + (int)r;
                rs[i].load(pS, d < a.dk, d * a.dv * 4, v, a.dv);
                rt[i].load(pD, d < a.dk && !no_after, d * a.dv * 4, v, a.dv);
            }
            rw.load(pW, in, row * 4, v, a.dv);
            re.load(pE, in && part == 0, row * 4, v, a.dv);
            ro.load(pO, in && part == 0, row * sizeof(T), v, a.dv);
        };
        fetch(g * 4);
        for (int v0 = 0; v0 < a.dv; v0 += 32) {
            const int v = v0 + (int)g * 4;
            const auto put = [&](uint16_t *to, const auto &f) {
#pragma unroll
                for (int p = 0; p < (int)(sizeof(f) / sizeof(f[0])); ++p) *reinterpret_cast<bf16x8 *>(to + p * kFrag + lane * 8) = f[p];
            };
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int n = wave8 + W8 * i;
                if (n < KT) {
                    float s[8], t[8];
                    rs[i].get(s), rt[i].get(t);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot = fmaf(s[e], t[e], dot);
                    bf16x8 f[3];
                    planes8<3>(s, f);
                    put(fS + n * 3 * kFrag, f);
                    planes8<3>(t, f);
                    put(fD + n * 3 * kFrag, f);
                }
            }
            if (busy) {
                float w[8];
                bf16x8 f[3];
                rw.get(w);
                if (part == 0) {
                    float o[8], e[8];
                    bf16x8 fo[NP];
                    ro.get(o), re.get(e);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        db = fmaf(w[i], e[i], db);
                        e[i] *= b;
                    }
                    planes8<NP>(o, fo);
                    put(fO + wave * NP * kFrag, fo);
                    planes8<3>(e, f);                   // V'
                    put(fV + wave * 3 * kFrag, f);
                }
                if (part == PARTS - 1) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] *= b;
                    planes8<3>(w, f);                   // beta dV', which is dv
                    put(fR + wave * 3 * kFrag, f);
                    rv.set(w);
                }
            }
            fetch(v + 32);                              // nothing past the last column
            rv.store(pV, in && part == PARTS - 1, row * sizeof(T), v, a.dv);
            dev::lds_barrier();                         // which leaves those loads in flight
            if (busy) {
                bf16x8 fo[NP], fr[3], fv[3];
                load_frags<NP>(fO + wave * NP * kFrag + lane * 8, fo);
                load_frags<3>(fR + wave * 3 * kFrag + lane * 8, fr);
                load_frags<3>(fV + wave * 3 * kFrag + lane * 8, fv);
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (n <= wave) {
                        bf16x8 f[3];
                        load_frags<3>(fV + n * 3 * kFrag + lane * 8, f);
                        if (part == 0) pr[0][n] = mm<NP, 3>(fo, f, pr[0][n]);
                        if (part == PARTS - 1) pr[2 - PARTS][n] = mm<3, 3>(fr, f, pr[2 - PARTS][n]);
                    }
#pragma unroll
                for (int n = 0; n < HT; ++n) {
                    bf16x8 f[3];
                    load_frags<3>(fS + (part * HT + n) * 3 * kFrag + lane * 8, f);
                    gq[n] = mm<NP, 3>(fo, f, gq[n]);
                    gr[n] = mm<3, 3>(fr, f, gr[n]);
                    load_frags<3>(fD + (part * HT + n) * 3 * kFrag + lane * 8, f);
                    gw[n] = mm<3, 3>(fv, f, gw[n]);
                }
            }
            dev::lds_barrier();
        }
        // dbeta: a row's four lanes
        db += __shfl_xor(db, 16);
        db += __shfl_xor(db, 32);
        if (part == 0 && g == 0 && in) a.dbeta[(int64_t)(c.begin + token) * a.hv + h] = db;
        // K^T's and Q^T's pieces of this wave, a few ahead of their use.
        constexpr int AHEAD = 2;
        bf16x8 fk[AHEAD][NP], fq[AHEAD][NP];
        const auto ask = [&](int i) {                   // piece i: k step i / HT, row tile i % HT
            const int at = ((part * HT + i % HT) * 2 + i / HT) * NP * kFrag;
            load_frags<NP>(a.kt + (keys + at) + lane * 8, fk[i % AHEAD]);
            load_frags<NP>(a.qt + (keys + at) + lane * 8, fq[i % AHEAD]);
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) ask(i);
        // Where this lane's results lie in k and q: offsets from bases that the wave
        // shares, clamped into the rows (results there are 0).
        const T *kbase = static_cast<const T *>(a.k) + (int64_t)c.begin * a.ks + hk * a.dk;
        const T *qbase = static_cast<const T *>(a.q) + (int64_t)c.begin * a.qs + hk * a.dk;
        T kr[4][HT], qr[4][HT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t t = min(row4 + j, c.len - 1);
#pragma unroll
            for (int n = 0; n < HT; ++n) {
                const uint32_t d = min((part * HT + n) * 16 + (int)r, a.dk - 1);
                kr[j][n] = kbase[t * (uint32_t)a.ks + d];
                qr[j][n] = qbase[t * (uint32_t)a.qs + d];
            }
        }
        const double last = cs[kC - 1];
        // the pairs' weights
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = row4 + j, u = n * 16 + (int)r;
                const float d = u <= t && n <= wave ? decay(cs[t] - cs[u]) : 0.f;
                if (part == 0) x[t * kLd + u] = u <= t ? pr[0][n][j] * d * a.scale : 0.f;
                if (part == PARTS - 1) y[t * kLd + u] = u < t ? -pr[2 - PARTS][n][j] * d : 0.f;
            }
        // The memory's part of the sums, before the pairs' is added.
        float wsum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = row4 + j;
            const float grown = decay(cs[t]), left = decay(last - cs[t]);
#pragma unroll
            for (int n = 0; n < HT; ++n) {
                gq[n][j] *= grown * a.scale;
                gr[n][j] *= -grown;
                gw[n][j] *= left;
                wsum = fmaf(gw[n][j], to_float(kr[j][n]), wsum);
            }
        }
        float all = fmaf(dot, decay(last), wsum);
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) all += __shfl_xor(all, s);
        if (lane == 0) extra[wave8] = all;
        dev::lds_barrier();
        if (busy) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                // rows i of dP e and dL e for the reads, columns for the writes
                bf16x8 fx[3], fy[3], fxt[3], fyt[3];
                const bool lower = ks <= wave / 2, upper = ks >= wave / 2;
                float v[8], w[8];
                const float *px = x + token * kLd + ks * 32 + g * 8, *py = px + kC * kLd;
                if (ks < half && lower) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = px[e], w[e] = py[e];
                    planes8<3>(v, fx);
                    planes8<3>(w, fy);
                }
                if (ks < half && upper) {
                    const float *tx = x + (ks * 32 + g * 8) * kLd + token, *ty = tx + kC * kLd;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = tx[e * kLd], w[e] = ty[e * kLd];
                    planes8<3>(v, fxt);
                    planes8<3>(w, fyt);
                }
#pragma unroll
                for (int n = 0; n < HT; ++n) {
                    const int i = ks * HT + n;
                    __builtin_amdgcn_sched_barrier(0);  // or all pieces' loads are hoisted, and spilled
                    if (ks < half) {
                        if (lower) {
                            gq[n] = mm<3, NP>(fx, fk[i % AHEAD], gq[n]);
                            gr[n] = mm<3, NP>(fy, fk[i % AHEAD], gr[n]);
                        }
                        if (upper) {
                            gw[n] = mm<3, NP>(fxt, fq[i % AHEAD], gw[n]);
                            gw[n] = mm<3, NP>(fyt, fk[i % AHEAD], gw[n]);
                        }
                    }
                    if (i + AHEAD < 2 * HT) ask(i + AHEAD);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float s = 0.f;
#pragma unroll
            for (int n = 0; n < HT; ++n) {
                s = fmaf(gq[n][j], to_float(qr[j][n]), s);
                s = fmaf(gr[n][j] - gw[n][j], to_float(kr[j][n]), s);
                tq[n][j] = SHARED ? tq[n][j] + gq[n][j] : gq[n][j];
                tk[n][j] = SHARED ? tk[n][j] + (gr[n][j] + gw[n][j]) : gr[n][j] + gw[n][j];
            }
            s = across(s);
            if (r == 0) dc[part][row4 + j] = s;
        }
        __syncthreads();
        if (wave8 == 0) {
            double s = PARTS > 1 ? (double)dc[0][lane] + dc[PARTS - 1][lane] : (double)dc[0][lane];
            if (lane == kC - 1u) {
#pragma unroll
                for (int i = 0; i < 4 * PARTS; ++i) s += extra[i];
            }
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const double u = __shfl_down(s, d);
                if ((int)lane + d < 64) s += u;
            }
            if ((int)lane < c.len) a.dg[(int64_t)(c.begin + lane) * a.hv + h] = (float)s;
        }
        if (!SHARED || h + 1 == (hk + 1) * group) break;
    }
    const uint32_t r = lane_ & 15;
    const int row4 = wave * 16 + (int)(lane_ >> 4) * 4;
    const __amdgpu_buffer_rsrc_t rq = rsrc_of(static_cast<T *>(a.dq) + ((int64_t)c.begin * a.hk + hk) * a.dk);
    const __amdgpu_buffer_rsrc_t rk = rsrc_of(static_cast<T *>(a.dkey) + ((int64_t)c.begin * a.hk + hk) * a.dk);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int t = row4 + j;
#pragma unroll
        for (int n = 0; n < HT; ++n) {
            const int d = (part * HT + n) * 16 + (int)r;
            const uint32_t at = t * (uint32_t)(a.hk * a.dk) + d;
            store_if(t < c.len && d < a.dk, rq, sizeof(T) * at, from_float<T>(tq[n][j]));
            store_if(t < c.len && d < a.dk, rk, sizeof(T) * at, from_float<T>(tk[n][j]));
        }
    }
}

template <class T, int KS>
hipError_t backward_ks(const DeltaArgs &a, hipStream_t s) {
    if (hipError_t e = launch_operands<T, KS, true>(a, s)) return e;
    if (walk_tiles(a) == 1) k_delta_bwd_walk<T, KS, 1><<<walk_grid(a, 16), 256, 0, s>>>(a);
    else k_delta_bwd_walk<T, KS, 2><<<walk_grid(a, 32), 256, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    const dim3 grid((int)delta_slots(a.tokens, a.n, !a.off), a.hk);
    const auto even = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    const bool vec = a.dv % 8 == 0 && even(a.dout) && even(a.dval) && even(a.dfinal);
    const auto chunk = [&](auto vec_) {
        constexpr bool VEC = decltype(vec_)::value;
        if (a.hv > a.hk) k_delta_bwd_chunk<T, KS, VEC, true><<<grid, KS == 4 ? 512 : 256, 0, s>>>(a);
        else k_delta_bwd_chunk<T, KS, VEC, false><<<grid, KS == 4 ? 512 : 256, 0, s>>>(a);
    };
    if (vec) chunk(std::true_type{});
    else chunk(std::false_type{});
    return hipGetLastError();
}

template <class T>
hipError_t backward(const DeltaArgs &a, hipStream_t s) {
    const int ks = delta_ksteps(a.dk);
    return ks == 1 ? backward_ks<T, 1>(a, s) : ks == 2 ? backward_ks<T, 2>(a, s) : backward_ks<T, 4>(a, s);
}

}  // namespace

hipError_t launch_delta_backward(const DeltaArgs &args, bool bf16, hipStream_t s) {
    DeltaArgs a = args;
    const DeltaWays w = delta_ways(a.tokens, a.n, !a.off);
    a.short_len = w.tokens ? kShort : -1;
    if (w.tokens)
        if (hipError_t e = launch_delta_short_backward(a, bf16, s)) return e;
    if (!w.chunks) return hipSuccess;
    return bf16 ? backward<bf16_t>(a, s) : backward<float>(a, s);
}

}  // namespace rn
