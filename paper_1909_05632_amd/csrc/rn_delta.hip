// The gated delta rule: one token a stream (the step), and whole sequences.
//
//   S <- e^g S;  S <- S + beta k (v - S^T k)^T;  out = scale S^T q.
//
// Sequences are taken in chunks of 64 tokens.  With c the sums of g within the
// chunk, S the memory before it and V' the values as written,
//   V' = beta E,  (I + A) E = V - e^c K S,   A_ij = e^(ci - cj) k_i . k_j beta_j  (j < i),
//   O  = scale e^c Q S + P V',               P_ij = scale e^(ci - cj) q_i . k_j   (j <= i),
//   S' = e^(c64) S + (e^(c64 - c) K)^T V'.
// E is v - S_t^T k, the error that each token meets.  (I + A)^-1 and P do not
// depend on S: k_delta_operands (rn_delta.hpp) makes them for all chunks at once.
// k_delta_walk then goes through a sequence's chunks in order; columns of S do not
// meet, so each block takes 16 or 32 of a head's.  Sequences of up to 32 tokens go
// token by token where a call has many (rn_delta_short.hip).
#include "rn_delta.hpp"

namespace rn {
namespace {

using namespace ops;

// ------------------------------------------------------------------ one token

// A block owns one stream's head.  Its memory is read once into registers and
// written once: VEC columns a thread, `lanes` threads across the columns, the
// 256 / lanes groups each with every such row.  Bound by HBM (the memory's
// 2 dk dv float32 outweigh all else): 1024 streams of 8 heads of 128 x 128, 218 us,
// 4.9 TB/s; one stream's 4 heads of 64 x 64 take 4.8 us, latency.
template <class T, int VEC, int ROWS>
__global__ __launch_bounds__(256) void k_delta_step(DeltaArgs a, int lanes) {
    __shared__ float sq[RN_DELTA_MAX_DIM], sk[RN_DELTA_MAX_DIM];
    __shared__ float red[256 * VEC];
    const int head = blockIdx.x, i = blockIdx.y;
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
    const dim3 blocks(a.hv, a.n);                       // one axis holds 2^32 threads, fewer than n hv blocks may have
    if (rows <= 4) k_delta_step<T, VEC, 4><<<blocks, 256, 0, s>>>(a, lanes);
    else if (rows <= 16) k_delta_step<T, VEC, 16><<<blocks, 256, 0, s>>>(a, lanes);
    else if constexpr (VEC == 1) k_delta_step<T, VEC, 64><<<blocks, 256, 0, s>>>(a, lanes);
}

// ------------------------------------------------------------------ chunks

// A sequence's chunks in order.  A block takes 16 CT columns of a head's memory,
// wave w the tokens 16 w .. + 15 of a chunk and the memory's row tiles w, w + 4;
// the memory stays in its owners' registers in float32, and goes through LDS as
// bf16 planes to the waves that multiply by it, as do V - e^c K S and V'.
// The left operands are read from memory in fragment order, straight into
// registers, each for the next chunk as soon as this one's use of it is over.
// S, V' and P have three planes in all products: outputs of bfloat16 data too are
// sums of float32 before they are rounded (with two planes in the output's products
// those differ from float32's by 1.4e-4 after rounding in place of 4e-5, and
// the walk below takes 230 us).
// Bound by a chunk's chain of four products with barriers between them, 2.9 us a
// chunk (bfloat16, 128 x 128, two blocks a CU), in which the matrix cores are busy a
// fifth of the time: 16384 tokens of 5 sequences and 16 heads in 256 us, 101
// TFLOP/s of the rule's own operations (25.8 GFLOP).
template <class T, int KS, int CT, bool SAVE>
__global__ __launch_bounds__(256, sizeof(T) == 4 && KS == 4 ? 1 : 2) void k_delta_walk(DeltaArgs a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3;
    constexpr int KP = KS * 32, RT = KP > 64 ? KP / 64 : 1;        // row tiles of the memory a wave owns
    constexpr int VT = 16 * CT, ldS = KP + 8, ldT = kC + 8;
    constexpr int kKeys = 4 * KS * NP * kFrag;
    __shared__ __align__(16) uint16_t sS[3 * VT * ldS], sR[3 * VT * ldT], sV[3 * VT * ldT], sL[3 * VT * ldT];
    __shared__ int sBad[VT];                            // a column's first token in the chunk that is not finite
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
    bf16x8 kf[KS][NP], qf[KS][NP], kt[RT][2][NP], mf[2][3], pf[2][3];
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
        const int64_t at = (slot * a.hv + h) * kTri * 3 * kFrag;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) load_frags<3>(a.pf + (at + tri(wave, min(ks, wave / 2)) * 3 * kFrag) + lane * 8, pf[ks]);
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
    if (threadIdx.x < VT) sBad[threadIdx.x] = kC;
    put_state();

    const auto step = [&](int chunk, auto more_) {
        constexpr bool more = decltype(more_)::value;   // every chunk but the last: 64 tokens, and one follows
        const int64_t next = slot0 + chunk + 1;
        const int len = more ? kC : span.len - chunk * kC;
        const bool busy = more || wave * 16 < len;      // any token of this wave
        const bool half2 = more || len > 32;            // tokens in the second 32
        grown = next_grown, left = next_left, beta = next_beta, whole = next_whole;
        if constexpr (SAVE) {
            const int64_t kept = kept_slot_of(span.begin, seq) + chunk;
            write_state(a.before + (kept * a.hv + h) * a.dk * a.dv + v0);
        }
        dev::lds_barrier();                             // the memory's planes are there
        f32x4 o[CT];
#pragma unroll
        for (int n = 0; n < CT; ++n) {
            f32x4 held{};
            o[n] = f32x4{};
            if (busy)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    bf16x8 s[3];
                    get8<3>(sS, VT * ldS, (n * 16 + r) * ldS + ks * 32 + g * 8, s);
                    held = mm<NP, 3>(kf[ks], s, held);
                    o[n] = mm<NP, 3>(qf[ks], s, o[n]);
                }
            // Where a gap (or k, g or beta: beta is NaN) is not finite, the column is
            // NaN from that token on; its products are made with 0, so that the tokens
            // before it keep theirs.  (The memory is then NaN, and so is every gap of the
            // chunks that follow.)
            f32x4 w;
            int bad = kC;
#pragma unroll
            for (int j = 3; j >= 0; --j) {
                const int t = wave * 16 + (int)g * 4 + j;
                const float gap = to_float(vv[n][j]) - grown[j] * held[j];
                const bool in = more || t < len, out = in && max(magnitude(gap), magnitude(beta[j])) >= kHuge;
                bad = out ? t : bad;
                w[j] = in && !out ? gap : 0.f;
                o[n][j] *= grown[j] * a.scale;
            }
            if (__any(bad < kC)) atomicMin(&sBad[n * 16 + r], bad);
            put4<3>(sR, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, w);
        }
        if constexpr (more) load_decays(next), load_rows(next), load_v(chunk + 1);
        dev::lds_barrier();
        int from[CT];                                   // the columns' first tokens of NaN
        bool spoilt = false;
#pragma unroll
        for (int n = 0; n < CT; ++n) from[n] = sBad[n * 16 + r], spoilt = spoilt || from[n] < kC;
        spoilt = __any(spoilt);
        const auto spoil = [&](int n, f32x4 &v) {       // rows of this wave's tokens
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = wave * 16 + (int)g * 4 + j >= from[n] ? kNaN : v[j];
        };
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
            if constexpr (SAVE) {
                f32x4 e = w;
                if (spoilt) spoil(n, e);
                const __amdgpu_buffer_rsrc_t rs = rsrc_of(a.err + ((int64_t)(span.begin + chunk * kC) * a.hv + h) * a.dv + v0);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    store_if(col_in[n] && (more || wave * 16 + (int)g * 4 + j < len), rs,
                             4 * (ooff + j * a.hv * a.dv + n * 16), (float)e[j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] *= beta[j] == beta[j] ? beta[j] : 0.f;
            put4<3>(sV, VT * ldT, (n * 16 + r) * ldT + wave * 16 + g * 4, w);
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
                    if (spoilt && from[n] < kC) S[i][n] = f32x4{kNaN, kNaN, kNaN, kNaN};
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
                        bf16x8 b[3];
                        get8<3>(sV, VT * ldT, (n * 16 + r) * ldT + ks * 32 + g * 8, b);
                        o[n] = mm<3, 3>(pf[ks], b, o[n]);
                    }
                if (spoilt) spoil(n, o[n]);
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
    if (hipError_t e = launch_operands<T, KS, false>(a, s)) return e;
    const auto walk = [&](auto ct) {
        constexpr int CT = decltype(ct)::value;
        const dim3 grid = walk_grid(a, 16 * CT);
        if (a.before) k_delta_walk<T, KS, CT, true><<<grid, 256, 0, s>>>(a);
        else k_delta_walk<T, KS, CT, false><<<grid, 256, 0, s>>>(a);
    };
    if (walk_tiles(a) == 1) walk(std::integral_constant<int, 1>{});
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

hipError_t launch_delta_forward(const DeltaArgs &args, bool bf16, hipStream_t s) {
    DeltaArgs a = args;
    const DeltaWays w = delta_ways(a.tokens, a.n, !a.off);
    a.short_len = w.tokens ? kShort : -1;
    if (w.tokens)
        if (hipError_t e = launch_delta_short_forward(a, bf16, s)) return e;
    if (!w.chunks) return hipSuccess;
    return bf16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}

}  // namespace rn
