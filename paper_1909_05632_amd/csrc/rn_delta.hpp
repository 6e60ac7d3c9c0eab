// Device code that the gated delta rule's kernels share.
#pragma once

#include <type_traits>

#include "rn_ops.hpp"
#include "rn_split.hpp"

namespace rn {
namespace ops {

constexpr int kC = RN_DELTA_CHUNK;   // tokens of a chunk
constexpr int kLd = kC + 4;          // row length of a 64-wide LDS tile, off the banks' stride

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// One 16x16 tile of A B on the float32 matrix cores, added to acc.  a(i, k) and
// b(k, j) read the operands; kk (a multiple of 4) is the summed length.  Lane l
// gives A's row l % 16 and B's column l % 16 at k = l / 16, and holds rows
// 4 (l / 16) .. + 3 of column l % 16 of the result.
template <class A, class B>
__device__ inline f32x4 tile_mm(int kk, A &&a, B &&b, f32x4 acc) {
    const int r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    for (int k = 0; k < kk; k += 4) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a(r, k + g), b(k + g, r), acc, 0, 0, 0);
    return acc;
}

// Sequence i's tokens, clipped to the arrays whatever the offsets say.
struct Span {
    int begin, len;
};
__device__ inline int offset_of(const DeltaArgs &a, int i) {
    const int64_t t = a.off ? a.off[i] : a.tokens / a.n * i;
    return (int)(t < 0 ? 0 : t < a.tokens ? t : a.tokens);
}
__device__ inline Span span_of(const DeltaArgs &a, int i) {
    const int b = offset_of(a, i), e = offset_of(a, i + 1);
    return {b, e > b ? e - b : 0};
}
// The slot of sequence i's first chunk among the operands (delta_slots), and among
// the memories kept (delta_kept_slots); the next chunks' follow.
__device__ inline int slot_of(const DeltaArgs &a, int begin, int i) {
    return a.short_len >= 0 ? begin / kShort : begin / kC + i;
}
__device__ inline int kept_slot_of(int begin, int i) { return begin / kC + i; }

// The sequence and chunk of a chunk slot: the last sequence whose first slot is
// not beyond it.  Slots that no chunk has give len 0, or a sequence taken token by
// token.
struct Chunk {
    int seq, begin, len;          // tokens begin .. begin + len - 1, len <= 64
    int whole;                    // tokens of the sequence
    bool last;                    // the sequence's last chunk
};
__device__ inline Chunk chunk_of(const DeltaArgs &a, int slot) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {                                   // 64 places at once
        const int step = (hi - lo + 63) / 64, at = lo + ((int)(threadIdx.x & 63) + 1) * step;
        const bool up = at <= hi && slot_of(a, offset_of(a, min(at, hi)), at) <= slot;
        lo += __popcll(__ballot(up)) * step;
        hi = min(hi, lo + step - 1);
    }
    const Span s = span_of(a, lo);
    const int64_t at = (int64_t)(slot - slot_of(a, s.begin, lo)) * kC;
    if (at < 0 || at >= s.len) return {lo, 0, 0, 0, false};
    return {lo, s.begin + (int)at, min(kC, s.len - (int)at), s.len, at + kC >= s.len};
}

// A walk's blocks take the sequences from the longest to the shortest, so that
// no long chain begins when others have ended; within one the column tiles of a
// head are 8 k blocks apart where heads are a multiple of 8, on one XCD, whose
// cache then serves its operands to all of them.  Beyond 64 sequences (a lane each)
// they stay in order: the more there are, the less the last one counts.
struct WalkBlock {
    int seq, head, tile;
};
__device__ inline WalkBlock walk_block(const DeltaArgs &a) {
    const int i = blockIdx.x;
    int seq = blockIdx.y;
    if (a.off && a.n > 1 && a.n <= 64) {
        const int lane = threadIdx.x & 63, len = lane < a.n ? span_of(a, lane).len : -1;
        int before = 0;
        for (int j = 0; j < a.n; ++j) {
            const int l = __builtin_amdgcn_readlane(len, j);
            before += l > len || (l == len && j < lane);
        }
        seq = __ffsll((unsigned long long)__ballot(before == seq)) - 1;
    }
    return {seq, i % a.hv, i / a.hv};
}
// Sequences on an axis of their own: one axis holds no more than 2^32 threads, and
// a larger grid is cut off without an error.
inline dim3 walk_grid(const DeltaArgs &a, int width) { return dim3(a.hv * ((a.dv + width - 1) / width), a.n); }

// Log decays (base 2) summed up to each token of a chunk, in double: differences
// of far tokens stay exact to float32 where the sums are large.  An empty memory
// (g = -infinity) is a decay of e^-10^6 = 0, whose differences are finite.
// Tokens past the end count as g = 0, and so do those of NaN or +infinity where `bad`
// is there to be told of them.  One wave calls it; lane = token.
__device__ inline double decay_sums(const DeltaArgs &a, const Chunk &c, int head, bool *bad = nullptr) {
    const int lane = threadIdx.x & 63;
    float g = lane < c.len ? a.g[(int64_t)(c.begin + lane) * a.hv + head] : 0.f;
    if (bad && !(g < __builtin_huge_valf())) *bad = true, g = 0.f;
    double s = (g < -1e6f ? -1e6 : (double)g) * 1.4426950408889634;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double t = __shfl_up(s, d);
        if (lane >= d) s += t;
    }
    return s;
}
// 2^d: the hardware's, exact to an ulp where the result is a normal float32.
__device__ inline float decay(double d) { return __builtin_amdgcn_exp2f((float)d); }

// What counts as infinite: the magnitudes that round to infinity as a bf16 plane, in
// float32 those from 3.39e38 on.  A product with a plane of them is NaN, also where
// the other factor is the 0 of a triangular operand, so that a token's would reach
// the tokens before it.
constexpr uint32_t kHuge = 0x7f7f8000;
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr float kNaN = __builtin_nanf("");

template <class T>
__device__ inline float load(const void *p, int64_t i) {
    return to_float(static_cast<const T *>(p)[i]);
}

// ---- products on the bf16 matrix cores
//
// A float32 operand is a sum of bf16 planes (rn_split.hpp), three for the bits
// of float32; a bfloat16 input is one plane exactly.  A product of operands of
// NA and NB planes takes the terms (i, j) with i + j < max(NA, NB): what is
// dropped is below the last plane kept.
//
// Fragment order: a 16 x 32 piece of an operand is 64 lanes x 8 bf16, lane l
// holding row (B operand: column) l % 16 at k = 8 (l / 16) .. + 7, so one
// 16-byte access a lane reads or writes it.  The result's lane l holds rows
// 4 (l / 16) .. + 3 of column l % 16.
using dev::bf16x8;
constexpr int kFrag = 512;           // bf16 of a fragment

template <int NA, int NB>
__device__ inline f32x4 mm(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], f32x4 acc) {
    constexpr int N = NA > NB ? NA : NB;
#pragma unroll
    for (int s = N - 1; s >= 0; --s)             // small terms first
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[s - i], acc, 0, 0, 0);
    return acc;
}

template <int N>
__device__ inline void load_frags(const uint16_t *p, bf16x8 (&f)[N]) {      // p: this lane's part of plane 0
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = *reinterpret_cast<const bf16x8 *>(p + i * kFrag);
}

// The N planes of a pair of float32 values, each plane's pair in one word.
template <int N>
__device__ inline void split_pair(float x, float y, uint32_t (&p)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p[i] = dev::round_pair(x, y);
        if (i + 1 < N) x -= dev::pair_lo(p[i]), y -= dev::pair_hi(p[i]);
    }
}

// Four consecutive k of one column into N planes of an LDS operand [column][ld].
template <int N>
__device__ inline void put4(uint16_t *lds, int plane, int at, const f32x4 v) {
    uint32_t a[N], b[N];
    split_pair<N>(v[0], v[1], a);
    split_pair<N>(v[2], v[3], b);
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<u32x2 *>(lds + i * plane + at) = u32x2{a[i], b[i]};
}
template <int N>
__device__ inline void get8(const uint16_t *lds, int plane, int at, bf16x8 (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = *reinterpret_cast<const bf16x8 *>(lds + i * plane + at);
}

// Loads that give 0 and stores that are dropped where `in` is false, without a
// branch: the compiler can then count what is in flight and wait for no more than
// it needs.  Offsets are in bytes from a base that the wave shares.
__device__ inline __amdgpu_buffer_rsrc_t rsrc_of(const void *base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, 0x7fffffff, 0x00027000);
}
template <class T>
__device__ inline T load_if(bool in, __amdgpu_buffer_rsrc_t from, uint32_t at) {
    const uint32_t off = in ? at : 0xfffffff0u;
    if constexpr (sizeof(T) == 16) return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b128(from, off, 0, 0));
    else if constexpr (sizeof(T) == 8) return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b64(from, off, 0, 0));
    else if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(from, off, 0, 0));
    else return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(from, off, 0, 0));
}
template <class T>
__device__ inline void store_if(bool in, __amdgpu_buffer_rsrc_t to, uint32_t at, T v) {
    const uint32_t off = in ? at : 0xfffffff0u;
    if constexpr (sizeof(T) == 16) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), to, off, 0, 0);
    else if constexpr (sizeof(T) == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), to, off, 0, 0);
    else if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), to, off, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), to, off, 0, 0);
}

// The 16 x 32 pieces of a lower triangular 64 x 64 operand that hold anything:
// piece (row block, k step) -> 0..5.
__device__ inline int tri(int rb, int ks) { return rb < 2 ? rb : rb * 2 - 2 + ks; }
constexpr int kTri = 6;
// The same of its transpose.
__device__ inline int tri_t(int rb, int ks) { return rb < 2 ? rb * 2 + ks : rb + 2; }

// What lanes of this wave wrote to LDS before is there for its other lanes after:
// the wave's LDS accesses run in order, so it is the compiler alone that must not move
// one past another's.
__device__ inline void wave_exchange() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---- the operands

// The chunk operands of the walks, in fragment order: the triangular inverse, P
// and the decays of a chunk and value head, and with the first of the value heads
// that share a key head its K, Q and K^T.  The forward walk multiplies by
// (I + A)^-1 with A_ij = e^(ci - cj) k_i . k_j beta_j and by P; the backward walk
// (BWD) by the transposes of P and of (I + A)^-1 with beta_i in beta_j's place,
// and by Q^T in place of Q.  A block takes a chunk slot and a value
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
// Forward, a token whose k, g or beta is not finite goes into the operands as one
// that writes nothing (k, g and beta 0), and is marked by a NaN in beta's place in
// dec: the walk makes NaN of what it reaches.
//
// A chain of small steps with barriers between them, so the LDS is kept small (four
// blocks a CU in bfloat16) and the blocks many; with enough of them bound by memory:
// 83 us for 16384 tokens of 16 value heads (4 key heads) of 128 bfloat16, which write
// 205 MB and read K and Q once a value head, 169 MB, 4.5 TB/s.
template <class T, int KS, bool VEC, bool BWD>
__global__ __launch_bounds__(256) void k_delta_operands(DeltaArgs a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3;
    constexpr int kKeys = 4 * KS * NP * kFrag;          // bf16 of one of kf, qf, kt
    extern __shared__ __align__(16) float lds[];
    float *x = lds, *y = x + kC * kLd;                  // A, then its inverse; P, over K's fragments
    uint16_t *skf = reinterpret_cast<uint16_t *>(y), *sqf = skf + kKeys;
    __shared__ double cs[kC];
    __shared__ float beta[kC];
    __shared__ uint32_t largest[kC];                    // magnitudes in k's rows
    const int slot = blockIdx.x, h = blockIdx.y, group = a.hv / a.hk, hk = h / group;
    const Chunk c = chunk_of(a, slot);
    const bool none = c.whole <= a.short_len;           // no chunk, or one of a sequence taken token by token
    if (BWD && h == 0 && threadIdx.x == 0) {
        int32_t *m = a.map + 4 * slot;
        m[0] = c.begin, m[1] = none ? 0 : c.len, m[2] = c.seq, m[3] = c.last;
    }
    if (none || c.len == 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int blocks = (c.len + 15) / 16;               // 16s of tokens
    const bool first = h % group == 0, busy = wave < blocks;
    const int64_t keys = ((int64_t)slot * a.hk + hk) * kKeys, ch = (int64_t)slot * a.hv + h;
    // K and Q as rows: the wave's 16 tokens.
    const int token = wave * 16 + r;
    bf16x8 ka[KS][NP], qa[KS][NP];
    uint32_t most = 0;
    const auto row = [&](const void *p, int64_t stride, int ks, bf16x8 (&f)[NP], bool key) {
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
        if (!BWD && key)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, magnitude(v[e]));
        uint32_t w[4][NP];
#pragma unroll
        for (int e = 0; e < 4; ++e) split_pair<NP>(v[2 * e], v[2 * e + 1], w[e]);
#pragma unroll
        for (int i = 0; i < NP; ++i) f[i] = __builtin_bit_cast(bf16x8, u32x4{w[0][i], w[1][i], w[2][i], w[3][i]});
    };
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        row(a.k, a.ks, ks, ka[ks], true);
        row(a.q, a.qs, ks, qa[ks], false);
    }
    if constexpr (!BWD) {
        most = max(most, __shfl_xor(most, 16));         // the row's four lanes
        most = max(most, __shfl_xor(most, 32));
        if (g == 0) largest[token] = most;
        if (most >= kHuge)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int i = 0; i < NP; ++i) ka[ks][i] = bf16x8{};
    }
    float marked = 0.f;                                 // wave 0, by tokens: beta, or NaN
    if (wave == 0) {
        bool bad = false;
        const double s = decay_sums(a, c, h, BWD ? nullptr : &bad), last = __shfl(s, 63);
        const float b = lane < c.len ? a.beta[(int64_t)(c.begin + lane) * a.hv + h] : 0.f;
        bad = bad || (!BWD && magnitude(b) >= kHuge);
        cs[lane] = s;
        beta[lane] = bad ? 0.f : b;
        a.dec[ch * 3 * kC + lane] = decay(s);
        a.dec[ch * 3 * kC + kC + lane] = decay(last - s);
        marked = bad ? kNaN : b;
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = ((wave * KS + ks) * NP + i) * kFrag + lane * 8;
            *reinterpret_cast<bf16x8 *>(skf + at) = ka[ks][i];
            if constexpr (BWD) *reinterpret_cast<bf16x8 *>(sqf + at) = qa[ks][i];
            if (first && busy) {
                *reinterpret_cast<bf16x8 *>(a.kf + keys + at) = ka[ks][i];
                if constexpr (!BWD) *reinterpret_cast<bf16x8 *>(a.qf + keys + at) = qa[ks][i];
            }
        }
    __syncthreads();
    if (wave == 0) a.dec[ch * 3 * kC + 2 * kC + lane] = !BWD && largest[lane] >= kHuge ? kNaN : marked;
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
    // K^T (and Q^T) as rows: element (d, token) from K's fragments.
    const auto transpose = [&](const uint16_t *from, uint16_t *to) {
        for (int i = wave; i < 2 * KS * 2; i += 4) {
            const int rt = i / 2, ks = i % 2, d = rt * 16 + r;
            if (ks * 32 >= c.len) continue;
            const int at = ((d / 32) * NP) * kFrag + (d % 32 / 8) * 16 * 8 + d % 8;      // of row block 0, token 0
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
                u16x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = ks * 32 + g * 8 + e;
                    v[e] = from[at + (t / 16) * KS * NP * kFrag + p * kFrag + (t % 16) * 8];
                }
                *reinterpret_cast<u16x8 *>(to + keys + (i * NP + p) * kFrag + lane * 8) = v;
            }
        }
    };
    if (first) transpose(skf, a.kt);
    if constexpr (BWD)
        if (first) transpose(sqf, a.qt);
    __syncthreads();                                    // K's fragments have been read
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int col = n * 16 + r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = wave * 16 + g * 4 + j;
            const float d = busy && n <= wave && col <= t ? decay(cs[t] - cs[col]) : 0.f;
            y[t * kLd + col] = col <= t ? d * w[n][j] * a.scale : 0.f;
            x[t * kLd + col] = col < t ? beta[BWD ? t : col] * d * u[n][j] : 0.f;
        }
    }
    __syncthreads();
    // A triangular matrix's pieces into fragments, a lane's eight columns of a row
    // (BWD: of the transpose).
    const auto pieces = [&](const float *m, uint16_t *to, int start, int stride) {
        for (int i = start; i < kTri; i += stride) {
            const int rb = BWD ? (i < 4 ? i / 2 : i - 2) : i < 2 ? i : i / 2 + 1, ks = BWD ? (i < 4 ? i & 1 : 1) : i < 2 ? 0 : i & 1;
            if (rb >= blocks || ks * 32 >= c.len) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = BWD ? m[(ks * 32 + g * 8 + e) * kLd + rb * 16 + r] : m[(rb * 16 + r) * kLd + ks * 32 + g * 8 + e];
            uint32_t q[4][3];
#pragma unroll
            for (int e = 0; e < 4; ++e) split_pair<3>(v[2 * e], v[2 * e + 1], q[e]);
#pragma unroll
            for (int o = 0; o < 3; ++o)
                *reinterpret_cast<u32x4 *>(to + (ch * kTri + i) * 3 * kFrag + o * kFrag + lane * 8) =
                    u32x4{q[0][o], q[1][o], q[2][o], q[3][o]};
        }
    };
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
        pieces(y, a.pf, wave - 1, 3);                   // P meanwhile
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
            wave_exchange();
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
    pieces(x, a.mf, wave, 4);
}

// Column tiles of a walk's block.  Two share the left operands' loads and one
// chain of barriers; one has the shorter chain, and more blocks, which is what counts
// until two-tile blocks (pairs) reach every CU.  Ragged sequences end at different
// times and leave room for more blocks.  Whole forward calls, us, one tile / two:
//   16384 bfloat16 tokens, 16 heads of 128 x 128: even, 128 pairs 386 / 501, 256
//     307 / 294, 512 295 / 246; ragged, 320 358 / 451, 512 317 / 360, 640 317 / 325,
//     768 312 / 299, 1024 310 / 294;
//   8192 float32 tokens, 8 heads of 128 x 128: even, 128 151 / 197, 256 156 / 135;
//     ragged, 384 172 / 182, 512 173 / 181, 768 186 / 156;
//   16384 float32 tokens, 4 heads of 64 x 64: even, 128 85 / 98, 256 85 / 87, 1024
//     91 / 86; ragged, 512 102 / 121, 768 104 / 112, 1024 105 / 108, 2048 139 / 130.
inline int walk_tiles(const DeltaArgs &a) {
    const int64_t pairs = (int64_t)a.n * a.hv * ((a.dv + 31) / 32);
    return a.dv <= 16 || pairs <= (a.off ? 512 : 255) ? 1 : 2;
}

template <class T, int KS, bool BWD>
hipError_t launch_operands(const DeltaArgs &a, hipStream_t s) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3;
    constexpr size_t tile = sizeof(float) * kC * kLd, frags = (BWD ? 2 : 1) * 2 * 4 * KS * NP * kFrag;
    constexpr size_t bytes = tile + (frags > tile ? frags : tile);
    const auto even = [&](const void *p, int64_t stride) {
        return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * sizeof(T) % 16 == 0;
    };
    const bool vec = a.dk % 8 == 0 && even(a.q, a.qs) && even(a.k, a.ks);
    auto *kernel = vec ? k_delta_operands<T, KS, true, BWD> : k_delta_operands<T, KS, false, BWD>;
    if (hipError_t e = allow_lds(kernel, bytes)) return e;
    kernel<<<dim3((int)delta_slots(a.tokens, a.n, !a.off), a.hv), 256, bytes, s>>>(a);
    return hipGetLastError();
}

}  // namespace ops
}  // namespace rn
