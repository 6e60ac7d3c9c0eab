// Device code that the gated delta rule's kernels share.
#pragma once

#include "rn_ops.hpp"
#include "rn_split.hpp"

namespace rn {
namespace ops {

constexpr int kC = RN_DELTA_CHUNK;   // tokens of a chunk
constexpr int kVT = 16;              // value columns of a block of the walks over chunks

typedef float f32x4 __attribute__((ext_vector_type(4)));

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
__device__ inline int slot_of(const Span &s, int i, int chunk) { return s.begin / kC + i + chunk; }

// The sequence and chunk of a chunk slot: the last sequence whose first slot is
// not beyond it.  Slots that no chunk has give len 0.
struct Chunk {
    int seq, begin, len;          // tokens begin .. begin + len - 1, len <= 64
};
__device__ inline Chunk chunk_of(const DeltaArgs &a, int slot) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (offset_of(a, mid) / kC + mid <= slot) lo = mid;
        else hi = mid - 1;
    }
    const Span s = span_of(a, lo);
    const int64_t at = (int64_t)(slot - slot_of(s, lo, 0)) * kC;
    if (at < 0 || at >= s.len) return {lo, 0, 0};
    return {lo, s.begin + (int)at, min(kC, s.len - (int)at)};
}

// Log decays summed up to each token of a chunk, in double: differences of far
// tokens stay exact to float32 where the sums are large.  An empty memory
// (g = -infinity) is a decay of e^-10^6 = 0, whose differences are finite.
// Tokens past the end count as g = 0.  One wave calls it; lane = token.
__device__ inline double decay_sums(const DeltaArgs &a, const Chunk &c, int head) {
    const int lane = threadIdx.x & 63;
    float g = lane < c.len ? a.g[(int64_t)(c.begin + lane) * a.hv + head] : 0.f;
    double s = g < -1e6f ? -1e6 : (double)g;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double t = __shfl_up(s, d);
        if (lane >= d) s += t;
    }
    return s;
}

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

// The same into three sums, by the terms' size: a matrix op waits for the one
// before it on the same sum, so a wave that has few tiles needs more sums.
struct Acc3 {
    f32x4 v[3] = {};
    __device__ f32x4 sum() const { return v[0] + (v[1] + v[2]); }
};
template <int NA, int NB>
__device__ inline void mm(const bf16x8 (&a)[NA], const bf16x8 (&b)[NB], Acc3 &acc) {
    constexpr int N = NA > NB ? NA : NB;
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int s = 0; s < N; ++s)
            if (s - i >= 0 && s - i < NB)
                acc.v[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[s - i], acc.v[s], 0, 0, 0);
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
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
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

// A store that is dropped where `in` is false, without a branch: the compiler
// can then count what is in flight and wait for no more than it needs.  Offsets
// are in bytes from a base that the wave shares.
__device__ inline __amdgpu_buffer_rsrc_t rsrc_of(void *base) {
    return __builtin_amdgcn_make_buffer_rsrc(base, 0, 0x7fffffff, 0x00027000);
}
template <class T>
__device__ inline void store_if(bool in, __amdgpu_buffer_rsrc_t to, uint32_t at, T v) {
    const uint32_t off = in ? at : 0xfffffff0u;
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), to, off, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), to, off, 0, 0);
}

// The 16 x 32 pieces of a lower triangular 64 x 64 operand that hold anything:
// piece (row block, k step) -> 0..5.
__device__ inline int tri(int rb, int ks) { return rb < 2 ? rb : rb * 2 - 2 + ks; }
constexpr int kTri = 6;

}  // namespace ops
}  // namespace rn
