// Device code that the gated delta rule's kernels share.
#pragma once

#include "rn_ops.hpp"

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

}  // namespace ops
}  // namespace rn
