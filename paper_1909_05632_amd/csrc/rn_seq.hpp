// Packed sequences as the kernels of the short convolution and the scan see them.
#pragma once

#include "rn_ops.hpp"

namespace rn {
namespace ops {

// Sequence i owns tokens offset(i) .. offset(i + 1) - 1.
struct Seqs {
    const int32_t *off;           // [n+1], or NULL: even lengths
    int n;
    int64_t tokens;
    int even;                     // tokens / n
    // Within the arrays whatever the offsets say.
    __device__ int offset(int i) const {
        const int64_t t = off ? off[i] : (int64_t)even * i;
        return (int)(t < 0 ? 0 : t < tokens ? t : tokens);
    }
    // The sequence that owns token t: the last that does not begin behind it.
    __device__ int of(int t) const {
        if (!off) return t / even;
        int lo = 0, hi = n - 1;
        while (lo < hi) {
            const int mid = lo + (hi - lo + 1) / 2;
            if (off[mid] <= t) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    }
};

// A sequence and its ends, around token t: begin <= t < end also where the offsets
// are not in order.
struct At {
    int seq, begin, end;
    __device__ At(const Seqs &s, int t) { set(s, s.of(t), t); }
    __device__ void set(const Seqs &s, int i, int t) {
        seq = i;
        begin = min(s.offset(i), t);
        end = max(s.offset(i + 1), t + 1);
    }
    // On to token t, the first behind this sequence: past empty ones.
    __device__ void next(const Seqs &s, int t) {
        int i = min(seq + 1, s.n - 1);
        while (i + 1 < s.n && s.offset(i + 1) <= t) ++i;
        set(s, i, t);
    }
};

// x / (1 + e^-x) by the hardware's exponential and reciprocal (an ulp each); its
// slope.  Where e^-x overflows both are what the limit is, 0.
__device__ inline float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * x));
}
__device__ inline float silu(float x) { return x * sigmoid(x); }
__device__ inline float silu_slope(float x) {
    const float g = sigmoid(x);
    return g * fmaf(x, 1.f - g, 1.f);
}

// VEC consecutive elements as float32, and back.
template <class T, int VEC>
__device__ inline void load_as(const T *p, float (&v)[VEC]) {
    const Pack<T, VEC> q = *reinterpret_cast<const Pack<T, VEC> *>(p);
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[j] = to_float(q.v[j]);
}
template <class T, int VEC>
__device__ inline void store_as(T *p, const float (&v)[VEC]) {
    Pack<T, VEC> q;
#pragma unroll
    for (int j = 0; j < VEC; ++j) q.v[j] = from_float<T>(v[j]);
    *reinterpret_cast<Pack<T, VEC> *>(p) = q;
}

}  // namespace ops
}  // namespace rn
