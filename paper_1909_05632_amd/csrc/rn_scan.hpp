// Device code that the selective scan's kernels share.
//
// L lanes carry a channel's states, kStates each (states that are not there have
// a = b = c = 0), so a wave has 64 / L channels and a block 256 / L.  Tokens go by
// tiles of kTile.  What only a channel needs of a token, its step size and products
// with it, is computed once, by the thread that loads it (quads of channels), and
// read from LDS by the channel's lanes.
#pragma once

#include "rn_seq.hpp"

namespace rn {
namespace ops {

constexpr int kScanThreads = 256, kStates = 4, kTile = RN_SCAN_KEEP;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A chunk of a sequence by its slot: sequence i has slots offset(i) / chunk + i and
// on, one at least (an empty sequence's has len 0); slots in between have seq -1.
struct ScanChunk {
    int seq, begin, len;          // tokens begin .. begin + len - 1
    bool first, last;             // of its sequence
    int64_t end;                  // slot among the chunks' ends, if its sequence has several
    __device__ bool alone() const { return first && last; }
};
__device__ inline ScanChunk scan_chunk_of(const ScanArgs &a, const Seqs &s, int64_t slot) {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {                                   // 64 places at once; uniform within a wave
        const int step = (hi - lo + 63) / 64, at = lo + ((int)(threadIdx.x & 63) + 1) * step;
        const bool up = at <= hi && (int64_t)s.offset(min(at, hi)) / a.chunk + at <= slot;
        lo += __popcll(__ballot(up)) * step;
        hi = min(hi, lo + step - 1);
    }
    const int begin = s.offset(lo), len = max(0, s.offset(lo + 1) - begin);
    const int64_t c = slot - (begin / a.chunk + lo), at = c * a.chunk;
    if (c < 0 || (at >= len && c > 0)) return {-1, 0, 0, false, false, 0};
    return {lo, begin + (int)at, (int)min((int64_t)a.chunk, len - at), c == 0, at + a.chunk >= len,
            scan_end_slot(a, begin) + c};
}

// The kept state of the chunk's first tile; the next tiles' follow.
__device__ inline int64_t scan_kept_slot(const ScanArgs &a, const Seqs &s, const ScanChunk &chunk) {
    const int begin = s.offset(chunk.seq);
    return begin / kTile + chunk.seq + (chunk.begin - begin) / kTile;
}

// The block's channels c0 .. c0 + CB - 1, of which those below c1 are there; all of one group.
template <int L>
struct ScanBlock {
    static constexpr int CB = kScanThreads / L;
    int group, c0, c1;
    __device__ ScanBlock(const ScanArgs &a, int i) {
        const int of = a.channels / a.groups, per = (of + CB - 1) / CB;
        group = i / per;
        c0 = group * of + i % per * CB;
        c1 = (group + 1) * of;
    }
};

template <int CTRL>
__device__ inline float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Sum over a channel's L lanes: 1 and 2 apart, then the other four of eight, the
// other eight of sixteen (which hold one value by then, so mirrored will do).
template <int L>
__device__ inline float over_states(float v) {
    if constexpr (L >= 2) v += dpp<0xb1>(v);
    if constexpr (L >= 4) v += dpp<0x4e>(v);
    if constexpr (L >= 8) v += dpp<0x141>(v);
    if constexpr (L >= 16) v += dpp<0x140>(v);
    return v;
}

// log(1 + e^x): with e = e^-|x| and q = e / (2 + e) <= 1/3, log(1 + e) is
// 2 artanh(q) = q P(q^2), P of degree 4 by least squares weighted towards its largest
// error, 4.5e-9 of it.  Relative error |x| 2^-24 from the exponent's rounding (as much
// as x, itself a rounded sum, brings along) and a few 2^-24.
__device__ inline float softplus(float x) {
    const float e = __builtin_amdgcn_exp2f(-fabsf(x) * kLog2e);
    const float q = e * __builtin_amdgcn_rcpf(2.f + e), r = q * q;
    float p = fmaf(r, 0.2801215648651123f, 0.2800177335739136f);
    p = fmaf(r, p, 0.4002152979373932f);
    p = fmaf(r, p, 0.666664183139801f);
    p = fmaf(r, p, 2.f);
    return fmaf(q, p, fmaxf(x, 0.f));
}

// A lane's states of channel c, number n0 and on, of an array [...][channels][states].
__device__ inline f32x4 load_states(const ScanArgs &a, const float *p, int64_t row, int c, int n0, bool live) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (!live || !p) return v;
    p += (row * a.channels + c) * a.states + n0;
    if (a.whole_states) {
        if (n0 < a.states) v = *reinterpret_cast<const f32x4 *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < kStates; ++i)
            if (n0 + i < a.states) v[i] = p[i];
    }
    return v;
}
__device__ inline void store_states(const ScanArgs &a, float *p, int64_t row, int c, int n0, bool live, f32x4 v) {
    if (!live || !p) return;
    p += (row * a.channels + c) * a.states + n0;
    if (a.whole_states) {
        if (n0 < a.states) *reinterpret_cast<f32x4 *>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < kStates; ++i)
            if (n0 + i < a.states) p[i] = v[i];
    }
}

// The same of an array of the library's own, [...][states / 4, rounded up][channels][4].
__device__ inline f32x4 *own_states(const ScanArgs &a, float *p, int64_t row, int c, int quad) {
    return reinterpret_cast<f32x4 *>(p) + (row * ((a.states + kStates - 1) / kStates) + quad) * a.channels + c;
}
__device__ inline f32x4 load_own(const ScanArgs &a, float *p, int64_t row, int c, int quad, bool live) {
    if (!live || quad * kStates >= a.states) return f32x4{0.f, 0.f, 0.f, 0.f};
    return *own_states(a, p, row, c, quad);
}
__device__ inline void store_own(const ScanArgs &a, float *p, int64_t row, int c, int quad, bool live, f32x4 v) {
    if (live && quad * kStates < a.states) *own_states(a, p, row, c, quad) = v;
}

// Four channels of a token; those that are not there are not touched.
template <class T>
__device__ inline Pack<T, 4> load_quad(const ScanArgs &a, const void *p, int64_t stride, int64_t token, int c, int c1) {
    const T *x = static_cast<const T *>(p) + token * stride + c;
    if (a.quads) return *reinterpret_cast<const Pack<T, 4> *>(x);
    Pack<T, 4> v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v.v[j] = x[c + j < c1 ? j : 0];
    return v;
}
template <class T>
__device__ inline void store_quad(const ScanArgs &a, void *p, int64_t token, int c, int c1, const float (&v)[4]) {
    T *x = static_cast<T *>(p) + token * a.channels + c;
    if (a.quads) {
        store_as<T, 4>(x, v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < c1) x[j] = from_float<T>(v[j]);
    }
}

// b and c of a tile, [kTile][4 L] each: a thread's elements, in flight and then in LDS.
template <class T, int L>
struct TileBC {
    static constexpr int N = kStates * L, PER = (kTile * N + kScanThreads - 1) / kScanThreads;
    T b[PER], c[PER];
    __device__ void load(const ScanArgs &a, int group, int begin, int len) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = threadIdx.x + i * kScanThreads, t = e / N, n = e % N;
            if (e < kTile * N && t < len && n < a.states) {
                const int64_t at = begin + t;
                b[i] = static_cast<const T *>(a.b)[at * a.bs + group * a.states + n];
                c[i] = static_cast<const T *>(a.c)[at * a.cs + group * a.states + n];
            }
        }
    }
    __device__ void store(const ScanArgs &a, int len, float (&sb)[kTile][N], float (&sc)[kTile][N]) const {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = threadIdx.x + i * kScanThreads, t = e / N, n = e % N;
            if (e < kTile * N) {
                const bool in = t < len && n < a.states;
                sb[t][n] = in ? to_float(b[i]) : 0.f;
                sc[t][n] = in ? to_float(c[i]) : 0.f;
            }
        }
    }
};

// Quads of a tile: thread i has quad i % (CB / 4) of token i / (CB / 4), and on.
template <int L>
struct Quads {
    static constexpr int CB = kScanThreads / L, ACROSS = CB / 4, ROWS = kScanThreads / ACROSS;
    static constexpr int PER = kTile / ROWS > 1 ? kTile / ROWS : 1;
    static __device__ int channel() { return threadIdx.x % ACROSS * 4; }
    static __device__ int row(int i) { return threadIdx.x / ACROSS + i * ROWS; }
};

// The lanes of a channel by its states.
template <class F>
inline void for_lanes_of(int states, F &&f) {
    using std::integral_constant;
    if (states <= 4) f(integral_constant<int, 1>{});
    else if (states <= 8) f(integral_constant<int, 2>{});
    else if (states <= 16) f(integral_constant<int, 4>{});
    else if (states <= 32) f(integral_constant<int, 8>{});
    else f(integral_constant<int, 16>{});
}

}  // namespace ops
}  // namespace rn
