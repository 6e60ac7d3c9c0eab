// Device code that the selective scan's kernels share.
//
// A lane carries a channel, 64 of one group a wave: nothing passes between lanes but
// the gradients of b and c, and a token's b and c, the same for all lanes, are
// scalars, which the loads' own unit brings.  A group of fewer than 64 channels leaves
// the wave's other lanes without work.
#pragma once

#include "rn_seq.hpp"

namespace rn {
namespace ops {

constexpr int kScanThreads = 256, kStates = 4, kTile = RN_SCAN_KEEP;
constexpr int kBatch = 8;         // tokens whose loads are on their way at once
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
        const bool up = at <= hi && (int64_t)(s.offset(min(at, hi)) >> a.log_chunk) + at <= slot;
        lo += __popcll(__ballot(up)) * step;
        hi = min(hi, lo + step - 1);
    }
    const int begin = s.offset(lo), len = max(0, s.offset(lo + 1) - begin);
    const int64_t c = slot - ((begin >> a.log_chunk) + lo), at = c << a.log_chunk;
    if (c < 0 || (at >= len && c > 0)) return {-1, 0, 0, false, false, 0};
    return {lo, begin + (int)at, (int)min(a.chunk(), len - at), c == 0, at + a.chunk() >= len,
            scan_end_slot(a, begin) + c};
}

// The kept state of the chunk's first tile; the next tiles' follow.
__device__ inline int64_t scan_kept_slot(const ScanArgs &a, const Seqs &s, const ScanChunk &chunk) {
    const int begin = s.offset(chunk.seq);
    return begin / kTile + chunk.seq + (chunk.begin - begin) / kTile;
}

// A wave's channels: 64 of a group, of which lane `me` has c, or goes along with the
// group's last where there is none.
struct ScanChannels {
    int group, c;
    bool live;
    __device__ ScanChannels(const ScanArgs &a, int block, int me) {
        const int of = a.channels / a.groups, per = (of + 63) / 64;
        group = block / per;
        const int at = group * of + block % per * 64 + me, last = (group + 1) * of - 1;
        live = at <= last;
        c = live ? at : last;
    }
};

template <int CTRL, int BANKS = 0xf>
__device__ inline float dpp(float v, float old = 0.f) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, v),
                                                                 CTRL, 0xf, BANKS, BANKS == 0xf));
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
// a log2(e) of a channel's states.  Finite where a is not NaN: exp(s a) is then 1 where s is 0, as
// of the tokens past a sequence's end, and an infinite a is the largest of its sign.  In two
// steps, for the second waits for a: behind the first tokens' loads (gradients of 256 episodes of
// 16 tokens 34.4 us, otherwise 35.1).
__device__ inline f32x4 load_decay(const ScanArgs &a, int c, int n0) {
    return load_states(a, a.a, 0, c, n0, true) * kLog2e;
}
__device__ inline float finite_decay(float v) {
    constexpr float kMost = 3.4028234663852886e38f;
    return v < -kMost ? -kMost : v > kMost ? kMost : v;
}
__device__ inline f32x4 finite_decay(f32x4 v) {
    return f32x4{finite_decay(v[0]), finite_decay(v[1]), finite_decay(v[2]), finite_decay(v[3])};
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
// Without a branch, p NULL or not.
__device__ inline void store_own_if(bool in, const ScanArgs &a, float *p, int64_t row, int c, int quad, f32x4 v) {
    const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(own_states(a, p, row, 0, 0), 0, 0x7fffffff, 0x00027000);
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const bool there = in && p && quad * kStates < a.states;
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rows, there ? (uint32_t)(quad * a.channels + c) * 16 : 0xfffffff0u, 0, 0);
}

// b and c in float32, as k_scan_pack leaves them: a token's and group's quads of
// states, four of b and then four of c each, the last of them 0.
struct Packed {
    float v;
};

// S of a token's b or c.  The address is one for the wave and on four bytes.
template <class BC, int S>
struct Scalars {
    uint32_t raw[sizeof(BC) == 2 ? S / 2 : S];
    __device__ void load(const BC *p) {
        typedef const __attribute__((address_space(4))) uint32_t *Constant;
        const Constant q = (Constant)(uintptr_t)p;
        if constexpr (std::is_same<BC, Packed>::value) {
#pragma unroll
            for (int i = 0; i < S; ++i) raw[i] = q[i / kStates * 2 * kStates + i % kStates];
        } else {
#pragma unroll
            for (int i = 0; i < (int)(S * sizeof(BC) / 4); ++i) raw[i] = q[i];
        }
    }
    __device__ float operator[](int i) const {
        if constexpr (sizeof(BC) == 4) return __uint_as_float(raw[i]);
        else return __uint_as_float(i % 2 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
    }
};

// An array's rows from one on: a lane's element of them.
template <class T>
__device__ inline __amdgpu_buffer_rsrc_t rows_from(const void *p, int64_t stride, int64_t row) {
    const char *base = static_cast<const char *>(p) + row * stride * (int)sizeof(T);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, 0x7fffffff, 0x00027000);
}
// Stores go without branches (what goes to kNowhere is past every array's end, and dropped), so
// that the number of them in flight is known, and a wait for loads not one for stores.
constexpr uint32_t kNowhere = 0xfffffff0u;
// The bits as loaded; as a float only where they are used, or each load would be waited for.
template <class T>
__device__ inline uint32_t row_load(__amdgpu_buffer_rsrc_t rows, uint32_t lane, int at) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_raw_buffer_load_b16(rows, lane, at, 0);
    else return __builtin_amdgcn_raw_buffer_load_b32(rows, lane, at, 0);
}
template <class T>
__device__ inline float row_float(uint32_t bits) {
    return __uint_as_float(sizeof(T) == 2 ? bits << 16 : bits);
}
template <class T>
__device__ inline void row_store(__amdgpu_buffer_rsrc_t rows, uint32_t lane, int at, T v) {
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), rows, lane, at, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), rows, lane, at, 0);
}

// Where a group's b or c (kind 1) of token t is: the caller's own, or as packed.
template <class BC>
struct TokenRows {
    const BC *at;
    int64_t stride;
    __device__ TokenRows(const ScanArgs &a, int kind, int group, int64_t t) {
        if constexpr (std::is_same<BC, Packed>::value) {
            at = reinterpret_cast<const Packed *>(a.packed) + kind * kStates;
            stride = (int64_t)a.groups * 2 * a.padded;
            at += t * stride + group * 2 * a.padded;
        } else {
            at = static_cast<const BC *>(kind ? a.c : a.b);
            stride = kind ? a.cs : a.bs;
            at += t * stride + group * a.states;
        }
    }
};

// f(states of a channel, rounded up to 4, 8, 16, 32 or 64).
template <class F>
inline void for_states(int states, F &&f) {
    using std::integral_constant;
    if (states <= 4) f(integral_constant<int, 4>{});
    else if (states <= 8) f(integral_constant<int, 8>{});
    else if (states <= 16) f(integral_constant<int, 16>{});
    else if (states <= 32) f(integral_constant<int, 32>{});
    else f(integral_constant<int, 64>{});
}

}  // namespace ops
}  // namespace rn
