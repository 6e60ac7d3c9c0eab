// Internal declarations of the operators in include/reuse_ops.h: kernel
// launchers (rn_norm.hip, rn_sample.hip, rn_delta.hip, rn_delta_short.hip,
// rn_delta_bwd.hip) and device helpers they share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "reuse_ops.h"

namespace rn {

// ------------------------------------------------------------------ launchers

struct NormArgs {
    int64_t rows;
    int width;
    const void *x, *dy;           // dy: backward only
    void *y;                      // dx in the backward call
    int64_t xs, dys, ys;          // row strides in elements
    const float *weight, *bias;
    float eps;
    float *stats;                 // [rows][2]; read by the backward call
    float *part;                  // [blocks][2][width] partial weight and bias gradients, or NULL
    int blocks;                   // row strips of the backward call
    float *dweight, *dbias;
    int accumulate;
};
int norm_blocks(int64_t rows, int width);
hipError_t launch_norm(const NormArgs &a, bool bf16, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs &a, bool bf16, hipStream_t s);

struct SampleArgs {
    int n, vocab;
    const void *logits;
    int64_t stride;
    const float *u;
    rn_sample_params p;
    int32_t *tokens;
    float *logprobs;
};
hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t s);

struct DeltaArgs {
    int n, hk, hv, dk, dv;
    int64_t tokens;
    float scale;
    int64_t qs, ks, vs;
    const void *q, *k, *v;
    const float *g, *beta;
    const int32_t *off;           // [n+1], or NULL: even lengths
    const int32_t *ids;           // step: slots, or NULL
    int short_len;                // sequences up to this length go token by token (-1: none)
    int slots;
    const float *state;           // first states, or NULL
    float *final_state;           // last states, or NULL (step: the state pool)
    void *out;
    // Per chunk slot (delta_slots) and key head, in fragment order (rn_delta.hpp):
    uint16_t *kf, *qf;            // K and Q as rows (qf: forward only)
    uint16_t *kt, *qt;            // K^T and Q^T as rows (qt: backward only)
    // Per chunk slot and value head:
    uint16_t *mf, *pf;            // the triangular inverse and P, three planes each
    float *dec;                   // [3][64] e^c, e^(c64 - c), beta
    float *before;                // [delta_kept_slots][hv][dk][dv] states before each chunk, or NULL (not kept)
    float *err;                   // [tokens][hv][dv] v - S^T k as each token met it, or NULL
    // Backward call:
    const void *dout;
    const float *dfinal;
    int32_t *map;                 // [slots][4] each chunk slot's first token, length, sequence, whether its last
    float *after;                 // [slots][hv][dk][dv] gradients of the states after each chunk but a sequence's last
    float *dwrite;                // [tokens][hv][dv] gradients of what each token wrote, beta err
    void *dq, *dkey, *dval;
    float *dg, *dbeta, *dstate;
};
// 32-wide steps of dk in the chunk kernels (powers of two).
inline int delta_ksteps(int dk) { return dk <= 32 ? 1 : dk <= 64 ? 2 : 4; }
// bf16 planes of an input.
inline int delta_planes(bool bf16) { return bf16 ? 1 : 3; }
// Token by token a sequence takes about 0.3 us a token and no scratch; by chunks
// the operands and the walk cost as much as some 35 tokens whatever the chunk
// holds (measured at dk 64 and 128), so short sequences go token by token.
constexpr int kShort = 32;
// Which of the two ways a call has sequences for; lengths are on the device, so
// ragged calls of few tokens a sequence launch both, and each takes its own.
struct DeltaWays {
    bool tokens, chunks;
};
inline DeltaWays delta_ways(int64_t tokens, int n, bool even) {
    const bool t = tokens <= (int64_t)kShort * n;
    if (even || tokens == 0) return {t, !t};
    if (tokens <= kShort) return {true, false};
    return {t, true};
}
// Slots of what is kept for the backward call, whichever way a sequence goes: chunk
// c of sequence i has slot off[i] / 64 + i + c, so every slot is below
// tokens / 64 + n and no two chunks share one.
inline int64_t delta_kept_slots(int64_t tokens, int n) { return tokens / RN_DELTA_CHUNK + n; }
// Slots of the chunk kernels' operands: the same, unless sequences of up to kShort
// tokens go token by token, which have none.  The others' chunks then have slots
// off[i] / 32 + c: a sequence of 33 tokens or more moves off / 32 on by its chunks
// at least.  (They would otherwise take operands of 64 tokens for every sequence.)
inline int64_t delta_slots(int64_t tokens, int n, bool even) {
    const DeltaWays w = delta_ways(tokens, n, even);
    return !w.chunks ? 0 : w.tokens ? tokens / kShort : delta_kept_slots(tokens, n);
}
static_assert(2 * kShort == RN_DELTA_CHUNK);
hipError_t launch_delta_step(const DeltaArgs &a, bool bf16, hipStream_t s);
hipError_t launch_delta_short_forward(const DeltaArgs &a, bool bf16, hipStream_t s);
hipError_t launch_delta_short_backward(const DeltaArgs &a, bool bf16, hipStream_t s);
hipError_t launch_delta_forward(const DeltaArgs &a, bool bf16, hipStream_t s);
hipError_t launch_delta_backward(const DeltaArgs &a, bool bf16, hipStream_t s);

// A grid of up to 2^31 blocks: one axis holds no more than 2^32 threads, and a
// larger one is cut off without an error.  block_index() may run past the last.
inline dim3 grid_of(int64_t blocks) {
    constexpr int64_t kRow = 1 << 20;
    return blocks <= kRow ? dim3((unsigned)blocks) : dim3((unsigned)kRow, (unsigned)((blocks + kRow - 1) / kRow));
}

// Allows a kernel the dynamic LDS of its launch (more than the default 64 KiB).
template <class K>
inline hipError_t allow_lds(K *kernel, size_t bytes) {
    if (bytes <= 64 * 1024) return hipSuccess;
    return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                               (int)bytes);
}

// ------------------------------------------------------------------ device helpers

namespace ops {

__device__ inline uint32_t block_index() { return blockIdx.x + blockIdx.y * gridDim.x; }

// bf16 as raw 16 bits, so that loads and conversions are explicit.
struct bf16_t {
    uint16_t bits;
};
__device__ inline float to_float(float v) { return v; }
__device__ inline float to_float(bf16_t v) { return __uint_as_float((uint32_t)v.bits << 16); }
template <class T> __device__ inline T from_float(float v);
template <> __device__ inline float from_float<float>(float v) { return v; }
// Rounded to nearest even; NaN stays NaN.
template <> __device__ inline bf16_t from_float<bf16_t>(float v) {
    return __builtin_bit_cast(bf16_t, static_cast<__bf16>(v));
}

// VEC consecutive elements in one access; the caller has checked alignment.
template <class T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
    T v[VEC];
};

}  // namespace ops
}  // namespace rn
