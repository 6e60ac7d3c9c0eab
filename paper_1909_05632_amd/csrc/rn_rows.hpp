// Rows of a width in the registers of the lanes that own them: what the kernels of
// rows (rn_norm.hip, rn_rms.hip) share, and the sum of partial column sums over
// blocks in a fixed order.
#pragma once

#include <type_traits>

#include "rn_ops.hpp"

namespace rn {
namespace ops {

constexpr int kThreads = 256;

// Sum over the G lanes of a row: G <= 64 lies in one wave, G = 256 is the block.
template <int G>
__device__ inline float row_sum(float v, float *lds) {
#pragma unroll
    for (int m = (G < 64 ? G : 64) / 2; m; m >>= 1) v += __shfl_xor(v, m);
    if constexpr (G > 64) {
        __syncthreads();                       // the last use of lds is over
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    }
    return v;
}

// Two sums at once, with one barrier: rows take two parts of the LDS in turn.
template <int G>
__device__ inline void row_sums(float &u, float &v, float (&lds)[2][8], int turn) {
#pragma unroll
    for (int m = (G < 64 ? G : 64) / 2; m; m >>= 1) u += __shfl_xor(u, m), v += __shfl_xor(v, m);
    if constexpr (G > 64) {
        float *l = lds[turn & 1];
        if ((threadIdx.x & 63) == 0) l[threadIdx.x >> 6] = u, l[4 + (threadIdx.x >> 6)] = v;
        __syncthreads();
        u = (l[0] + l[1]) + (l[2] + l[3]), v = (l[4] + l[5]) + (l[6] + l[7]);
    }
}

template <int VEC>
__device__ inline void load_f32(const float *p, float (&v)[VEC], float none) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[j] = none;
    if (!p) return;
    if constexpr (VEC == 1) {
        v[0] = *p;
    } else {
#pragma unroll
        for (int j = 0; j < VEC; j += 4) {
            const Pack<float, 4> q = *reinterpret_cast<const Pack<float, 4> *>(p + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[j + i] = q.v[i];
        }
    }
}

// The lanes of a row and their registers by the row's vectors: small rows share
// a wave (no LDS, several rows in flight), larger ones take the block.
template <class T, int VEC, class F>
bool for_shape(int width, F &&f) {
    const int nv = width / VEC;
    auto go = [&](auto g, auto i) { f(g, i); return true; };
    using std::integral_constant;
    if (nv <= 8) return go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (nv <= 16) return go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (nv <= 32) return go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    if (nv <= 64) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (nv <= 128) return go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    if (nv <= 256) return go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    if (nv <= 512) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    if (nv <= 1024) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    if (nv <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 8>{});
    if constexpr (VEC == 1) {
        if (nv <= 4096) return go(integral_constant<int, 256>{}, integral_constant<int, 16>{});
        if (nv <= 8192) return go(integral_constant<int, 256>{}, integral_constant<int, 32>{});
    }
    return false;
}

inline bool aligned(const void *p, int64_t stride, int size) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0;
}

// out[c] (+)= the sum over b of part[b][c], in a fixed order: 16 columns a block, 64
// threads a column each adding every 64th part, then a tree.
template <class Out>
__device__ inline void column_sums(const float *part, int64_t columns, int parts, uint32_t block, Out &&out) {
    __shared__ float lds[64][17];
    const int col = threadIdx.x % 16, k = threadIdx.x / 16;
    const int64_t c = (int64_t)block * 16 + col;
    float s = 0.f;
    if (c < columns)
        for (int b = k; b < parts; b += 64) s += part[b * columns + c];
    lds[k][col] = s;
    __syncthreads();
    for (int m = 32; m; m >>= 1) {
        if (k < m) lds[k][col] += lds[k + m][col];
        __syncthreads();
    }
    if (k == 0 && c < columns) out(c, lds[0][col]);
}
inline int64_t column_blocks(int64_t columns) { return (columns + 15) / 16; }       // of 1024 threads
inline dim3 column_grid(int64_t columns) { return grid_of(column_blocks(columns)); }

}  // namespace ops
}  // namespace rn
