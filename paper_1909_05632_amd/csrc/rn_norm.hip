// Layer norm, forward and backward.
//
//   mean = sum x / W, var = sum (x - mean)^2 / W, rstd = 1 / sqrt(var + eps),
//   y = (x - mean) rstd w + b;  with t = dy w and xh = (x - mean) rstd:
//   dx = rstd (t - sum(t) / W - xh sum(t xh) / W), dw = sum_rows dy xh, db = sum_rows dy.
//
// A few operations per element: bound by HBM.  A row stays in the registers of
// the G lanes that own it, so x (and dy) are read once and the variance is the
// sum of squared distances from the mean that is already known, with none of
// the cancellation of sum x^2 - mean^2.  16384 rows of 4096 bfloat16: forward 62 us
// (4.3 TB/s, a large copy reaches 4.8), backward 83, the columns' sums 7; one row of
// 512 float32: 2.7 us, latency.
#include "rn_ops.hpp"

namespace rn {
namespace {

using namespace ops;

// t - s1 is 0 where it should be (a row of one element, equal ones): contracted,
// the product in t would enter the difference with more bits than it has in s1.
#pragma clang fp contract(off)

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

// G lanes take a row, each ITEMS vectors of VEC elements (vector lane + G i), so
// G ITEMS VEC >= width.  A block walks rows with a stride of the grid.
template <class T, int VEC, int G, int ITEMS>
__global__ __launch_bounds__(kThreads) void k_norm(NormArgs a) {
    __shared__ float lds[4];
    constexpr int RPB = kThreads / G;
    const int lane = threadIdx.x % G, sub = threadIdx.x / G;
    const int nv = a.width / VEC;
    const float inv = 1.0f / (float)a.width;
    // Every lane takes part in its row's sums: rows past the end are walked as
    // empty ones, so the loop's trips are equal within a block.
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t r = r0 + sub;
        const bool live = r < a.rows;
        const T *x = static_cast<const T *>(a.x) + r * a.xs;
        Pack<T, VEC> p[ITEMS];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (live && lane + G * i < nv) p[i] = *reinterpret_cast<const Pack<T, VEC> *>(x + (lane + G * i) * VEC);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (live && lane + G * i < nv)
#pragma unroll
                for (int j = 0; j < VEC; ++j) s += to_float(p[i].v[j]);
        const float mean = row_sum<G>(s, lds) * inv;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (live && lane + G * i < nv)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float d = to_float(p[i].v[j]) - mean;
                    q = fmaf(d, d, q);
                }
        const float rstd = 1.0f / sqrtf(row_sum<G>(q, lds) * inv + a.eps);
        if (!live) continue;
        T *y = static_cast<T *>(a.y) + r * a.ys;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (lane + G * i) * VEC;
            if (lane + G * i >= nv) continue;
            float w[VEC], b[VEC];
            load_f32<VEC>(a.weight ? a.weight + c : nullptr, w, 1.f);
            load_f32<VEC>(a.bias ? a.bias + c : nullptr, b, 0.f);
            Pack<T, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) o.v[j] = from_float<T>(fmaf((to_float(p[i].v[j]) - mean) * rstd, w[j], b[j]));
            *reinterpret_cast<Pack<T, VEC> *>(y + c) = o;
        }
        if (a.stats && lane == 0) {
            a.stats[2 * r] = mean;
            a.stats[2 * r + 1] = rstd;
        }
    }
}

// Rows too wide for the registers: one block a row, read three times (the
// second and third time from the caches).
template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_wide(NormArgs a) {
    __shared__ float lds[4];
    const float inv = 1.0f / (float)a.width;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + r * a.xs;
        float s = 0.f;
        for (int c = threadIdx.x; c < a.width; c += kThreads) s += to_float(x[c]);
        const float mean = row_sum<kThreads>(s, lds) * inv;
        float q = 0.f;
        for (int c = threadIdx.x; c < a.width; c += kThreads) {
            const float d = to_float(x[c]) - mean;
            q = fmaf(d, d, q);
        }
        const float rstd = 1.0f / sqrtf(row_sum<kThreads>(q, lds) * inv + a.eps);
        T *y = static_cast<T *>(a.y) + r * a.ys;
        for (int c = threadIdx.x; c < a.width; c += kThreads)
            y[c] = from_float<T>(fmaf((to_float(x[c]) - mean) * rstd, a.weight ? a.weight[c] : 1.f,
                                      a.bias ? a.bias[c] : 0.f));
        if (a.stats && threadIdx.x == 0) {
            a.stats[2 * r] = mean;
            a.stats[2 * r + 1] = rstd;
        }
    }
}

// dx, and each block's part of dw and db: a lane keeps the same columns for
// every row its block walks, so their sums stay in its registers; the 256 / G
// row groups of a block are added in LDS at the end.  A row's loads are on their
// way during the row before it where the registers allow (16384 rows of 4096
// bfloat16: 83 us, 4.9 TB/s; 116 us without).
template <class T, int VEC, int G, int ITEMS>
__global__ __launch_bounds__(kThreads) void k_norm_bwd(NormArgs a) {
    __shared__ float lds[2][8];
    constexpr int RPB = kThreads / G;
    constexpr int N = ITEMS * VEC;
    constexpr bool AHEAD = N <= 32;
    const int lane = threadIdx.x % G, sub = threadIdx.x / G;
    const int nv = a.width / VEC;
    const float inv = 1.0f / (float)a.width;
    float w[N], dw[N], db[N];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        float t[VEC];
        load_f32<VEC>(a.weight && lane + G * i < nv ? a.weight + (lane + G * i) * VEC : nullptr, t, 1.f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) w[i * VEC + j] = t[j], dw[i * VEC + j] = 0.f, db[i * VEC + j] = 0.f;
    }
    // Loads are from places clamped into the arrays, without branches, so that
    // those of the next row can stay in flight; what lies outside is not used.
    Pack<T, VEC> px[ITEMS], py[ITEMS], nx[ITEMS], ny[ITEMS];
    float mean, rstd, next_mean, next_rstd;
    const auto fetch = [&](int64_t r0) {
        const int64_t r = r0 + sub < a.rows ? r0 + sub : a.rows - 1;
        const T *x = static_cast<const T *>(a.x) + r * a.xs, *dy = static_cast<const T *>(a.dy) + r * a.dys;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = (lane + G * i < nv ? lane + G * i : nv - 1) * VEC;
            nx[i] = *reinterpret_cast<const Pack<T, VEC> *>(x + at);
            ny[i] = *reinterpret_cast<const Pack<T, VEC> *>(dy + at);
        }
        next_mean = a.stats[2 * r], next_rstd = a.stats[2 * r + 1];
    };
    const int64_t stride = (int64_t)gridDim.x * RPB;
    if constexpr (AHEAD) fetch((int64_t)blockIdx.x * RPB);
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += stride) {
        const int64_t r = r0 + sub;
        const bool live = r < a.rows;
        if constexpr (!AHEAD) fetch(r0);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) px[i] = nx[i], py[i] = ny[i];
        mean = next_mean, rstd = next_rstd;
        if constexpr (AHEAD) fetch(r0 + stride);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (live && lane + G * i < nv)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float d = to_float(py[i].v[j]), xh = (to_float(px[i].v[j]) - mean) * rstd;
                    const float t = d * w[i * VEC + j];
                    s1 += t;
                    s2 = fmaf(t, xh, s2);
                    dw[i * VEC + j] = fmaf(d, xh, dw[i * VEC + j]);
                    db[i * VEC + j] += d;
                }
        row_sums<G>(s1, s2, lds, turn++);
        s1 *= inv, s2 *= inv;
        if (!live) continue;
        T *dx = static_cast<T *>(a.y) + r * a.ys;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (lane + G * i >= nv) continue;
            Pack<T, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float t = to_float(py[i].v[j]) * w[i * VEC + j], xh = (to_float(px[i].v[j]) - mean) * rstd;
                o.v[j] = from_float<T>(rstd * (t - s1 - xh * s2));
            }
            *reinterpret_cast<Pack<T, VEC> *>(dx + (lane + G * i) * VEC) = o;
        }
    }
    if (!a.part) return;
    float *part = a.part + (size_t)blockIdx.x * 2 * a.width;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (lane + G * i < nv)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    part[(lane + G * i) * VEC + j] = dw[i * VEC + j];
                    part[a.width + (lane + G * i) * VEC + j] = db[i * VEC + j];
                }
    } else {
        __shared__ float sum[kThreads * 2];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __syncthreads();
            sum[2 * threadIdx.x] = dw[i];
            sum[2 * threadIdx.x + 1] = db[i];
            __syncthreads();
            const int c = (lane + G * (i / VEC)) * VEC + i % VEC;
            if (sub == 0 && lane + G * (i / VEC) < nv) {
                float u = 0.f, v = 0.f;
                for (int k = 0; k < RPB; ++k) u += sum[2 * (k * G + lane)], v += sum[2 * (k * G + lane) + 1];
                part[c] = u;
                part[a.width + c] = v;
            }
        }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_bwd_wide(NormArgs a) {
    __shared__ float lds[4];
    const float inv = 1.0f / (float)a.width;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + r * a.xs, *dy = static_cast<const T *>(a.dy) + r * a.dys;
        const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1];
        float s1 = 0.f, s2 = 0.f;
        for (int c = threadIdx.x; c < a.width; c += kThreads) {
            const float t = to_float(dy[c]) * (a.weight ? a.weight[c] : 1.f);
            s1 += t;
            s2 = fmaf(t, (to_float(x[c]) - mean) * rstd, s2);
        }
        s1 = row_sum<kThreads>(s1, lds) * inv;
        s2 = row_sum<kThreads>(s2, lds) * inv;
        T *dx = static_cast<T *>(a.y) + r * a.ys;
        for (int c = threadIdx.x; c < a.width; c += kThreads) {
            const float t = to_float(dy[c]) * (a.weight ? a.weight[c] : 1.f);
            dx[c] = from_float<T>(rstd * (t - s1 - (to_float(x[c]) - mean) * rstd * s2));
        }
    }
}

// The wide rows' part of dw and db: a thread per column, a strip of rows per
// blockIdx.y.  It runs before dx is written, which may lie over x or dy.
template <class T>
__global__ __launch_bounds__(kThreads) void k_norm_cols(NormArgs a) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.width) return;
    float dw = 0.f, db = 0.f;
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float d = to_float(static_cast<const T *>(a.dy)[r * a.dys + c]);
        dw = fmaf(d, (to_float(static_cast<const T *>(a.x)[r * a.xs + c]) - a.stats[2 * r]) * a.stats[2 * r + 1], dw);
        db += d;
    }
    float *part = a.part + (size_t)blockIdx.y * 2 * a.width;
    part[c] = dw;
    part[a.width + c] = db;
}

// Sums the strips in a fixed order: 16 columns a block, 64 threads a column each
// adding every 64th strip, then a tree.
__global__ __launch_bounds__(1024) void k_norm_reduce(NormArgs a) {
    __shared__ float lds[64][17];
    const int col = threadIdx.x % 16, k = threadIdx.x / 16;
    const int64_t c = (int64_t)block_index() * 16 + col, columns = (int64_t)2 * a.width;
    float s = 0.f;
    if (c < columns)
        for (int b = k; b < a.blocks; b += 64) s += a.part[b * columns + c];
    lds[k][col] = s;
    __syncthreads();
    for (int m = 32; m; m >>= 1) {
        if (k < m) lds[k][col] += lds[k + m][col];
        __syncthreads();
    }
    if (k == 0 && c < columns) {
        float *out = c < a.width ? a.dweight : a.dbias;
        const int64_t i = c < a.width ? c : c - a.width;
        if (out) out[i] = a.accumulate ? out[i] + lds[0][col] : lds[0][col];
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

bool aligned(const void *p, int64_t stride, int size) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0;
}

// 16-byte accesses where every row of every array allows them.
template <class T>
bool vectors(const NormArgs &a, bool bwd) {
    constexpr int VEC = 16 / sizeof(T);
    return a.width % VEC == 0 && aligned(a.x, a.xs, sizeof(T)) && aligned(a.y, a.ys, sizeof(T)) &&
           aligned(a.weight, 0, 4) && (bwd ? aligned(a.dy, a.dys, sizeof(T)) : aligned(a.bias, 0, 4));
}

template <class T, int VEC>
bool forward(const NormArgs &a, hipStream_t s) {
    return for_shape<T, VEC>(a.width, [&](auto g, auto i) {
        constexpr int RPB = kThreads / decltype(g)::value;
        const int64_t blocks = (a.rows + RPB - 1) / RPB;
        k_norm<T, VEC, decltype(g)::value, decltype(i)::value>
            <<<(int)(blocks < 16384 ? blocks : 16384), kThreads, 0, s>>>(a);
    });
}

template <class T, int VEC>
bool backward(const NormArgs &a, hipStream_t s) {
    return for_shape<T, VEC>(a.width, [&](auto g, auto i) {
        k_norm_bwd<T, VEC, decltype(g)::value, decltype(i)::value><<<a.blocks, kThreads, 0, s>>>(a);
    });
}

template <class T>
hipError_t run_forward(const NormArgs &a, hipStream_t s) {
    if (!(vectors<T>(a, false) ? forward<T, 16 / sizeof(T)>(a, s) : forward<T, 1>(a, s)))
        k_norm_wide<T><<<(int)(a.rows < 16384 ? a.rows : 16384), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t run_backward(const NormArgs &a, hipStream_t s) {
    if (a.rows > 0 && !(vectors<T>(a, true) ? backward<T, 16 / sizeof(T)>(a, s) : backward<T, 1>(a, s))) {
        if (a.part) {
            k_norm_cols<T><<<dim3((a.width + kThreads - 1) / kThreads, a.blocks), kThreads, 0, s>>>(a);
            if (hipError_t e = hipGetLastError()) return e;
        }
        k_norm_bwd_wide<T><<<(int)(a.rows < 16384 ? a.rows : 16384), kThreads, 0, s>>>(a);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if (a.part) {
        k_norm_reduce<<<grid_of(((int64_t)2 * a.width + 15) / 16), 1024, 0, s>>>(a);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace

// Row strips of the backward call: up to 512 blocks, each with 8 rows or more.
int norm_blocks(int64_t rows, int) {
    const int64_t b = (rows + 7) / 8;
    return (int)(b < 1 ? 1 : b < 512 ? b : 512);
}

hipError_t launch_norm(const NormArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? run_forward<bf16_t>(a, s) : run_forward<float>(a, s);
}

hipError_t launch_norm_backward(const NormArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? run_backward<bf16_t>(a, s) : run_backward<float>(a, s);
}

}  // namespace rn
