// Residual norm, forward and backward, with an output in 8 bits.
//
//   h = x + residual (rounded to the data type), rstd = 1 / sqrt(sum h^2 / W + eps),
//   y = h rstd w;  with t = dy w and n = h rstd:
//   dx = dh + rstd (t - n sum(t n) / W), dw = sum_rows dy n.
// In 8 bits (e4m3) a row's largest |h w| becomes 448: rstd cancels in q, which is
// then a function of h and w alone, and enters the row's scale.
//
// A few operations per element: bound by HBM.  A row stays in the registers of the
// G lanes that own it, so every input is read once.  16384 x 4096 bfloat16: forward 92 us
// (5.8 TB/s), backward 109 and 5 for the sum over blocks (4.9 TB/s); 1024 x 8192 to 8
// bits 17 us (3.4 TB/s: there is a tenth of the bytes to have on their way).
#include "rn_rows.hpp"

namespace rn {
namespace {

using namespace ops;

// h w has one rounding, as its definition says, whatever it is used in.
#pragma clang fp contract(off)

constexpr float kE4m3Max = 448.f;

// Largest of the G lanes of a row; lds must not be in use.
template <int G>
__device__ inline float row_max(float v, float *lds) {
#pragma unroll
    for (int m = (G < 64 ? G : 64) / 2; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    if constexpr (G > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
    }
    return v;
}

// What a row's |h w| are multiplied by, in two factors: 448 / largest, and a power of two
// where that would be infinite.
struct Steps {
    float up, step;
    __device__ explicit Steps(float largest) : up(largest < 0x1p-100f ? 0x1p60f : 1.f) {
        step = largest > 0.f ? kE4m3Max / (largest * up) : 0.f;
    }
};

// A row's scale.  NaN where the sum of its squares is infinite or NaN: finite values whose
// squares overflow have an rstd of 0, and a scale of 0 would be that of a row of zeros.
__device__ inline float scale_of(float squares, float largest, float rstd) {
    return squares < __builtin_huge_valf() ? largest * rstd / kE4m3Max : __builtin_nanf("");
}

// e4m3, to nearest even; two values' bits.
__device__ inline uint32_t e4m3_pair(float x, float y) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) & 0xffffu;
}

template <int VEC>
__device__ inline void store_e4m3(uint8_t *p, const float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        *p = (uint8_t)e4m3_pair(v[0], 0.f);
    } else {
        Pack<uint32_t, VEC / 4> o;
#pragma unroll
        for (int j = 0; j < VEC; j += 4) o.v[j / 4] = e4m3_pair(v[j], v[j + 1]) | e4m3_pair(v[j + 2], v[j + 3]) << 16;
        *reinterpret_cast<Pack<uint32_t, VEC / 4> *>(p) = o;
    }
}

// G lanes take a row, each ITEMS vectors of VEC elements (vector lane + G i), so
// G ITEMS VEC >= width.  A block walks rows with a stride of the grid.
template <class T, int VEC, int G, int ITEMS>
__global__ __launch_bounds__(kThreads) void k_rms(RmsArgs a) {
    __shared__ float lds[4], most[4];
    constexpr int RPB = kThreads / G;
    const int lane = threadIdx.x % G, sub = threadIdx.x / G;
    const int nv = a.width / VEC;
    const float inv = 1.0f / (float)a.width;
    // Rows past the end are walked as empty ones: the loop's trips are equal within a block.
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
        const int64_t r = r0 + sub;
        const bool live = r < a.rows;
        const T *x = static_cast<const T *>(a.x) + r * a.xs, *add = static_cast<const T *>(a.residual) + r * a.rs;
        Pack<T, VEC> p[ITEMS], o[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (live && lane + G * i < nv) {
                p[i] = *reinterpret_cast<const Pack<T, VEC> *>(x + (lane + G * i) * VEC);
                if (a.residual) o[i] = *reinterpret_cast<const Pack<T, VEC> *>(add + (lane + G * i) * VEC);
            }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (live && lane + G * i < nv)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    if (a.residual) p[i].v[j] = from_float<T>(to_float(p[i].v[j]) + to_float(o[i].v[j]));
                    s = fmaf(to_float(p[i].v[j]), to_float(p[i].v[j]), s);
                }
        if (a.total && live) {
            T *total = static_cast<T *>(a.total) + r * a.width;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (lane + G * i < nv) *reinterpret_cast<Pack<T, VEC> *>(total + (lane + G * i) * VEC) = p[i];
        }
        s = row_sum<G>(s, lds);
        const float rstd = 1.0f / sqrtf(s * inv + a.eps);
        float largest = 0.f;
        if (a.q) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
                if (live && lane + G * i < nv) {
                    float w[VEC];
                    load_f32<VEC>(a.weight ? a.weight + (lane + G * i) * VEC : nullptr, w, 1.f);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) largest = fmaxf(largest, fabsf(to_float(p[i].v[j]) * w[j]));
                }
            largest = row_max<G>(largest, most);
        }
        if (!live) continue;
        const Steps to_q(largest);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (lane + G * i) * VEC;
            if (lane + G * i >= nv) continue;
            float w[VEC];
            load_f32<VEC>(a.weight ? a.weight + c : nullptr, w, 1.f);
            if (a.y) {
                Pack<T, VEC> y;
#pragma unroll
                for (int j = 0; j < VEC; ++j) y.v[j] = from_float<T>(to_float(p[i].v[j]) * rstd * w[j]);
                *reinterpret_cast<Pack<T, VEC> *>(static_cast<T *>(a.y) + r * a.width + c) = y;
            }
            if (a.q) {
                float t[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) t[j] = to_float(p[i].v[j]) * w[j] * to_q.up * to_q.step;
                store_e4m3<VEC>(a.q + r * a.width + c, t);
            }
        }
        if (lane == 0) {
            if (a.rstd) a.rstd[r] = rstd;
            if (a.q) a.scales[r] = scale_of(s, largest, rstd);
        }
    }
}

// Rows too wide for the registers: one block a row, read two or three times (the
// later times from the caches).  y and total may lie over x and the residual:
// each element is read by the thread that writes it, before it does.
template <class T>
__global__ __launch_bounds__(kThreads) void k_rms_wide(RmsArgs a) {
    __shared__ float lds[4], most[4];
    const float inv = 1.0f / (float)a.width;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + r * a.xs, *add = static_cast<const T *>(a.residual) + r * a.rs;
        T *total = a.total ? static_cast<T *>(a.total) + r * a.width : nullptr;
        float s = 0.f, largest = 0.f;
        for (int c = threadIdx.x; c < a.width; c += kThreads) {
            const T h = a.residual ? from_float<T>(to_float(x[c]) + to_float(add[c])) : x[c];
            if (total) total[c] = h;
            s = fmaf(to_float(h), to_float(h), s);
            if (a.q) largest = fmaxf(largest, fabsf(to_float(h) * (a.weight ? a.weight[c] : 1.f)));
        }
        s = row_sum<kThreads>(s, lds);
        const float rstd = 1.0f / sqrtf(s * inv + a.eps);
        if (a.q) largest = row_max<kThreads>(largest, most);
        const Steps to_q(largest);
        for (int c = threadIdx.x; c < a.width; c += kThreads) {
            const float h = to_float(total ? total[c] : a.residual ? from_float<T>(to_float(x[c]) + to_float(add[c])) : x[c]);
            const float w = a.weight ? a.weight[c] : 1.f;
            if (a.y) static_cast<T *>(a.y)[r * a.width + c] = from_float<T>(h * rstd * w);
            if (a.q) a.q[r * a.width + c] = (uint8_t)e4m3_pair(h * w * to_q.up * to_q.step, 0.f);
        }
        if (threadIdx.x == 0) {
            if (a.rstd) a.rstd[r] = rstd;
            if (a.q) a.scales[r] = scale_of(s, largest, rstd);
        }
    }
}

// dx, and each block's part of dw: a lane keeps the same columns for every row its
// block walks, so their sums stay in its registers; the 256 / G row groups of a
// block are added in LDS at the end.  A row's loads are on their way during the row
// before it, where the registers allow.
template <class T, int VEC, int G, int ITEMS>
__global__ __launch_bounds__(kThreads) void k_rms_bwd(RmsArgs a) {
    __shared__ float lds[2][8];
    constexpr int RPB = kThreads / G;
    constexpr int N = ITEMS * VEC;
    constexpr bool AHEAD = N <= 32;
    const int lane = threadIdx.x % G, sub = threadIdx.x / G;
    const int nv = a.width / VEC;
    const float inv = 1.0f / (float)a.width;
    float w[N], dw[N];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        float t[VEC];
        load_f32<VEC>(a.weight && lane + G * i < nv ? a.weight + (lane + G * i) * VEC : nullptr, t, 1.f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) w[i * VEC + j] = t[j], dw[i * VEC + j] = 0.f;
    }
    // Loads are from places clamped into the arrays, without branches, so that
    // those of the next row can stay in flight; what lies outside is not used.
    Pack<T, VEC> px[ITEMS], py[ITEMS], pt[ITEMS], nx[ITEMS], ny[ITEMS], nt[ITEMS];
    float rstd, next_rstd;
    const T *dtotal = static_cast<const T *>(a.dtotal ? a.dtotal : a.dy);
    const int64_t dts = a.dtotal ? a.dts : a.dys;
    const auto fetch = [&](int64_t r0) {
        const int64_t r = r0 + sub < a.rows ? r0 + sub : a.rows - 1;
        const T *x = static_cast<const T *>(a.x) + r * a.xs, *dy = static_cast<const T *>(a.dy) + r * a.dys;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int at = (lane + G * i < nv ? lane + G * i : nv - 1) * VEC;
            nx[i] = *reinterpret_cast<const Pack<T, VEC> *>(x + at);
            ny[i] = *reinterpret_cast<const Pack<T, VEC> *>(dy + at);
            nt[i] = *reinterpret_cast<const Pack<T, VEC> *>(dtotal + r * dts + at);
        }
        next_rstd = a.rstd[r];
    };
    const int64_t stride = (int64_t)gridDim.x * RPB;
    if constexpr (AHEAD) fetch((int64_t)blockIdx.x * RPB);
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += stride) {
        const int64_t r = r0 + sub;
        const bool live = r < a.rows;
        if constexpr (!AHEAD) fetch(r0);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) px[i] = nx[i], py[i] = ny[i], pt[i] = nt[i];
        rstd = next_rstd;
        if constexpr (AHEAD) fetch(r0 + stride);
        float s = 0.f, none = 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (live && lane + G * i < nv)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float d = to_float(py[i].v[j]), n = to_float(px[i].v[j]) * rstd;
                    s = fmaf(d * w[i * VEC + j], n, s);
                    dw[i * VEC + j] = fmaf(d, n, dw[i * VEC + j]);
                }
        row_sums<G>(s, none, lds, turn++);
        s *= inv;
        if (!live) continue;
        T *dx = static_cast<T *>(a.y) + r * a.width;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (lane + G * i >= nv) continue;
            Pack<T, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float t = to_float(py[i].v[j]) * w[i * VEC + j], n = to_float(px[i].v[j]) * rstd;
                const float g = rstd * fmaf(-n, s, t);
                o.v[j] = from_float<T>(a.dtotal ? g + to_float(pt[i].v[j]) : g);
            }
            *reinterpret_cast<Pack<T, VEC> *>(dx + (lane + G * i) * VEC) = o;
        }
    }
    if (!a.part) return;
    float *part = a.part + (size_t)blockIdx.x * a.width;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (lane + G * i < nv)
#pragma unroll
                for (int j = 0; j < VEC; ++j) part[(lane + G * i) * VEC + j] = dw[i * VEC + j];
    } else {
        __shared__ float sum[kThreads];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __syncthreads();
            sum[threadIdx.x] = dw[i];
            __syncthreads();
            if (sub == 0 && lane + G * (i / VEC) < nv) {
                float u = 0.f;
                for (int k = 0; k < RPB; ++k) u += sum[k * G + lane];
                part[(lane + G * (i / VEC)) * VEC + i % VEC] = u;
            }
        }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void k_rms_bwd_wide(RmsArgs a) {
    __shared__ float lds[4];
    const float inv = 1.0f / (float)a.width;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + r * a.xs, *dy = static_cast<const T *>(a.dy) + r * a.dys;
        const T *dtotal = static_cast<const T *>(a.dtotal) + r * a.dts;
        const float rstd = a.rstd[r];
        float s = 0.f;
        for (int c = threadIdx.x; c < a.width; c += kThreads)
            s = fmaf(to_float(dy[c]) * (a.weight ? a.weight[c] : 1.f), to_float(x[c]) * rstd, s);
        s = row_sum<kThreads>(s, lds) * inv;
        T *dx = static_cast<T *>(a.y) + r * a.width;
        for (int c = threadIdx.x; c < a.width; c += kThreads) {
            const float t = to_float(dy[c]) * (a.weight ? a.weight[c] : 1.f);
            const float g = rstd * fmaf(-to_float(x[c]) * rstd, s, t);
            dx[c] = from_float<T>(a.dtotal ? g + to_float(dtotal[c]) : g);
        }
    }
}

// The wide rows' part of dw: a thread per column, a strip of rows per blockIdx.y.
// It runs before dx is written, which may lie over total or dy.
template <class T>
__global__ __launch_bounds__(kThreads) void k_rms_cols(RmsArgs a) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.width) return;
    float dw = 0.f;
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y)
        dw = fmaf(to_float(static_cast<const T *>(a.dy)[r * a.dys + c]),
                  to_float(static_cast<const T *>(a.x)[r * a.xs + c]) * a.rstd[r], dw);
    a.part[(size_t)blockIdx.y * a.width + c] = dw;
}

__global__ __launch_bounds__(1024) void k_rms_reduce(RmsArgs a) {
    column_sums(a.part, a.width, a.blocks, block_index(), [&](int64_t c, float v) { a.dweight[c] = a.accumulate ? a.dweight[c] + v : v; });
}

// 16-byte accesses where every row of every array allows them.
template <class T>
bool vectors(const RmsArgs &a) {
    constexpr int VEC = 16 / sizeof(T);
    const int size = sizeof(T);
    return a.width % VEC == 0 && aligned(a.x, a.xs, size) && aligned(a.residual, a.rs, size) &&
           aligned(a.dy, a.dys, size) && aligned(a.dtotal, a.dts, size) && aligned(a.y, a.width, size) &&
           aligned(a.total, a.width, size) && aligned(a.weight, 0, 4) && reinterpret_cast<uintptr_t>(a.q) % VEC == 0;
}

template <class T, int VEC>
bool forward(const RmsArgs &a, hipStream_t s) {
    return for_shape<T, VEC>(a.width, [&](auto g, auto i) {
        constexpr int RPB = kThreads / decltype(g)::value;
        const int64_t blocks = (a.rows + RPB - 1) / RPB;
        k_rms<T, VEC, decltype(g)::value, decltype(i)::value><<<(int)(blocks < 16384 ? blocks : 16384), kThreads, 0, s>>>(a);
    });
}

template <class T, int VEC>
bool backward(const RmsArgs &a, hipStream_t s) {
    return for_shape<T, VEC>(a.width, [&](auto g, auto i) {
        k_rms_bwd<T, VEC, decltype(g)::value, decltype(i)::value><<<a.blocks, kThreads, 0, s>>>(a);
    });
}

template <class T>
hipError_t run_forward(const RmsArgs &a, hipStream_t s) {
    if (!(vectors<T>(a) ? forward<T, 16 / sizeof(T)>(a, s) : forward<T, 1>(a, s)))
        k_rms_wide<T><<<(int)(a.rows < 16384 ? a.rows : 16384), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t run_backward(const RmsArgs &a, hipStream_t s) {
    if (a.rows > 0 && !(vectors<T>(a) ? backward<T, 16 / sizeof(T)>(a, s) : backward<T, 1>(a, s))) {
        if (a.part) {
            k_rms_cols<T><<<dim3((a.width + kThreads - 1) / kThreads, a.blocks), kThreads, 0, s>>>(a);
            if (hipError_t e = hipGetLastError()) return e;
        }
        k_rms_bwd_wide<T><<<(int)(a.rows < 16384 ? a.rows : 16384), kThreads, 0, s>>>(a);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if (a.part) {
        k_rms_reduce<<<column_grid(a.width), 1024, 0, s>>>(a);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_rms(const RmsArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? run_forward<bf16_t>(a, s) : run_forward<float>(a, s);
}

hipError_t launch_rms_backward(const RmsArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? run_backward<bf16_t>(a, s) : run_backward<float>(a, s);
}

}  // namespace rn
