// Short causal convolution of each channel by itself, and its gradients.
//
//   pre_t = b + sum_(k < K) w_k x_(t-K+1+k),  out = silu(pre) or pre.
// With p_t = dJ/dpre_t = dout_t silu'(pre_t):
//   dx_t = sum_k w_k p_(t+K-1-k),  dw_k = sum_t p_t x_(t-K+1+k),  db = sum_t p_t,
// and the window's rows and the final window's gradient where those reach beyond
// the sequence.
//
// Bound by HBM, and nearly so by its arithmetic (vector instructions in 7 of 10
// cycles).  A thread takes VEC channels (16 bytes) of a run of tokens, with the last
// K - 1 inputs in registers; a run begins with the K - 1 tokens before it and, backward,
// goes on for the K - 1 behind it, from the caches.  16384 ragged tokens of 4096
// channels, bfloat16: forward 56 us (4.9 TB/s), backward 104 (4.3 TB/s) and 5.5 for the
// weights' sums over blocks.
#include "rn_rows.hpp"
#include "rn_seq.hpp"

namespace rn {
namespace {

using namespace ops;

constexpr int kAhead = 4;         // rows whose loads are on their way at once

// The channels' weights, and their inputs at the last K - 1 tokens, oldest first.
template <class T, int VEC, int K>
struct Taps {
    static constexpr int W = K > 1 ? K - 1 : 1;
    float w[K][VEC], b[VEC], x[W][VEC];

    __device__ void weights(const CausalArgs &a, int c) {
        float f[VEC * K];
        const float *p = a.weight + (int64_t)c * K;
        if constexpr (VEC > 1) {                    // on 16 bytes
            load_f32<VEC * K>(p, f, 0.f);
        } else {
#pragma unroll
            for (int i = 0; i < VEC * K; ++i) f[i] = p[i];
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][j] = f[j * K + k];
            b[j] = a.bias ? a.bias[c + j] : 0.f;
        }
    }
    // The K - 1 inputs before token t of a sequence that begins at `begin`.
    __device__ void before(const CausalArgs &a, int seq, int begin, int t, int c) {
#pragma unroll
        for (int i = 0; i + 1 < K; ++i) row(a, seq, begin, t - (K - 1) + i, c, x[i]);
    }
    // Input t, which lies in the window where it is before `begin`.
    static __device__ void row(const CausalArgs &a, int seq, int begin, int t, int c, float (&v)[VEC]) {
        if (t >= begin) {
            load_as<T, VEC>(static_cast<const T *>(a.x) + (int64_t)t * a.xs + c, v);
        } else if (a.window) {
            load_as<T, VEC>(static_cast<const T *>(a.window) + ((int64_t)seq * (K - 1) + (t - begin + K - 1)) * a.channels + c, v);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] = 0.f;
        }
    }
    // One rounding a product and sum, oldest tap first, the bias last.
    __device__ float pre(int j, float now) const {
#pragma clang fp contract(off)
        float s = 0.f;
#pragma unroll
        for (int k = 0; k + 1 < K; ++k) s = k ? s + w[k][j] * x[k][j] : w[k][j] * x[k][j];
        return (K > 1 ? s + w[K - 1][j] * now : w[0][j] * now) + b[j];
    }
    __device__ void push(const float (&now)[VEC]) {
        if constexpr (K > 1) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
#pragma unroll
                for (int k = 0; k + 2 < K; ++k) x[k][j] = x[k + 1][j];
                x[K - 2][j] = now[j];
            }
        }
    }
};

// Where a thread works: `lanes` threads side by side over the channels, 256 / lanes
// runs of a.run tokens a block.  The blocks behind the last run take the sequences' ends,
// where those are wanted: a large grid is rounded up, so there may be such blocks anyway.
struct Place {
    int c;                        // first channel, or beyond the last
    int64_t run;                  // run of tokens, or row of the sequences' ends
    bool ends;
    int block;                    // row of blocks
    __device__ Place(const CausalArgs &a, int vec) {
        const int across = (a.channels + a.lanes * vec - 1) / (a.lanes * vec);
        const uint32_t i = block_index(), y = i / across;
        c = (int)(i % across * a.lanes + threadIdx.x % a.lanes) * vec;
        const int per = kThreads / a.lanes;
        ends = y >= (uint32_t)a.run_blocks;
        block = (int)(ends ? y - a.run_blocks : y);
        run = (int64_t)block * per + threadIdx.x / a.lanes;
    }
};

// Row `run` of the final windows: of the sequence run / (K - 1) its input
// len - (K - 1) + i, or the window's where the sequence is shorter.
template <class T, int VEC, int K>
__device__ inline void final_row(const CausalArgs &a, const Seqs &s, const Place &p) {
    if constexpr (K > 1) {
        if (!a.final_window || p.run >= (int64_t)a.n * (K - 1)) return;
        const int seq = (int)(p.run / (K - 1)), i = (int)(p.run % (K - 1));
        const int begin = s.offset(seq), end = max(begin, s.offset(seq + 1));
        float v[VEC];
        Taps<T, VEC, K>::row(a, seq, begin, max(end - (K - 1) + i, begin - (K - 1)), p.c, v);
        store_as<T, VEC>(static_cast<T *>(a.final_window) + p.run * a.channels + p.c, v);
    }
}

template <class T, int VEC, int K>
__global__ __launch_bounds__(kThreads) void k_conv_seq(CausalArgs a) {
    const Place p(a, VEC);
    if (p.c >= a.channels) return;
    const Seqs s{a.off, a.n, a.tokens, a.even};
    if (p.ends) return final_row<T, VEC, K>(a, s, p);
    const int64_t from = max(p.run * a.run, (int64_t)s.offset(0));
    const int to = (int)min((p.run + 1) * a.run, (int64_t)s.offset(a.n));      // what no sequence owns is left alone
    if (from >= to) return;
    int t = (int)from;
    At at(s, t);
    Taps<T, VEC, K> taps;
    taps.weights(a, p.c);
    taps.before(a, at.seq, at.begin, t, p.c);
    const T *x = static_cast<const T *>(a.x) + p.c;
    T *out = static_cast<T *>(a.out) + p.c;
    Pack<T, VEC> next[kAhead];
    const auto fetch = [&](int from) {                  // the next rows are on their way while these are worked on
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            next[u] = *reinterpret_cast<const Pack<T, VEC> *>(x + (int64_t)min(from + u, to - 1) * a.xs);
    };
    fetch(t);
    for (; t < to; t += kAhead) {
        float now[kAhead][VEC];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int j = 0; j < VEC; ++j) now[u][j] = to_float(next[u].v[j]);
        fetch(t + kAhead);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (t + u >= to) break;
            if (t + u >= at.end) {
                at.next(s, t + u);
                taps.before(a, at.seq, at.begin, t + u, p.c);
            }
            float y[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                y[j] = taps.pre(j, now[u][j]);
                if (a.silu) y[j] = silu(y[j]);
            }
            store_as<T, VEC>(out + (int64_t)(t + u) * a.channels, y);
            taps.push(now[u]);
        }
    }
}

// Row `run` of the windows' gradient: window input i of a sequence is seen by its
// tokens 0..i, and is a row of the final window where the sequence is that short.
template <class T, int VEC, int K>
__device__ inline void window_row(const CausalArgs &a, const Seqs &s, const Place &p) {
    if constexpr (K > 1) {
        if (!a.dwindow || p.run >= (int64_t)a.n * (K - 1)) return;
        const int seq = (int)(p.run / (K - 1)), i = (int)(p.run % (K - 1));
        const int begin = s.offset(seq), end = max(begin, s.offset(seq + 1)), len = end - begin;
        Taps<T, VEC, K> taps;
        taps.weights(a, p.c);
        float d[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) d[j] = 0.f;
        if (a.dfinal && i >= len)
            load_as<T, VEC>(static_cast<const T *>(a.dfinal) + ((int64_t)seq * (K - 1) + i - len) * a.channels + p.c, d);
        taps.before(a, seq, begin, begin, p.c);
#pragma unroll
        for (int t = 0; t + 1 < K; ++t) {
            if (t > i || t >= len) break;
            float now[VEC], g[VEC];
            load_as<T, VEC>(static_cast<const T *>(a.x) + (int64_t)(begin + t) * a.xs + p.c, now);
            load_as<T, VEC>(static_cast<const T *>(a.dout) + (int64_t)(begin + t) * a.channels + p.c, g);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                if (a.silu) g[j] *= silu_slope(taps.pre(j, now[j]));
#pragma unroll
                for (int k = 0; k < K; ++k)
                    if (k == i - t) d[j] = fmaf(taps.w[k][j], g[j], d[j]);
            }
            taps.push(now);
        }
        store_as<T, VEC>(static_cast<T *>(a.dwindow) + p.run * a.channels + p.c, d);
    }
}

template <class T, int VEC, int K>
__global__ __launch_bounds__(kThreads) void k_conv_bwd(CausalArgs a) {
    constexpr int N = (K + 1) * VEC;
    __shared__ float sum[N][kThreads];
    const Place p(a, VEC);
    const Seqs s{a.off, a.n, a.tokens, a.even};
    if (p.ends) {
        if (p.c < a.channels) window_row<T, VEC, K>(a, s, p);
        return;
    }
    float dw[K][VEC], db[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        db[j] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) dw[k][j] = 0.f;
    }
    const int64_t from = max(p.run * a.run, (int64_t)s.offset(0));
    const int to = (int)min((p.run + 1) * a.run, (int64_t)s.offset(a.n));
    if (from < to && p.c < a.channels) {
        const int first = (int)from;
        int t = first;
        At at(s, t);
        Taps<T, VEC, K> taps;
        taps.weights(a, p.c);
        taps.before(a, at.seq, at.begin, t, p.c);
        const T *x = static_cast<const T *>(a.x) + p.c, *dout = static_cast<const T *>(a.dout) + p.c;
        T *dx = static_cast<T *>(a.dx) + p.c;
        float d[K][VEC];          // dx of token t - k, as far as tokens up to t give it
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < VEC; ++j) d[k][j] = 0.f;
        // The tokens behind the run that its own are seen by.
        const auto stop_of = [&] { return max(to, min(to + K - 1, at.end)); };
        int stop = at.end < to ? to : stop_of();
        // The next rows are on their way while these are worked on.
        Pack<T, VEC> next_x[kAhead], next_g[kAhead];
        const auto fetch = [&](int from) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t row = min((int64_t)from + u, a.tokens - 1);
                next_x[u] = *reinterpret_cast<const Pack<T, VEC> *>(x + row * a.xs);
                next_g[u] = *reinterpret_cast<const Pack<T, VEC> *>(dout + row * a.channels);
            }
        };
        fetch(t);
        for (; t < stop; t += kAhead) {
            float now[kAhead][VEC], g[kAhead][VEC];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int j = 0; j < VEC; ++j) now[u][j] = to_float(next_x[u].v[j]), g[u][j] = to_float(next_g[u].v[j]);
            fetch(t + kAhead);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = t + u;
                if (i >= stop) break;
                if (i >= at.end) {
                    at.next(s, i);
                    taps.before(a, at.seq, at.begin, i, p.c);
                    if (at.end >= to) stop = stop_of();
                }
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    if (a.silu) g[u][j] *= silu_slope(taps.pre(j, now[u][j]));
#pragma unroll
                    for (int k = K - 1; k > 0; --k) d[k][j] = fmaf(taps.w[K - 1 - k][j], g[u][j], d[k - 1][j]);
                    d[0][j] = taps.w[K - 1][j] * g[u][j];
                    if (i < to) {
                        db[j] += g[u][j];
#pragma unroll
                        for (int k = 0; k + 1 < K; ++k) dw[k][j] = fmaf(g[u][j], taps.x[k][j], dw[k][j]);
                        dw[K - 1][j] = fmaf(g[u][j], now[u][j], dw[K - 1][j]);
                    }
                }
                const int low = max(first, at.begin);
                if (i - (K - 1) >= low) store_as<T, VEC>(dx + (int64_t)(i - (K - 1)) * a.channels, d[K - 1]);
                if (i + 1 == at.end) {         // the sequence's last: what no later token adds to
#pragma unroll
                    for (int k = 0; k + 1 < K; ++k) {
                        if (i - k < low || i - k >= to) continue;
                        float v[VEC];
#pragma unroll
                        for (int j = 0; j < VEC; ++j) v[j] = 0.f;
                        if (a.dfinal)
                            load_as<T, VEC>(static_cast<const T *>(a.dfinal) + ((int64_t)at.seq * (K - 1) + K - 2 - k) * a.channels + p.c, v);
#pragma unroll
                        for (int j = 0; j < VEC; ++j) v[j] += d[k][j];
                        store_as<T, VEC>(dx + (int64_t)(i - k) * a.channels, v);
                    }
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) d[k][j] = 0.f;
                }
                taps.push(now[u]);
            }
        }
    }
    // The block's runs in a fixed order: part [block][channels][K], then [channels].
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
#pragma unroll
        for (int k = 0; k < K; ++k) sum[j * K + k][threadIdx.x] = dw[k][j];
        sum[VEC * K + j][threadIdx.x] = db[j];
    }
    __syncthreads();
    const int across = a.lanes * VEC, c0 = p.c - (int)(threadIdx.x % a.lanes) * VEC;
    float *part = a.part + (int64_t)p.block * a.channels * (K + 1);
    for (int i = threadIdx.x; i < across * (K + 1); i += kThreads) {
        const int c = i < across * K ? i / K : i - across * K, k = i < across * K ? i % K : K;
        if (c0 + c >= a.channels) continue;
        const float *row = sum[k < K ? c % VEC * K + k : VEC * K + c % VEC] + c / VEC;
        float v = 0.f;
        for (int r = 0; r < kThreads; r += a.lanes) v += row[r];
        part[k < K ? (int64_t)(c0 + c) * K + k : (int64_t)a.channels * K + c0 + c] = v;
    }
}

__global__ __launch_bounds__(1024) void k_conv_reduce(CausalArgs a) {
    const int64_t weights = (int64_t)a.channels * a.taps;
    column_sums(a.part, weights + a.channels, a.run_blocks, block_index(), [&](int64_t c, float v) {
        if (c < weights) a.dweight[c] = v;
        else a.dbias[c - weights] = v;
    });
}

// A token of each stream: its window moves up by one.
template <class T, int VEC, int K>
__global__ __launch_bounds__(kThreads) void k_conv_step(CausalArgs a) {
    const int across = a.channels / VEC;
    const int64_t i = (int64_t)block_index() * kThreads + threadIdx.x;
    const int r = (int)(i / across), c = (int)(i % across) * VEC;
    if (i >= (int64_t)a.n * across) return;
    const int64_t slot = a.ids ? a.ids[r] : r;
    T *out = static_cast<T *>(a.out) + (int64_t)r * a.channels + c;
    float y[VEC];
    if (slot < 0 || slot >= a.slots) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) y[j] = 0.f;
        return store_as<T, VEC>(out, y);
    }
    Taps<T, VEC, K> taps;
    T *window = static_cast<T *>(a.final_window) + (slot * (K - 1)) * a.channels + c;
    float now[VEC];
    load_as<T, VEC>(static_cast<const T *>(a.x) + (int64_t)r * a.xs + c, now);
#pragma unroll
    for (int k = 0; k + 1 < K; ++k) load_as<T, VEC>(window + (int64_t)k * a.channels, taps.x[k]);
    taps.weights(a, c);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        // A stream's next token depends on what is rounded here, and the call's time does
        // not: the library's exponential and a true quotient, where sequences take the
        // hardware's (an ulp each; 83 us in place of 58 for 16384 x 4096).
        y[j] = taps.pre(j, now[j]);
        if (a.silu) y[j] *= 1.f / (1.f + expf(-y[j]));
    }
    store_as<T, VEC>(out, y);
    taps.push(now);
#pragma unroll
    for (int k = 0; k + 1 < K; ++k) store_as<T, VEC>(window + (int64_t)k * a.channels, taps.x[k]);
}

template <class F>
void for_taps(int taps, F &&f) {
    using std::integral_constant;
    if (taps == 1) f(integral_constant<int, 1>{});
    else if (taps == 2) f(integral_constant<int, 2>{});
    else if (taps == 3) f(integral_constant<int, 3>{});
    else f(integral_constant<int, 4>{});
}

// 16-byte accesses where every row of every array allows them.
template <class T>
bool vectors(const CausalArgs &a) {
    constexpr int VEC = 16 / sizeof(T), size = sizeof(T);
    if (a.channels % VEC || !aligned(a.x, a.xs, size) || !aligned(a.weight, 0, 4)) return false;
    for (const void *p : {a.window, static_cast<const void *>(a.final_window), static_cast<const void *>(a.out), a.dout,
                          a.dfinal, static_cast<const void *>(a.dx), static_cast<const void *>(a.dwindow)})
        if (!aligned(p, 0, size)) return false;
    return true;
}

// Threads side by side: a wave's worth, or what few channels need.
int lanes_of(int channels, int vec) {
    int l = 64;
    while (l > 8 && (l / 2) * vec >= channels) l /= 2;
    return l;
}

// Tokens a thread: half as many where that leaves fewer than 2048 waves of 8 channels
// a lane.  16384 x 4096 bfloat16 forward take 56 us with 32 and 59 with 64, backward 112
// and 103; 2048 x 2048 forward 9 us with 8 and 17 with 32, backward 24 with 8 and 66 with 64.
int run_of(int64_t tokens, int channels, bool backward) {
    int r = backward ? 64 : 32;
    while (r > 8 && tokens * channels / (8 * 64) / r < 2048) r /= 2;
    return r;
}

template <class T, int VEC>
hipError_t run(CausalArgs a, bool backward, hipStream_t s) {
    a.lanes = lanes_of(a.channels, VEC);
    a.run = run_of(a.tokens, a.channels, backward);
    const int64_t per = kThreads / a.lanes;
    const bool ends = a.taps > 1 && (backward ? a.dwindow : a.final_window);
    const int64_t runs = (a.tokens + a.run - 1) / a.run, rows = ends ? (int64_t)a.n * (a.taps - 1) : 0;
    a.run_blocks = (int)((runs + per - 1) / per);
    const int64_t across = (a.channels + a.lanes * VEC - 1) / (a.lanes * VEC);
    const int64_t blocks = across * (a.run_blocks + (rows + per - 1) / per);
    if (blocks > 0)
        for_taps(a.taps, [&](auto k) {
            constexpr int K = decltype(k)::value;
            if (backward) k_conv_bwd<T, VEC, K><<<grid_of(blocks), kThreads, 0, s>>>(a);
            else k_conv_seq<T, VEC, K><<<grid_of(blocks), kThreads, 0, s>>>(a);
        });
    if (hipError_t e = hipGetLastError()) return e;
    if (backward) k_conv_reduce<<<column_grid((int64_t)a.channels * (a.taps + 1)), 1024, 0, s>>>(a);
    return hipGetLastError();
}

template <class T, int VEC>
hipError_t run_step(const CausalArgs &a, hipStream_t s) {
    const int64_t threads = (int64_t)a.n * (a.channels / VEC);
    for_taps(a.taps, [&](auto k) {
        k_conv_step<T, VEC, decltype(k)::value><<<grid_of((threads + kThreads - 1) / kThreads), kThreads, 0, s>>>(a);
    });
    return hipGetLastError();
}

template <class T>
hipError_t dispatch(const CausalArgs &a, bool backward, hipStream_t s) {
    return vectors<T>(a) ? run<T, 16 / sizeof(T)>(a, backward, s) : run<T, 1>(a, backward, s);
}

}  // namespace

// Rows of partial weight gradients: the most that a call of this size has, whatever
// its alignment (kThreads / 64 runs of tokens a block, or more).
int64_t causal_parts(int64_t tokens, int channels) {
    const int64_t per = (int64_t)run_of(tokens, channels, true) * (ops::kThreads / 64);
    return (tokens + per - 1) / per;
}

hipError_t launch_causal(const CausalArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? dispatch<bf16_t>(a, false, s) : dispatch<float>(a, false, s);
}
hipError_t launch_causal_backward(const CausalArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? dispatch<bf16_t>(a, true, s) : dispatch<float>(a, true, s);
}
hipError_t launch_causal_step(const CausalArgs &a, bool bf16, hipStream_t s) {
    if (bf16) return vectors<bf16_t>(a) ? run_step<bf16_t, 8>(a, s) : run_step<bf16_t, 1>(a, s);
    return vectors<float>(a) ? run_step<float, 4>(a, s) : run_step<float, 1>(a, s);
}

}  // namespace rn
