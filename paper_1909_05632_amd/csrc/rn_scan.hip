// The selective scan forward: sequences, and one token of each stream.
//
//   s = softplus(dt + bias),  h_i <- exp(s a_i) h_i + s b_i u,  y = sum_i c_i h_i + d u,
//   out = y silu(z).
//
// Bound by its arithmetic: for each token, channel and state an exponential and
// four multiplications or multiply-adds.  A channel's states stay in the registers
// of its lanes (rn_scan.hpp) from a chunk's first token to its last.  Where there
// are too few channels and sequences for the GPU, sequences are cut into chunks:
// each chunk's end from a state of 0 (k_scan_seq<LOCAL>), then the states that the
// chunks begin with, one after the other (k_scan_join: a chunk's decay is that of
// its summed step sizes), then every chunk with its state.
#include "rn_scan.hpp"

namespace rn {
namespace {

using namespace ops;

// LOCAL: of every chunk but a sequence's last, the state at its end from 0, and its
// summed step sizes.
template <class T, int L, bool LOCAL>
__global__ __launch_bounds__(kScanThreads) void k_scan_seq(ScanArgs a) {
    constexpr int N = kStates * L, CB = ScanBlock<L>::CB;
    using Q = Quads<L>;
    __shared__ float step[kTile][CB][2];                // s, s u
    __shared__ __attribute__((aligned(16))) float sb[kTile][N], sc[kTile][N];
    __shared__ float sy[LOCAL ? 1 : kTile][CB];
    const uint32_t block = block_index();
    const ScanBlock<L> where(a, (int)(block % a.blocks));
    const int64_t slot = block / a.blocks;
    if (slot >= a.chunks) return;
    const Seqs seqs{a.off, a.n, a.tokens};
    const ScanChunk chunk = scan_chunk_of(a, seqs, slot);
    if (chunk.seq < 0 || (LOCAL && chunk.last)) return;

    const int lane = threadIdx.x % L, mine = threadIdx.x / L, c = where.c0 + mine;
    const bool live = c < where.c1;
    f32x4 decay = load_states(a, a.a, 0, c, lane * kStates, live) * kLog2e;
    f32x4 h = {0.f, 0.f, 0.f, 0.f};
    if (!LOCAL) h = chunk.alone() ? load_states(a, a.state, chunk.seq, c, lane * kStates, live)
                                  : load_own(a, a.ends, chunk.end, c, lane, live);
    float total = 0.f;

    // This thread's quad of channels.
    const int q0 = where.c0 + Q::channel();
    const bool there = q0 < where.c1 && Q::row(0) < kTile;
    float bias[4], d[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool in = there && q0 + j < where.c1;
        bias[j] = in && a.dt_bias ? a.dt_bias[q0 + j] : 0.f;
        d[j] = in && a.d && !LOCAL ? a.d[q0 + j] : 0.f;
    }
    Pack<T, 4> u[Q::PER], dt[Q::PER], z[Q::PER], next_u[Q::PER], next_dt[Q::PER], next_z[Q::PER];
    TileBC<T, L> bc;
    const auto fetch = [&](int t0) {
        bc.load(a, where.group, chunk.begin + t0, chunk.len - t0);
        if (!there) return;
#pragma unroll
        for (int i = 0; i < Q::PER; ++i) {
            const int64_t t = chunk.begin + min(t0 + Q::row(i), chunk.len - 1);
            next_u[i] = load_quad<T>(a, a.u, a.us, t, q0, where.c1);
            next_dt[i] = load_quad<T>(a, a.dt, a.dts, t, q0, where.c1);
            if (!LOCAL && a.z) next_z[i] = load_quad<T>(a, a.z, a.zs, t, q0, where.c1);
        }
    };
    if (chunk.len > 0) fetch(0);
    const int64_t kept = scan_kept_slot(a, seqs, chunk);
    for (int t0 = 0; t0 < chunk.len; t0 += kTile) {
        if (!LOCAL && a.kept) store_own(a, a.kept, kept + t0 / kTile, c, lane, live, h);
        bc.store(a, chunk.len - t0, sb, sc);
#pragma unroll
        for (int i = 0; i < Q::PER; ++i) {
            u[i] = next_u[i], dt[i] = next_dt[i], z[i] = next_z[i];
            const int t = Q::row(i);
            if (t >= kTile) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float s = 0.f, x = 0.f;                 // past the end, and where no channel is: nothing happens
                if (there && t0 + t < chunk.len && q0 + j < where.c1) {
                    s = to_float(dt[i].v[j]) + bias[j];
                    if (a.softplus) s = softplus(s);
                    x = s * to_float(u[i].v[j]);
                }
                step[t][Q::channel() + j][0] = s;
                step[t][Q::channel() + j][1] = x;
            }
        }
        __syncthreads();
        if (t0 + kTile < chunk.len) fetch(t0 + kTile);
        float kept_y = 0.f;
#pragma unroll
        for (int t = 0; t < kTile; ++t) {
            const float s = step[t][mine][0], x = step[t][mine][1];
            const f32x4 b = *reinterpret_cast<const f32x4 *>(&sb[t][lane * kStates]);
            const f32x4 cc = *reinterpret_cast<const f32x4 *>(&sc[t][lane * kStates]);
            float y = 0.f;
#pragma unroll
            for (int i = 0; i < kStates; ++i) {
                h[i] = fmaf(x, b[i], __builtin_amdgcn_exp2f(s * decay[i]) * h[i]);
                if (!LOCAL) y = fmaf(cc[i], h[i], y);
            }
            if (LOCAL) {
                total += s;
            } else {
                y = over_states<L>(y);                  // lane i keeps token i's, of every L
                kept_y = lane == t % L ? y : kept_y;
                if (t % L == L - 1) sy[t - (L - 1) + lane][mine] = kept_y;
            }
        }
        __syncthreads();
        if (LOCAL || !there) continue;
#pragma unroll
        for (int i = 0; i < Q::PER; ++i) {
            const int t = Q::row(i);
            if (t >= kTile || t0 + t >= chunk.len) continue;
            float o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                o[j] = fmaf(d[j], to_float(u[i].v[j]), sy[t][Q::channel() + j]);
                if (a.z) o[j] *= silu(to_float(z[i].v[j]));
            }
            store_quad<T>(a, a.out, chunk.begin + t0 + t, q0, where.c1, o);
        }
    }
    if (LOCAL) {
        store_own(a, a.ends, chunk.end, c, lane, live, h);
        if (live && lane == 0) a.sums[chunk.end * a.channels + c] = total;
    } else if (chunk.last) {
        store_states(a, a.final_state, chunk.seq, c, lane * kStates, live, h);
    }
}

// A thread four states: what each chunk of a sequence begins with, in place of its
// end.  BACK: the same from the last chunk to the first, for gradients (state:
// dfinal).  Loads of kJoin chunks are on their way at once.
constexpr int kJoin = 8;
template <bool BACK>
__global__ __launch_bounds__(kScanThreads) void k_scan_join(ScanArgs a) {
    const int quads = (a.states + kStates - 1) / kStates;
    const int64_t per = (int64_t)a.channels * quads, i = (int64_t)block_index() * kScanThreads + threadIdx.x;
    if (i >= per * a.n) return;
    const int seq = (int)(i / per), quad = (int)(i % per / a.channels), c = (int)(i % a.channels);
    const Seqs seqs{a.off, a.n, a.tokens};
    const int begin = seqs.offset(seq), len = max(0, seqs.offset(seq + 1) - begin);
    const int64_t slot = scan_end_slot(a, begin), count = (len + a.chunk - 1) / a.chunk;
    if (count < 2) return;
    const f32x4 decay = load_states(a, a.a, 0, c, quad * kStates, true) * kLog2e;
    f32x4 h = load_states(a, BACK ? a.dfinal : a.state, seq, c, quad * kStates, true);
    for (int64_t k = 0; k < count; k += kJoin) {
        f32x4 end[kJoin];
        float s[kJoin];
#pragma unroll
        for (int u = 0; u < kJoin; ++u) {               // past the last one: the last one's, not used
            const int64_t m = min(k + u, count - 1), j = slot + (BACK ? count - 1 - m : m);
            end[u] = *own_states(a, a.ends, j, c, quad), s[u] = a.sums[j * a.channels + c];
        }
#pragma unroll
        for (int u = 0; u < kJoin; ++u) {
            if (k + u >= count) break;
            *own_states(a, a.ends, slot + (BACK ? count - 1 - k - u : k + u), c, quad) = h;
#pragma unroll
            for (int n = 0; n < kStates; ++n) h[n] = fmaf(__builtin_amdgcn_exp2f(s[u] * decay[n]), h[n], end[u][n]);
        }
    }
}

// ------------------------------------------------------------------ a lane a channel

// S states in the registers of one lane, for S = 4, 8, 16, 32 and 64: nothing passes
// between lanes, and a token's b and c, the same for all of them, are scalars, which
// the loads' own unit brings.  A wave takes 64 channels of a chunk by itself.
constexpr int kBatch = 8;         // tokens whose loads are on their way at once

template <class T, int S>
struct Scalars {
    uint32_t raw[S * sizeof(T) / 4];
    __device__ void load(const T *p) {
        typedef const __attribute__((address_space(4))) uint32_t *Constant;
        const Constant q = (Constant)(uintptr_t)p;
#pragma unroll
        for (int i = 0; i < (int)(S * sizeof(T) / 4); ++i) raw[i] = q[i];
    }
    __device__ float operator[](int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(raw[i]);
        else return __uint_as_float(i % 2 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
    }
};

// An array's rows from one on: a lane's element of them.
template <class T>
__device__ inline __amdgpu_buffer_rsrc_t rows_from(const void *p, int64_t stride, int64_t row) {
    const char *base = static_cast<const char *>(p) + row * stride * (int)sizeof(T);
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, 0x7fffffff, 0x00027000);
}
template <class T>
__device__ inline uint32_t row_load(__amdgpu_buffer_rsrc_t rows, uint32_t lane, int at) {
    if constexpr (sizeof(T) == 2) return (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(rows, lane, at, 0) << 16;
    else return __builtin_amdgcn_raw_buffer_load_b32(rows, lane, at, 0);
}
template <class T>
__device__ inline void row_store(__amdgpu_buffer_rsrc_t rows, uint32_t lane, int at, T v) {
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), rows, lane, at, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), rows, lane, at, 0);
}

template <class T, int S, bool LOCAL>
__global__ __launch_bounds__(64) void k_scan_lane(ScanArgs a) {
    const uint32_t block = block_index();
    const int of = a.channels / a.groups, per = (of + 63) / 64, cblock = (int)(block % (per * a.groups));
    const int group = cblock / per, c = group * of + cblock % per * 64 + (int)threadIdx.x, c1 = (group + 1) * of;
    const int64_t slot = block / (per * a.groups);
    if (slot >= a.chunks) return;
    const Seqs seqs{a.off, a.n, a.tokens};
    ScanChunk chunk = scan_chunk_of(a, seqs, slot);
    if (chunk.seq < 0 || (LOCAL && chunk.last)) return;
    chunk.begin = __builtin_amdgcn_readfirstlane(chunk.begin), chunk.len = __builtin_amdgcn_readfirstlane(chunk.len);
    const bool live = c < c1;
    const int at = live ? c : c1 - 1;                   // lanes without a channel go along with the last one
    float decay[S], h[S];
#pragma unroll
    for (int q = 0; q < S / kStates; ++q) {
        const f32x4 d = load_states(a, a.a, 0, at, q * kStates, true) * kLog2e;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        if (!LOCAL) s = chunk.alone() ? load_states(a, a.state, chunk.seq, at, q * kStates, true)
                                      : load_own(a, a.ends, chunk.end, at, q, true);
#pragma unroll
        for (int i = 0; i < kStates; ++i) decay[q * kStates + i] = d[i], h[q * kStates + i] = s[i];
    }
    const float bias = a.dt_bias ? a.dt_bias[at] : 0.f, d = a.d && !LOCAL ? a.d[at] : 0.f;
    const int64_t kept = scan_kept_slot(a, seqs, chunk);
    float total = 0.f;
    // A lane's own numbers, put by so that the tokens' loop can be a loop: unrolled, it
    // would have the scalars of all its tokens at once.
    __shared__ float sx[kBatch][2][64];                 // s, then y; s u
    const int me = threadIdx.x;
    const uint32_t lane = (uint32_t)at * sizeof(T), to_lane = live ? lane : 0xfffffff0u;
    uint32_t ru[kBatch], rdt[kBatch], rz[kBatch];
    const auto fetch = [&](int t0) {                    // tokens past the last are it
        const int64_t first = chunk.begin + t0;
        const auto u = rows_from<T>(a.u, a.us, first), dt = rows_from<T>(a.dt, a.dts, first);
        const auto z = rows_from<T>(LOCAL || !a.z ? a.u : a.z, LOCAL || !a.z ? a.us : a.zs, first);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int r = min(i, chunk.len - t0 - 1) * (int)sizeof(T);
            ru[i] = row_load<T>(u, lane, r * (int)a.us), rdt[i] = row_load<T>(dt, lane, r * (int)a.dts);
            if (!LOCAL) rz[i] = row_load<T>(z, lane, r * (int)(a.z ? a.zs : a.us));
        }
    };
    constexpr int AT = S * sizeof(T) <= 32 ? (LOCAL ? 4 : 2) : 1;    // tokens whose scalars are there at once (a wave has 100)
    const T *b_at = static_cast<const T *>(a.b) + chunk.begin * a.bs + group * S;
    const T *c_at = static_cast<const T *>(a.c) + chunk.begin * a.cs + group * S;
    if (chunk.len > 0) fetch(0);
    for (int t0 = 0; t0 < chunk.len; t0 += kBatch) {
        // The step sizes of all tokens at once, for each is a long chain.
        const int m = min(kBatch, chunk.len - t0);
        float v[kBatch], gate[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            v[i] = __uint_as_float(ru[i]);
            if (!LOCAL) gate[i] = a.z ? silu(__uint_as_float(rz[i])) : 1.f;
            float s = __uint_as_float(rdt[i]) + bias;
            if (a.softplus) s = softplus(s);
            sx[i][0][me] = i < m ? s : 0.f, sx[i][1][me] = i < m ? s * v[i] : 0.f;     // past the end nothing happens
        }
        if (t0 + kBatch < chunk.len) fetch(t0 + kBatch);
        if (!LOCAL && a.kept && t0 % kTile == 0)
#pragma unroll
            for (int q = 0; q < S / kStates; ++q)
                store_own(a, a.kept, kept + t0 / kTile, c, q, live, f32x4{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]});
#pragma unroll 1
        for (int i = 0; i < m; i += AT) {
            Scalars<T, S> b[AT], cc[AT];
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                b[k].load(b_at);
                if (!LOCAL) cc[k].load(c_at);
                if (t0 + i + k + 1 < chunk.len) b_at += a.bs, c_at += a.cs;
            }
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                const float s = sx[i + k][0][me], x = sx[i + k][1][me];
                float y[S / kStates];                   // by quads, then in a tree: the sums of the other kernels
#pragma unroll
                for (int q = 0; q < S / kStates; ++q) {
                    y[q] = 0.f;
#pragma unroll
                    for (int n = q * kStates; n < (q + 1) * kStates; ++n) {
                        h[n] = fmaf(x, b[k][n], __builtin_amdgcn_exp2f(s * decay[n]) * h[n]);
                        if (!LOCAL) y[q] = fmaf(cc[k][n], h[n], y[q]);
                    }
                }
#pragma unroll
                for (int w = 1; w < S / kStates; w *= 2)
#pragma unroll
                    for (int q = 0; q < S / kStates; q += 2 * w) y[q] += y[q + w];
                if (LOCAL) total += s;
                else sx[i + k][0][me] = y[0];
            }
        }
        if (!LOCAL) {
            const auto out = rows_from<T>(a.out, a.channels, chunk.begin + t0);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i < m)
                    row_store<T>(out, to_lane, i * a.channels * (int)sizeof(T), from_float<T>(fmaf(d, v[i], sx[i][0][me]) * gate[i]));
        }
    }
#pragma unroll
    for (int q = 0; q < S / kStates; ++q) {
        const f32x4 v = {h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]};
        if (LOCAL) store_own(a, a.ends, chunk.end, c, q, live, v);
        else if (chunk.last) store_states(a, a.final_state, chunk.seq, c, q * kStates, live, v);
    }
    if (LOCAL && live) a.sums[chunk.end * a.channels + c] = total;
}

// ------------------------------------------------------------------ one token

// Blocks walk the streams with the grid's second axis; L lanes a channel.
template <class T, int L>
__global__ __launch_bounds__(kScanThreads) void k_scan_step(ScanArgs a) {
    const int lane = threadIdx.x % L, n0 = lane * kStates;
    const int c = (int)(blockIdx.x * (kScanThreads / L) + threadIdx.x / L);
    if (c >= a.channels) return;                        // a channel's lanes at once
    const int group = c / (a.channels / a.groups);
    const f32x4 decay = load_states(a, a.a, 0, c, n0, true) * kLog2e;
    const float bias = a.dt_bias ? a.dt_bias[c] : 0.f, d = a.d ? a.d[c] : 0.f;
    for (int r = blockIdx.y; r < a.n; r += gridDim.y) {
        const int64_t slot = a.ids ? a.ids[r] : r;
        T *out = static_cast<T *>(a.out) + (int64_t)r * a.channels + c;
        if (slot < 0 || slot >= a.slots) {
            if (lane == 0) *out = from_float<T>(0.f);
            continue;
        }
        f32x4 h = load_states(a, a.final_state, slot, c, n0, true);
        const float u = to_float(static_cast<const T *>(a.u)[r * a.us + c]);
        float s = to_float(static_cast<const T *>(a.dt)[r * a.dts + c]) + bias;
        const float z = a.z ? to_float(static_cast<const T *>(a.z)[r * a.zs + c]) : 0.f;
        const T *pb = static_cast<const T *>(a.b) + r * a.bs + group * a.states + n0;
        const T *pc = static_cast<const T *>(a.c) + r * a.cs + group * a.states + n0;
        float b[kStates], cc[kStates];
#pragma unroll
        for (int i = 0; i < kStates; ++i) {
            const bool in = n0 + i < a.states;
            b[i] = in ? to_float(pb[i]) : 0.f, cc[i] = in ? to_float(pc[i]) : 0.f;
        }
        if (a.softplus) s = softplus(s);
        const float x = s * u;
        float y = 0.f;
#pragma unroll
        for (int i = 0; i < kStates; ++i) {
            h[i] = fmaf(x, b[i], __builtin_amdgcn_exp2f(s * decay[i]) * h[i]);
            y = fmaf(cc[i], h[i], y);
        }
        store_states(a, a.final_state, slot, c, n0, true, h);
        y = fmaf(d, u, over_states<L>(y));
        if (lane == 0) *out = from_float<T>(a.z ? y * silu(z) : y);
    }
}

inline dim3 join_grid(const ScanArgs &a) {
    const int64_t quads = (a.states + kStates - 1) / kStates;
    return grid_of((a.n * quads * a.channels + kScanThreads - 1) / kScanThreads);
}

// A lane a channel: where all of its states are whole quads, a power of two of them,
// and b and c are on the four bytes that scalar loads need.
template <class T>
bool by_lane(const ScanArgs &a) {
    const auto on_4 = [](const void *p, int64_t stride) {
        return reinterpret_cast<uintptr_t>(p) % 4 == 0 && stride * (int)sizeof(T) % 4 == 0;
    };
    return a.states >= 4 && (a.states & (a.states - 1)) == 0 && on_4(a.b, a.bs) && on_4(a.c, a.cs);
}

template <class T>
hipError_t forward(const ScanArgs &a, hipStream_t s) {
    if (by_lane<T>(a)) {
        const dim3 grid = grid_of((int64_t)a.groups * ((a.channels / a.groups + 63) / 64) * a.chunks);
        for_lanes_of(a.states, [&](auto l) {
            constexpr int S = decltype(l)::value * kStates;
            if (a.parts) {
                k_scan_lane<T, S, true><<<grid, 64, 0, s>>>(a);
                k_scan_join<false><<<join_grid(a), kScanThreads, 0, s>>>(a);
            }
            k_scan_lane<T, S, false><<<grid, 64, 0, s>>>(a);
        });
        return hipGetLastError();
    }
    const dim3 grid = grid_of(a.blocks * a.chunks);
    for_lanes_of(a.states, [&](auto l) {
        constexpr int L = decltype(l)::value;
        if (a.parts) {
            k_scan_seq<T, L, true><<<grid, kScanThreads, 0, s>>>(a);
            k_scan_join<false><<<join_grid(a), kScanThreads, 0, s>>>(a);
        }
        k_scan_seq<T, L, false><<<grid, kScanThreads, 0, s>>>(a);
    });
    return hipGetLastError();
}

template <class T>
hipError_t step(const ScanArgs &a, hipStream_t s) {
    for_lanes_of(a.states, [&](auto l) {
        constexpr int L = decltype(l)::value, CB = kScanThreads / L;
        const int across = (a.channels + CB - 1) / CB, rows = (2048 + across - 1) / across;
        k_scan_step<T, L><<<dim3(across, a.n < rows ? a.n : rows), kScanThreads, 0, s>>>(a);
    });
    return hipGetLastError();
}

}  // namespace

int scan_lanes(int states) {
    int l = 0;
    ops::for_lanes_of(states, [&](auto x) { l = decltype(x)::value; });
    return l;
}
int64_t scan_blocks(int channels, int groups, int states) {
    const int cb = ops::kScanThreads / scan_lanes(states);
    return (int64_t)groups * ((channels / groups + cb - 1) / cb);
}
// Chunks so long that all tokens' are kBlocks blocks, but no shorter than kShortest:
// below, what the chunks' ends cost is more than what they free.
int scan_chunk(int64_t tokens, int channels, int groups, int states) {
    constexpr int64_t kBlocks = 8192, kShortest = 64;
    int64_t c = (tokens * groups * ((channels / groups + 63) / 64) + kBlocks - 1) / kBlocks;
    c = (c + RN_SCAN_KEEP - 1) / RN_SCAN_KEEP * RN_SCAN_KEEP;
    return (int)(c < kShortest ? kShortest : c < (1 << 30) ? c : 1 << 30);
}

hipError_t launch_scan(const ScanArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}
hipError_t launch_scan_step(const ScanArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? step<bf16_t>(a, s) : step<float>(a, s);
}
hipError_t launch_scan_join_back(const ScanArgs &a, hipStream_t s) {
    k_scan_join<true><<<join_grid(a), kScanThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace rn
