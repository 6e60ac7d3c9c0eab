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
                                  : load_states(a, a.ends, chunk.end, c, lane * kStates, live);
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
    for (int t0 = 0; t0 < chunk.len; t0 += kTile) {
        if (!LOCAL && a.kept)
            store_states(a, a.kept, scan_kept_slot(seqs.offset(chunk.seq), chunk.seq) + (chunk.begin + t0 - seqs.offset(chunk.seq)) / kTile,
                         c, lane * kStates, live, h);
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
                h[i] = fmaf(__builtin_amdgcn_exp2f(s * decay[i]), h[i], x * b[i]);
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
        store_states(a, a.ends, chunk.end, c, lane * kStates, live, h);
        if (live && lane == 0) a.sums[chunk.end * a.channels + c] = total;
    } else if (chunk.last) {
        store_states(a, a.final_state, chunk.seq, c, lane * kStates, live, h);
    }
}

// A thread a state: what each chunk of a sequence begins with, in place of its end.
// BACK: the same from the last chunk to the first, for gradients (state: dfinal).
template <bool BACK>
__global__ __launch_bounds__(kScanThreads) void k_scan_join(ScanArgs a) {
    const int64_t per = (int64_t)a.channels * a.states, i = (int64_t)block_index() * kScanThreads + threadIdx.x;
    if (i >= per * a.n) return;
    const int seq = (int)(i / per);
    const int64_t at = i % per;
    const int c = (int)(at / a.states);
    const Seqs seqs{a.off, a.n, a.tokens};
    const int begin = seqs.offset(seq), len = max(0, seqs.offset(seq + 1) - begin);
    const int64_t slot = scan_end_slot(a, begin), count = (len + a.chunk - 1) / a.chunk;
    if (count < 2) return;
    const float decay = a.a[at] * kLog2e;
    const float *from = BACK ? a.dfinal : a.state;
    float h = from ? from[i] : 0.f;
    for (int64_t k = 0; k < count; ++k) {
        const int64_t j = slot + (BACK ? count - 1 - k : k);
        const bool more = k + 1 < count;                // of the last one nothing was computed
        const float end = more ? a.ends[j * per + at] : 0.f, s = more ? a.sums[j * a.channels + c] : 0.f;
        a.ends[j * per + at] = h;
        h = fmaf(__builtin_amdgcn_exp2f(s * decay), h, end);
    }
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
            h[i] = fmaf(__builtin_amdgcn_exp2f(s * decay[i]), h[i], x * b[i]);
            y = fmaf(cc[i], h[i], y);
        }
        store_states(a, a.final_state, slot, c, n0, true, h);
        y = fmaf(d, u, over_states<L>(y));
        if (lane == 0) *out = from_float<T>(a.z ? y * silu(z) : y);
    }
}

template <class T>
hipError_t forward(const ScanArgs &a, hipStream_t s) {
    const dim3 grid = grid_of(a.blocks * a.chunks);
    for_lanes_of(a.states, [&](auto l) {
        constexpr int L = decltype(l)::value;
        if (a.parts) {
            k_scan_seq<T, L, true><<<grid, kScanThreads, 0, s>>>(a);
            k_scan_join<false><<<grid_of(((int64_t)a.n * a.channels * a.states + kScanThreads - 1) / kScanThreads), kScanThreads, 0, s>>>(a);
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
    constexpr int64_t kBlocks = 1024, kShortest = 256;
    int64_t c = (tokens * scan_blocks(channels, groups, states) + kBlocks - 1) / kBlocks;
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
    k_scan_join<true><<<grid_of(((int64_t)a.n * a.channels * a.states + kScanThreads - 1) / kScanThreads), kScanThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace rn
