// The selective scan forward: sequences, and one token of each stream.
//
//   s = softplus(dt + bias),  h_i <- exp(s a_i) h_i + s b_i u,  y = sum_i c_i h_i + d u,
//   out = y silu(z).
//
// Bound by its arithmetic: for each token, channel and state an exponential and
// four multiplications or multiply-adds, 24 cycles a wave.  A channel's states stay
// in the registers of its lane from a chunk's first token to its last.  Where there
// are too few channels and sequences for the GPU, sequences are cut into chunks:
// each chunk's end from a state of 0 (k_scan_seq<LOCAL>), then the states that the
// chunks begin with, one after the other (k_scan_join: a chunk's decay is that of
// its summed step sizes), then every chunk with its state.
//
// 16384 ragged tokens of 4096 channels of 16 states, bfloat16: 190 to 213 us for the
// chunks' ends, 18 to 20 for what they begin with, 270 to 298 for all tokens (by the card's
// clock), vector instructions in 98% and 88% of the cycles: a token's step size, gate and
// stores are a quarter of them.  The whole call 447 us; of 4 states 260, of 32 880, of 64 1793.
#include "rn_scan.hpp"

namespace rn {
namespace {

using namespace ops;

// b and c as Packed, where the kernels do not read the caller's own.
template <class T>
__global__ __launch_bounds__(kScanThreads) void k_scan_pack(ScanArgs a) {
    const int64_t i = (int64_t)block_index() * kScanThreads + threadIdx.x, row = i / (2 * a.padded);
    const int at = (int)(i % (2 * a.padded)), n = at / (2 * kStates) * kStates + at % kStates, group = (int)(row % a.groups);
    const int64_t t = row / a.groups;
    if (t >= a.tokens) return;
    float v = 0.f;
    if (n < a.states)
        v = to_float(at % (2 * kStates) < kStates ? static_cast<const T *>(a.b)[t * a.bs + group * a.states + n]
                                                  : static_cast<const T *>(a.c)[t * a.cs + group * a.states + n]);
    a.packed[i] = v;
}

// A thread four states: what each chunk of a sequence begins with, in place of its
// end.  BACK: the same from the last chunk to the first, for gradients (state:
// dfinal).  Loads of kJoin chunks are on their way at once (18 us for 16384 tokens; of 16
// 19.5, of 32 24).
constexpr int kJoin = 8;
template <bool BACK>
__global__ __launch_bounds__(kScanThreads) void k_scan_join(ScanArgs a) {
    const int quads = (a.states + kStates - 1) / kStates;
    const int64_t per = (int64_t)a.channels * quads, i = (int64_t)block_index() * kScanThreads + threadIdx.x;
    if (i >= per * a.n) return;
    const int seq = (int)(i / per), quad = (int)(i % per / a.channels), c = (int)(i % a.channels);
    const Seqs seqs{a.off, a.n, a.tokens, a.even};
    const int begin = seqs.offset(seq), len = max(0, seqs.offset(seq + 1) - begin);
    const int64_t slot = scan_end_slot(a, begin), count = (len + a.chunk() - 1) >> a.log_chunk;
    if (count < 2) return;
    const f32x4 decay = finite_decay(load_decay(a, c, quad * kStates));
    f32x4 h = load_states(a, BACK ? a.dfinal : a.state, seq, c, quad * kStates, true);
    // The chunks of k, k + kJoin, .. one after the other.  GROWS: a chunk's factor may be past
    // float32 and its product with the state not, so such go in factors that are not.
    const auto walk = [&](auto grows) {
        const float most = fmaxf(fmaxf(decay[0], decay[1]), fmaxf(decay[2], decay[3]));
        const float least = fminf(fminf(decay[0], decay[1]), fminf(decay[2], decay[3]));
        for (int64_t k = 0; k < count; k += kJoin) {
            f32x4 end[kJoin];
            float s[kJoin], lo = 0.f, hi = 0.f;
#pragma unroll
            for (int u = 0; u < kJoin; ++u) {           // past the last one: the last one's, not used
                const int64_t m = min(k + u, count - 1), j = slot + (BACK ? count - 1 - m : m);
                end[u] = *own_states(a, a.ends, j, c, quad), s[u] = a.sums[j * a.channels + c];
            }
            if constexpr (decltype(grows)::value) {
#pragma unroll
                for (int u = 0; u < kJoin; ++u) lo = fminf(lo, s[u]), hi = fmaxf(hi, s[u]);
            }
            const bool past = hi * most > 126.f || lo * least > 126.f;
#pragma unroll
            for (int u = 0; u < kJoin; ++u) {
                if (k + u >= count) break;
                *own_states(a, a.ends, slot + (BACK ? count - 1 - k - u : k + u), c, quad) = h;
                f32x4 x = s[u] * decay;
                if (decltype(grows)::value && past)
#pragma unroll
                    for (int n = 0; n < kStates; ++n) {   // 2^378: more than any state but 0 has room for
                        h[n] *= __builtin_amdgcn_exp2f(fminf(fmaxf(x[n] - 126.f, 0.f), 126.f));
                        h[n] *= __builtin_amdgcn_exp2f(fminf(fmaxf(x[n] - 252.f, 0.f), 126.f));
                        x[n] = x[n] > 126.f ? 126.f : x[n];
                    }
#pragma unroll
                for (int n = 0; n < kStates; ++n) h[n] = fmaf(__builtin_amdgcn_exp2f(x[n]), h[n], end[u][n]);
            }
        }
    };
    // With steps by softplus and no a above 0 (which is how such layers are made) states only
    // decay, and nothing is looked at: 16384 tokens 19 us, otherwise 21.
    const bool may = !a.softplus || !(decay[0] <= 0.f && decay[1] <= 0.f && decay[2] <= 0.f && decay[3] <= 0.f);
    if (may) walk(std::true_type{});
    else walk(std::false_type{});
}

// ------------------------------------------------------------------ sequences

// A wave takes 64 channels of a chunk by itself, all S states of a channel in the
// registers of its lane.  LOCAL: of every chunk but a sequence's last, the state at
// its end from 0, and its summed step sizes.  Five waves a SIMD up to 16 states (302 us
// without the bound, 290 with it, 10% more with one of six); bfloat16 ones of 16 put two or
// three registers by in scratch for that.  Of 32 and 64 states three and two waves fit, and
// 28 to 90 of a token's scalars are kept in vector registers' lanes, from where vector
// instructions fetch them.
template <class T, class BC, int S, bool LOCAL>
__global__ __launch_bounds__(64, S <= 16 ? 5 : 1) void k_scan_seq(ScanArgs a) {
    const uint32_t block = block_index();
    const int me = threadIdx.x;
    const ScanChannels where(a, (int)(block % a.blocks), me);
    const int64_t slot = block / a.blocks;
    if (slot >= a.chunks) return;
    const Seqs seqs{a.off, a.n, a.tokens, a.even};
    ScanChunk chunk = scan_chunk_of(a, seqs, slot);
    if (chunk.seq < 0 || (LOCAL && chunk.last)) return;
    chunk.begin = __builtin_amdgcn_readfirstlane(chunk.begin), chunk.len = __builtin_amdgcn_readfirstlane(chunk.len);
    const bool live = where.live;
    const int c = where.c;
    float decay[S], h[S];
#pragma unroll
    for (int q = 0; q < S / kStates; ++q) {
        const f32x4 d = load_decay(a, c, q * kStates);
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        if (!LOCAL) s = chunk.alone() ? load_states(a, a.state, chunk.seq, c, q * kStates, true)
                                      : load_own(a, a.ends, chunk.end, c, q, true);
#pragma unroll
        for (int i = 0; i < kStates; ++i) decay[q * kStates + i] = d[i], h[q * kStates + i] = s[i];
    }
    const float bias = a.dt_bias ? a.dt_bias[c] : 0.f, d = a.d && !LOCAL ? a.d[c] : 0.f;
    const int64_t kept = scan_kept_slot(a, seqs, chunk);
    float total = 0.f;
    // A lane's own numbers, put by so that the tokens' loop can be a loop: unrolled, it
    // would have the scalars of all its tokens at once.
    __shared__ float sx[kBatch][2][64];                 // s, then y; s u
    const uint32_t lane = (uint32_t)c * sizeof(T), to_lane = live ? lane : kNowhere;
    uint32_t ru[kBatch], rdt[kBatch], rz[kBatch];
    const auto fetch = [&](int t0) {                    // tokens past the last are it
        const int64_t first = chunk.begin + t0;
        const auto u = rows_from<T>(a.u, a.us, first), dt = rows_from<T>(a.dt, a.dts, first);
        const auto z = rows_from<T>(LOCAL || !a.z ? a.u : a.z, LOCAL || !a.z ? a.us : a.zs, first);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int r = min(i, chunk.len - 1 - t0) * (int)sizeof(T);
            ru[i] = row_load<T>(u, lane, r * (int)a.us), rdt[i] = row_load<T>(dt, lane, r * (int)a.dts);
            if (!LOCAL) rz[i] = row_load<T>(z, lane, r * (int)(a.z ? a.zs : a.us));
        }
    };
    constexpr int AT = S * sizeof(BC) <= 32 ? (LOCAL ? 4 : 2) : 1;    // tokens whose scalars are there at once (a wave has 100)
    TokenRows<BC> rows_b(a, 0, where.group, chunk.begin), rows_c(a, 1, where.group, chunk.begin);
    if (chunk.len > 0) fetch(0);
#pragma unroll
    for (int n = 0; n < S; ++n) decay[n] = finite_decay(decay[n]);
    for (int t0 = 0; t0 < chunk.len; t0 += kBatch) {
        // The step sizes of all tokens at once, for each is a long chain.
        const int m = min(kBatch, chunk.len - t0);
        float v[kBatch], gate[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            v[i] = row_float<T>(ru[i]);
            if (!LOCAL) gate[i] = a.z ? silu(row_float<T>(rz[i])) : 1.f;
            float s = row_float<T>(rdt[i]) + bias;
            if (a.softplus) s = softplus(s);
            sx[i][0][me] = i < m ? s : 0.f, sx[i][1][me] = i < m ? s * v[i] : 0.f;     // past the end nothing happens
        }
        fetch(min(t0 + kBatch, chunk.len - 1));         // without a branch, so that nothing waits for it here
        if (!LOCAL)
#pragma unroll
            for (int q = 0; q < S / kStates; ++q)
                store_own_if(live && t0 % kTile == 0, a, a.kept, kept + t0 / kTile, c, q,
                             f32x4{h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]});
#pragma unroll 1
        for (int i = 0; i < m; i += AT) {
            Scalars<BC, S> b[AT], cc[AT];
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                b[k].load(rows_b.at);
                if (!LOCAL) cc[k].load(rows_c.at);
                if (t0 + i + k + 1 < chunk.len) rows_b.at += rows_b.stride, rows_c.at += rows_c.stride;
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
                row_store<T>(out, i < m ? to_lane : kNowhere, i * a.channels * (int)sizeof(T),
                             from_float<T>(fmaf(d, v[i], sx[i][0][me]) * gate[i]));
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

// Bound by the states' bytes: 1024 streams of 2048 channels of 16 states, 58 us (4.9
// TB/s) where the pool is in the last-level cache, 88 otherwise (3.2 TB/s: short of a copy's
// 4.7, with one vector of states a lane on its way beside eleven small loads; not taken
// further).  Loads and stores that pass by the caches: 80 and 81.
// L lanes carry a channel, four states each, so that a wave's accesses are one piece;
// blocks walk the streams with the grid's second axis.
template <class T, int L, bool WHOLE>
__global__ __launch_bounds__(kScanThreads) void k_scan_step(ScanArgs a) {
    const int lane = threadIdx.x % L, n0 = lane * kStates;
    const int c = (int)(blockIdx.x * (kScanThreads / L) + threadIdx.x / L);
    if (c >= a.channels) return;                        // a channel's lanes at once
    const int group = c / (a.channels / a.groups);
    f32x4 decay = load_decay(a, c, n0);
    const float bias = a.dt_bias ? a.dt_bias[c] : 0.f, d = a.d ? a.d[c] : 0.f;
    if (a.slots == 0) {                                 // no state to read
        for (int r = blockIdx.y; r < a.n; r += gridDim.y)
            if (lane == 0) static_cast<T *>(a.out)[(int64_t)r * a.channels + c] = from_float<T>(0.f);
        return;
    }
    // The next stream's numbers are on their way while this one's are worked on: loads
    // without branches, from a place of the array where there is nothing to read.
    struct Stream {
        bool there;
        int64_t slot;
        float h[kStates];
        T u, dt, z, b[kStates], c[kStates];
    };
    const T *z_rows = static_cast<const T *>(a.z ? a.z : a.u);
    const int64_t zs = a.z ? a.zs : a.us;
    const auto fetch = [&](int row) {
        Stream s;
        const int64_t r = min(row, a.n - 1), slot = a.ids ? a.ids[r] : r;
        s.there = slot >= 0 && slot < a.slots;
        s.slot = s.there ? slot : 0;
        const float *p = a.final_state + (s.slot * a.channels + c) * a.states;
        if constexpr (WHOLE) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(p + min(n0, a.states - kStates));
#pragma unroll
            for (int i = 0; i < kStates; ++i) s.h[i] = v[i];
        }
        const T *pb = static_cast<const T *>(a.b) + r * a.bs + group * a.states;
        const T *pc = static_cast<const T *>(a.c) + r * a.cs + group * a.states;
#pragma unroll
        for (int i = 0; i < kStates; ++i) {
            const int at = min(n0 + i, a.states - 1);
            if constexpr (!WHOLE) s.h[i] = p[at];
            s.b[i] = pb[at], s.c[i] = pc[at];
        }
        s.u = static_cast<const T *>(a.u)[r * a.us + c], s.dt = static_cast<const T *>(a.dt)[r * a.dts + c];
        s.z = z_rows[r * zs + c];
        return s;
    };
    Stream next = fetch(blockIdx.y);
    decay = finite_decay(decay);
    for (int r = blockIdx.y; r < a.n; r += gridDim.y) {
        const Stream now = next;
        next = fetch(r + gridDim.y);
        T *out = static_cast<T *>(a.out) + (int64_t)r * a.channels + c;
        if (!now.there) {
            if (lane == 0) *out = from_float<T>(0.f);
            continue;
        }
        const float u = to_float(now.u);
        float s = to_float(now.dt) + bias;
        if (a.softplus) s = softplus(s);
        const float x = s * u;
        float y = 0.f;
        f32x4 h;
#pragma unroll
        for (int i = 0; i < kStates; ++i) {
            const bool in = n0 + i < a.states;
            h[i] = fmaf(x, in ? to_float(now.b[i]) : 0.f, __builtin_amdgcn_exp2f(s * decay[i]) * (in ? now.h[i] : 0.f));
            y = fmaf(in ? to_float(now.c[i]) : 0.f, h[i], y);
        }
        store_states(a, a.final_state, now.slot, c, n0, true, h);
        y = fmaf(d, u, over_states<L>(y));
        if (lane == 0) *out = from_float<T>(a.z ? y * silu(to_float(now.z)) : y);
    }
}

inline dim3 join_grid(const ScanArgs &a) {
    const int64_t quads = (a.states + kStates - 1) / kStates;
    return grid_of((a.n * quads * a.channels + kScanThreads - 1) / kScanThreads);
}

template <class T, class BC>
hipError_t sequences(const ScanArgs &a, hipStream_t s) {
    const dim3 grid = grid_of(a.blocks * a.chunks);
    for_states(a.states, [&](auto states) {
        constexpr int S = decltype(states)::value;
        if (a.parts) {
            k_scan_seq<T, BC, S, true><<<grid, 64, 0, s>>>(a);
            k_scan_join<false><<<join_grid(a), kScanThreads, 0, s>>>(a);
        }
        k_scan_seq<T, BC, S, false><<<grid, 64, 0, s>>>(a);
    });
    return hipGetLastError();
}

template <class T>
hipError_t forward(const ScanArgs &a, hipStream_t s) {
    if (scan_direct(a, sizeof(T) == 2)) return sequences<T, T>(a, s);
    if (hipError_t e = launch_scan_pack(a, sizeof(T) == 2, s)) return e;
    return sequences<T, Packed>(a, s);
}

template <class T>
hipError_t step(const ScanArgs &a, hipStream_t s) {
    for_states(a.states, [&](auto states) {
        constexpr int L = decltype(states)::value / kStates, CB = kScanThreads / L;
        const int across = (a.channels + CB - 1) / CB, rows = (2048 + across - 1) / across;
        const dim3 grid(across, a.n < rows ? a.n : rows);
        if (a.whole_states) k_scan_step<T, L, true><<<grid, kScanThreads, 0, s>>>(a);
        else k_scan_step<T, L, false><<<grid, kScanThreads, 0, s>>>(a);
    });
    return hipGetLastError();
}

}  // namespace

int64_t scan_blocks(int channels, int groups) { return (int64_t)groups * ((channels / groups + 63) / 64); }

// Chunks so long that all tokens' are as many blocks as fill the GPU (8 waves a SIMD
// forward; half of that backward, where each block has W waves).  16384 ragged tokens of
// 4096 channels forward, 8192 blocks: the ends 208 us, the join 19, all tokens 300; 4096
// blocks: 256, 13 and 322.
// No shorter than two tiles, or one where sequences are of 64 to 1024 tokens on average:
// 618 tokens of 3218 channels of 64 states forward 197 us with four tiles, 119 with two, 100
// with one, training 732 of 222 of 16 127, 80 and 70; but 146 sequences of 21 tokens
// forward 52, 52 and 92, and training 3 of 2480 121, 103 and 120.  One chunk of four tiles
// for all tokens where it holds them: no sequence has several, which is known here then
// (training 9 of 5 tokens 60, otherwise 73).
// Around the ends of the rule, chunks of one tile and of two, us: 2048 tokens of 256 channels
// of 16 states forward, a mean of 56: 32 and 43, of 64: 32 and 43, of 1024: 43 and 47, of
// 2048: 47 and 49; 4096 of 512: 50 and 56, 50 and 57, 64 and 60, 67 and 59; the same with
// gradients 143 and 149, 139 and 145, 158 and 150, 170 and 154, of 64 states 741 and 711,
// 723 and 690, 641 and 614, 639 and 606.  (Four tiles: slower in all of these.)
// States and direction, which the rule does not look at, shift where the two meet.
int scan_log_chunk(int64_t tokens, int n, int channels, int groups, bool backward) {
    const int64_t blocks = backward ? 4096 : 8192, want = (tokens * scan_blocks(channels, groups) + blocks - 1) / blocks;
    const int64_t mean = n > 0 ? tokens / n : 0;
    int l = tokens <= 64 ? 6 : mean >= 64 && mean <= 1024 ? 4 : 5;
    static_assert(RN_SCAN_KEEP == 16);
    while (l < 30 && ((int64_t)1 << l) < want) ++l;
    return l;
}

// States of a channel as the kernels see them.
int scan_padded(int states) {
    int p = 4;
    while (p < states) p *= 2;
    return p;
}
// Whether the caller's own rows of b and c do: on four bytes, and of as many states.
bool scan_direct(const ScanArgs &a, bool bf16) {
    const auto on_4 = [&](const void *p, int64_t stride) {
        return reinterpret_cast<uintptr_t>(p) % 4 == 0 && (a.tokens < 2 || stride * (bf16 ? 2 : 4) % 4 == 0);
    };
    return a.padded == a.states && on_4(a.b, a.bs) && on_4(a.c, a.cs);
}
hipError_t launch_scan_pack(const ScanArgs &a, bool bf16, hipStream_t s) {
    if (a.tokens == 0) return hipSuccess;
    const dim3 grid = grid_of((a.tokens * a.groups * 2 * a.padded + ops::kScanThreads - 1) / ops::kScanThreads);
    if (bf16) k_scan_pack<ops::bf16_t><<<grid, ops::kScanThreads, 0, s>>>(a);
    else k_scan_pack<float><<<grid, ops::kScanThreads, 0, s>>>(a);
    return hipGetLastError();
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
