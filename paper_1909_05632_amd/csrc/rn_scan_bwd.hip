// Gradients of the selective scan.
//
// With s, h and y as forward, e_i = exp(s a_i), k_i = e_i h_i' (h' the state before),
// p = dout silu(z) = dJ/dy, and from a sequence's last token on
//   g_i <- g_i + c_i p   (dJ/dh_i after the token):
//   ds = sum_i g_i a_i k_i + u sum_i g_i b_i,   du = s sum_i g_i b_i + d p,
//   ddt = ds softplus'(dt + bias),  dz = dout y silu'(z),
//   da_i += s g_i k_i,  db_i = sum over channels g_i s u,  dc_i = sum over channels h_i p,
//   g_i <- e_i g_i.
// A chunk goes by tiles of RN_SCAN_KEEP tokens from its last: the states of a tile
// are computed again from the one that the forward call kept, into registers.
// Where sequences are cut into chunks, what g is at their ends comes first, as
// forward (k_scan_back: each chunk's g at its begin from 0).
//
// Bound by its arithmetic: for each token, channel and state one and a half
// exponentials, 15 multiplications or multiply-adds, and a third of that again for the
// sums over channels: those of a wave in registers (over_channels), of all waves by
// another kernel, each in a fixed order.  8192 ragged tokens of 2048 channels of 16
// states, bfloat16: k_scan_bwd 276 to 293 us (by the card's clock), vector instructions
// in 3 of 4 of its cycles; k_scan_back 75, its join 15, the sums over blocks 20.
#include "rn_rows.hpp"
#include "rn_scan.hpp"

namespace rn {
namespace {

using namespace ops;

// Two lanes whose numbers differ in one bit: the one without it gets a of both, the
// one with it b of both.
template <int BIT>
__device__ inline float exchange(float a, float b) {
    if constexpr (BIT == 5 || BIT == 4) {
        const auto r = BIT == 5
            ? __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false)
            : __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        const bool up = threadIdx.x >> BIT & 1;
        const float keep = up ? b : a;
        if constexpr (BIT == 3) return keep + dpp<0x128>(up ? a : b);           // 8 on in a row of 16
        else return keep + dpp<0x114, 0xa>(b, dpp<0x104, 0x5>(a));              // 4 on, and 4 back
    }
}
// 16 values a lane, summed over the wave's lanes: of value i, the sum is with the lanes
// 4 i .. 4 i + 3.  Every step joins two lanes, which keep half of the values each; the
// last two add.
__device__ inline float over_channels(float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = exchange<5>(v[i], v[i + 8]);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = exchange<4>(v[i], v[i + 4]);
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = exchange<3>(v[i], v[i + 2]);
    float r = exchange<2>(v[0], v[1]);
    r += dpp<0x4e>(r);
    return r + dpp<0xb1>(r);
}

// A channel's element of u, dt, z and dout at a token, as loaded.
struct Raw {
    uint32_t u, dt, z, dout;
};
template <class T>
struct RawRows {
    __amdgpu_buffer_rsrc_t u, dt, z, dout;
    int us, dts, zs, os;
    __device__ RawRows(const ScanArgs &a, int64_t t)    // without z, dout is read in its place
        : u(rows_from<T>(a.u, a.us, t)), dt(rows_from<T>(a.dt, a.dts, t)),
          z(rows_from<T>(a.z ? a.z : a.dout, a.z ? a.zs : a.channels, t)), dout(rows_from<T>(a.dout, a.channels, t)),
          us((int)a.us), dts((int)a.dts), zs((int)(a.z ? a.zs : a.channels)), os(a.channels) {}
    __device__ Raw load(uint32_t lane, int row) const {
        const int r = row * (int)sizeof(T);
        return {row_load<T>(u, lane, r * us), row_load<T>(dt, lane, r * dts), row_load<T>(z, lane, r * zs),
                row_load<T>(dout, lane, r * os)};
    }
};

// dJ/d(state before each chunk but a sequence's first), from 0 behind it, and the
// chunk's summed step sizes.
template <class T, class BC, int S>
__global__ __launch_bounds__(64) void k_scan_back(ScanArgs a) {
    __shared__ float in[kBatch][2][64];                 // s, p
    const uint32_t block = block_index();
    const int me = threadIdx.x;
    const ScanChannels where(a, (int)(block % a.blocks), me);
    const int64_t slot = block / a.blocks;
    if (slot >= a.chunks) return;
    const Seqs seqs{a.off, a.n, a.tokens, a.even};
    ScanChunk chunk = scan_chunk_of(a, seqs, slot);
    if (chunk.seq < 0 || chunk.first) return;
    chunk.begin = __builtin_amdgcn_readfirstlane(chunk.begin), chunk.len = __builtin_amdgcn_readfirstlane(chunk.len);
    const int c = where.c;
    float decay[S], g[S];
#pragma unroll
    for (int q = 0; q < S / kStates; ++q) {
        const f32x4 d = load_decay(a, c, q * kStates);
#pragma unroll
        for (int i = 0; i < kStates; ++i) decay[q * kStates + i] = d[i], g[q * kStates + i] = 0.f;
    }
    const float bias = a.dt_bias ? a.dt_bias[c] : 0.f;
    const uint32_t lane = (uint32_t)c * sizeof(T);
    float total = 0.f;
    Raw raw[kBatch];
    const auto fetch = [&](int t0) {
        const RawRows<T> rows(a, chunk.begin + t0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) raw[i] = rows.load(lane, min(i, chunk.len - t0 - 1));
    };
    const int last = (chunk.len - 1) / kBatch * kBatch;
    constexpr int AT = S * sizeof(BC) <= 32 ? 4 : S <= 16 ? 2 : 1;          // tokens whose scalars are there at once
    TokenRows<BC> rows_c(a, 1, where.group, chunk.begin + chunk.len - 1);
    fetch(last);
#pragma unroll
    for (int n = 0; n < S; ++n) decay[n] = finite_decay(decay[n]);
    for (int t0 = last; t0 >= 0; t0 -= kBatch) {
        const int m = min(kBatch, chunk.len - t0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            float s = row_float<T>(raw[i].dt) + bias, p = row_float<T>(raw[i].dout);
            if (a.softplus) s = softplus(s);
            if (a.z) p *= silu(row_float<T>(raw[i].z));
            in[i][0][me] = i < m ? s : 0.f, in[i][1][me] = i < m ? p : 0.f;           // past the end nothing happens
        }
        fetch(max(t0 - kBatch, 0));                     // without a branch, so that nothing waits for it here
#pragma unroll 1
        for (int i = (m + AT - 1) / AT * AT - 1; i >= 0; i -= AT) {
            Scalars<BC, S> cc[AT];
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                cc[k].load(rows_c.at);
                if (i - k < m && t0 + i - k > 0) rows_c.at -= rows_c.stride;
            }
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                const float s = in[i - k][0][me], p = in[i - k][1][me];
#pragma unroll
                for (int n = 0; n < S; ++n) g[n] = __builtin_amdgcn_exp2f(s * decay[n]) * fmaf(cc[k][n], p, g[n]);
                total += s;
            }
        }
    }
#pragma unroll
    for (int q = 0; q < S / kStates; ++q)
        store_own(a, a.ends, chunk.end, c, q, where.live, f32x4{g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]});
    if (where.live) a.sums[chunk.end * a.channels + c] = total;
}

// A block takes 64 channels, wave w of W their states 4 w .. 4 w + 3.  A token is
// loaded, and its results are stored, by one of them.  Two waves a SIMD: at three, the
// states of a tile do not fit the registers.  As many of its tokens' decays as fit too
// stay there for the way back (timed in turn: 8 of 16 286 us; none 300; 10, with a spill, 287).
// Two sizes are off that, and slow for their work.  33 to 64 states (W = 16): sixteen waves
// have 128 registers each, and 98 are put by in 328 bytes of scratch a lane, a tile's states
// among them: 8192 tokens of 2048 channels of 64 states 2454 us, where those of 32 take 580.
// 1 to 4 (W = 1): 33 KB of LDS a wave leave room for one a SIMD, 186 us.
template <class T, int W>
__global__ __launch_bounds__(64 * W, W == 16 ? 4 : 2) void k_scan_bwd(ScanArgs a) {
    // Tokens between barriers: sums of all waves for a whole tile of 64 states are more than the LDS.
    constexpr int PART = W <= 8 ? kTile : kTile / 2;
    constexpr int SAVED = W == 1 || W == 16 ? 0 : W == 2 ? 6 : 8;
    constexpr int OWN = kTile / W, N = kStates * W, THREADS = 64 * W, PER = kTile * N / THREADS;
    __shared__ float in[kTile][5][64];                  // of each token s, u, p, softplus', dout silu'(z)
    __shared__ float sums[W][PART][3][64];              // sum g a k, sum g b and sum c h, by wave
    __shared__ __attribute__((aligned(16))) float sb[kTile][N], sc[kTile][N];
    const uint32_t block = block_index();
    const int cblock = (int)(block % a.blocks), me = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const ScanChannels where(a, cblock, me);
    const int64_t walker = block / a.blocks;
    if (walker >= a.walkers) return;
    const Seqs seqs{a.off, a.n, a.tokens, a.even};
    const int c = where.c;
    f32x4 decay = load_decay(a, c, w * kStates);
    const float bias = a.dt_bias ? a.dt_bias[c] : 0.f, d = a.d ? a.d[c] : 0.f;
    const uint32_t lane = (uint32_t)c * sizeof(T), to_lane = where.live ? lane : kNowhere;
    f32x4 da = {0.f, 0.f, 0.f, 0.f};
    float dd = 0.f, dbias = 0.f;
    for (int64_t slot = walker; slot < a.chunks; slot += a.walkers) {
        ScanChunk chunk = scan_chunk_of(a, seqs, slot);
        if (chunk.seq < 0) continue;
        chunk.begin = __builtin_amdgcn_readfirstlane(chunk.begin), chunk.len = __builtin_amdgcn_readfirstlane(chunk.len);
        f32x4 g = chunk.alone() ? load_states(a, a.dfinal, chunk.seq, c, w * kStates, true)
                                : load_own(a, a.ends, chunk.end, c, w, true);
        const int64_t kept = scan_kept_slot(a, seqs, chunk);
        Raw raw[OWN];
        T raw_b[PER], raw_c[PER];
        f32x4 next_h;
        const auto fetch = [&](int t0) {
            next_h = load_own(a, a.kept, kept + t0 / kTile, c, w, true);
            const RawRows<T> rows(a, chunk.begin + t0);
#pragma unroll
            for (int j = 0; j < OWN; ++j) raw[j] = rows.load(lane, min(w * OWN + j, chunk.len - t0 - 1));
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = threadIdx.x + i * THREADS, n = min(e % N, a.states - 1);
                const int64_t t = chunk.begin + min(t0 + e / N, chunk.len - 1);
                raw_b[i] = static_cast<const T *>(a.b)[t * a.bs + where.group * a.states + n];
                raw_c[i] = static_cast<const T *>(a.c)[t * a.cs + where.group * a.states + n];
            }
        };
        const int last = chunk.len > 0 ? (chunk.len - 1) / kTile * kTile : -1;
        if (last >= 0) fetch(last);
        decay = finite_decay(decay);
        for (int t0 = last; t0 >= 0; t0 -= kTile) {
            const int m = min(kTile, chunk.len - t0);
#pragma unroll
            for (int j = 0; j < OWN; ++j) {
                const int t = w * OWN + j;
                const float r = row_float<T>(raw[j].dt) + bias, z = row_float<T>(raw[j].z);
                float p = row_float<T>(raw[j].dout);
                if (a.z) {
                    const float gate = sigmoid(z);
                    in[t][4][me] = p * gate * fmaf(z, 1.f - gate, 1.f);
                    p *= z * gate;
                }
                // Past the end, and where no channel is, nothing happens.
                const bool live = where.live && t < m;
                in[t][0][me] = t < m ? (a.softplus ? softplus(r) : r) : 0.f;
                in[t][1][me] = live ? row_float<T>(raw[j].u) : 0.f;
                in[t][2][me] = live ? p : 0.f;
                in[t][3][me] = a.softplus ? sigmoid(r) : 1.f;
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = threadIdx.x + i * THREADS, t = e / N, n = e % N;
                const bool there = t < m && n < a.states;
                sb[t][n] = there ? to_float(raw_b[i]) : 0.f, sc[t][n] = there ? to_float(raw_c[i]) : 0.f;
            }
            f32x4 e[kTile];                             // decays of the last SAVED tokens
            f32x4 h[kTile + 1];                         // before each token, and after the last
            h[0] = next_h;
            __syncthreads();
            fetch(max(t0 - kTile, 0));                  // without a branch, so that nothing waits for it here
            // What a token needs is on its way from LDS during the one before.
            struct Token {
                float s, u, p;
                f32x4 b, c;
            };
            const auto token = [&](int t) {
                return Token{in[t][0][me], in[t][1][me], in[t][2][me], *reinterpret_cast<const f32x4 *>(&sb[t][w * kStates]),
                             *reinterpret_cast<const f32x4 *>(&sc[t][w * kStates])};
            };
            Token next = token(0);
#pragma unroll
            for (int t = 0; t < kTile; ++t) {
                const Token now = next;
                next = token(t + 1 < kTile ? t + 1 : t);
                __builtin_amdgcn_sched_barrier(0);
                const float x = now.s * now.u;
#pragma unroll
                for (int i = 0; i < kStates; ++i) {
                    const float now_e = __builtin_amdgcn_exp2f(now.s * decay[i]);
                    if (t >= kTile - SAVED) e[t][i] = now_e;
                    h[t + 1][i] = fmaf(x, now.b[i], now_e * h[t][i]);
                }
            }
            const auto part_bc = rows_from<float>(a.part_bc, 2 * a.states, (int64_t)cblock * a.tokens + chunk.begin + t0);
#pragma unroll
            for (int part = kTile - PART; part >= 0; part -= PART) {
#pragma unroll
                for (int t2 = part + PART - 2; t2 >= part; t2 -= 2) {
                    float v[16];                            // [token][db, dc][state]
#pragma unroll
                    for (int t = t2 + 1; t >= t2; --t) {
                        const Token now = next;
                        if (t > 0) next = token(t - 1);
                        __builtin_amdgcn_sched_barrier(0);
                        const float st = now.s, x = st * now.u, pt = now.p;
                        const f32x4 b = now.b, cc = now.c;
                        float *o = v + (t - t2) * 8, ak = 0.f, gb = 0.f, y = 0.f;
#pragma unroll
                        for (int i = 0; i < kStates; ++i) {
                            const float te = t >= kTile - SAVED ? e[t][i] : __builtin_amdgcn_exp2f(st * decay[i]);
                            g[i] = fmaf(cc[i], pt, g[i]);
                            const float gk = g[i] * (te * h[t][i]);
                            ak = fmaf(gk, decay[i], ak);
                            da[i] = fmaf(gk, st, da[i]);
                            gb = fmaf(b[i], g[i], gb);
                            y = fmaf(cc[i], h[t + 1][i], y);
                            o[i] = g[i] * x;
                            o[4 + i] = h[t + 1][i] * pt;
                            g[i] *= te;
                        }
                        sums[w][t - part][0][me] = ak, sums[w][t - part][1][me] = gb;
                        sums[w][t - part][2][me] = y;
                    }
                    const float r = over_channels(v);
                    const int t = t2 + me / 32, n = w * kStates + me / 4 % 4;
                    const bool there = me % 4 == 0 && t < m && n < a.states;
                    row_store<float>(part_bc, there ? ((t * 2 + me / 16 % 2) * a.states + n) * 4 : kNowhere, 0, r);
                }
                __syncthreads();
                const int64_t first = chunk.begin + t0;
                const auto du = rows_from<T>(a.du, a.channels, first), ddt = rows_from<T>(a.ddt, a.channels, first);
                const auto dz = rows_from<T>(a.dz, a.channels, first);
#pragma unroll
                for (int j = 0; j < OWN; ++j) {
                    const int t = w * OWN + j;
                    if (t < part || t >= part + PART) continue;     // a wave's one token, where there are two parts
                    const uint32_t to = t < m ? to_lane : kNowhere;
                    float ak = 0.f, gb = 0.f, y = 0.f;
#pragma unroll
                    for (int k = 0; k < W; ++k) {
                        ak += sums[k][t - part][0][me], gb += sums[k][t - part][1][me];
                        y += sums[k][t - part][2][me];
                    }
                    const float ut = in[t][1][me], pt = in[t][2][me], dr = fmaf(ut, gb, ak * kLn2) * in[t][3][me];
                    dd = fmaf(pt, ut, dd), dbias += t < m ? dr : 0.f;
                    const int at = t * a.channels * (int)sizeof(T);
                    row_store<T>(du, to, at, from_float<T>(fmaf(in[t][0][me], gb, d * pt)));
                    row_store<T>(ddt, to, at, from_float<T>(dr));
                    row_store<T>(dz, a.dz ? to : kNowhere, at, from_float<T>(in[t][4][me] * fmaf(d, ut, y)));
                }
                if (part) __syncthreads();              // sums is written again; behind the last part the next tile's barrier is
            }
        }
        if (chunk.first) store_states(a, a.dstate, chunk.seq, c, w * kStates, where.live, g);
    }
    store_states(a, a.part_a, walker, c, w * kStates, where.live, da);
    __syncthreads();
    in[w % kTile][0][me] = dd, in[w % kTile][1][me] = dbias;
    __syncthreads();
    if (w < 2 && where.live)
        for (int kind = w; kind < 2; kind += W < 2 ? W : 2) {
            float v = 0.f;
            for (int k = 0; k < W; ++k) v += in[k][kind][me];
            a.part_d[(walker * 2 + kind) * a.channels + c] = v;
        }
}

// Sums over blocks, each in a fixed order: of da by the first blocks, of dd and the bias'
// gradient by the next, of db and dc by the rest.  One kernel: 256 episodes of 16 tokens
// 68 us in place of 76 with one each.
template <class T>
__global__ __launch_bounds__(1024) void k_scan_sums(ScanArgs a, uint32_t of_a, uint32_t of_d) {
    const uint32_t block = block_index();
    if (block < of_a) {
        column_sums(a.part_a, (int64_t)a.channels * a.states, (int)a.walkers, block, [&](int64_t c, float v) { a.da[c] = v; });
        return;
    }
    if (block < of_a + of_d) {
        column_sums(a.part_d, (int64_t)2 * a.channels, (int)a.walkers, block - of_a, [&](int64_t c, float v) {
            float *to = c < a.channels ? a.dd : a.ddt_bias;
            if (to) to[c < a.channels ? c : c - a.channels] = v;
        });
        return;
    }
    const int64_t per = (int64_t)a.groups * a.states, i = (int64_t)(block - of_a - of_d) * 1024 + threadIdx.x;
    if (i >= 2 * per * a.tokens) return;
    const int n = (int)(i % a.states), group = (int)(i / a.states % a.groups), kind = (int)(i / per % 2);
    const int64_t t = i / per / 2;
    const Seqs seqs{a.off, a.n, a.tokens, a.even};
    if (t < seqs.offset(0) || t >= seqs.offset(a.n)) return;    // no sequence's
    const int64_t of = a.blocks / a.groups;
    const float *p = a.part_bc + ((group * of * a.tokens + t) * 2 + kind) * a.states + n;
    const int64_t on = a.tokens * 2 * a.states;
    float v = 0.f;
#pragma unroll 8
    for (int64_t k = 0; k < of; ++k) v += p[k * on];
    static_cast<T *>(kind ? a.dc : a.db)[t * per + group * a.states + n] = from_float<T>(v);
}

template <class T>
hipError_t backward(const ScanArgs &a, hipStream_t s) {
    hipError_t e = hipSuccess;
    const bool direct = scan_direct(a, sizeof(T) == 2);
    if (a.parts && !direct) e = launch_scan_pack(a, sizeof(T) == 2, s);
    if (e) return e;
    for_states(a.states, [&](auto states) {
        constexpr int S = decltype(states)::value;
        const dim3 grid = grid_of(a.blocks * a.chunks);
        if (a.parts) {
            if (direct) k_scan_back<T, T, S><<<grid, 64, 0, s>>>(a);
            else k_scan_back<T, Packed, S><<<grid, 64, 0, s>>>(a);
            e = launch_scan_join_back(a, s);
        }
        k_scan_bwd<T, S / kStates><<<grid_of(a.blocks * a.walkers), 64 * (S / kStates), 0, s>>>(a);
    });
    if (e) return e;
    if ((e = hipGetLastError())) return e;
    const int64_t of_a = column_blocks((int64_t)a.channels * a.states);
    const int64_t of_d = a.dd || a.ddt_bias ? column_blocks((int64_t)2 * a.channels) : 0;
    const int64_t of_bc = (2 * a.tokens * a.groups * a.states + 1023) / 1024;
    k_scan_sums<T><<<grid_of(of_a + of_d + of_bc), 1024, 0, s>>>(a, (uint32_t)of_a, (uint32_t)of_d);
    return hipGetLastError();
}

}  // namespace

// Blocks over the chunks, each of which has a part of da, dd and the bias' gradient.
int64_t scan_walkers(int64_t chunks, int64_t blocks) {
    const int64_t w = (4096 + blocks - 1) / blocks;
    return chunks < w ? (chunks > 0 ? chunks : 1) : w;
}

hipError_t launch_scan_backward(const ScanArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? backward<bf16_t>(a, s) : backward<float>(a, s);
}

}  // namespace rn
