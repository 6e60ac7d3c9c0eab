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
// Bound by its arithmetic: for each token, channel and state two exponentials, 14
// multiplications or multiply-adds, and a sixth of that again for the sums over
// channels: those of a wave in registers (sum_channels), of a block in LDS, of all
// blocks by another kernel, each in a fixed order.
#include "rn_rows.hpp"
#include "rn_scan.hpp"

namespace rn {
namespace {

using namespace ops;

// 32 values a lane, summed over the lanes of a wave that carry other channels (lane
// bits log2(L)..5).  Every step joins two lanes: each keeps half of the values that
// both have.  Then lane l has value i of all channels at v[i & (R - 1)], R = 32 / (64 / L),
// for those i whose upper bits are its own channel bits, the highest first.
template <int BIT>
__device__ inline float exchange(float a, float b) {    // lanes without the bit: a of both, with it: b of both
    if constexpr (BIT == 5 || BIT == 4) {
        const auto r = BIT == 5
            ? __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false)
            : __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        const bool up = threadIdx.x >> BIT & 1;
        const float keep = up ? b : a, give = up ? a : b;
        if constexpr (BIT == 3) return keep + dpp<0x128>(give);                 // 8 on in a row of 16
        else if constexpr (BIT == 2) return keep + __shfl_xor(give, 4);
        else if constexpr (BIT == 1) return keep + dpp<0x4e>(give);
        else return keep + dpp<0xb1>(give);
    }
}
template <int L, int BIT = 5, int COUNT = 32>
__device__ inline void sum_channels(float (&v)[32]) {
    if constexpr ((1 << BIT) >= L && COUNT > 1) {
#pragma unroll
        for (int i = 0; i < COUNT / 2; ++i) v[i] = exchange<BIT>(v[i], v[i + COUNT / 2]);
        if constexpr (BIT > 0) sum_channels<L, BIT - 1, COUNT / 2>(v);
    } else if constexpr ((1 << BIT) >= L) {             // one value left: of both lanes
        v[0] += dpp<0xb1>(v[0]);
    }
}

// What a quad of channels is at a token, as loaded.
template <class T>
struct Raw {
    Pack<T, 4> u, dt, z, dout;
};

template <class T>
__device__ inline Raw<T> load_raw(const ScanArgs &a, int64_t t, int c, int c1) {
    Raw<T> r;
    r.u = load_quad<T>(a, a.u, a.us, t, c, c1);
    r.dt = load_quad<T>(a, a.dt, a.dts, t, c, c1);
    r.dout = load_quad<T>(a, a.dout, a.channels, t, c, c1);
    if (a.z) r.z = load_quad<T>(a, a.z, a.zs, t, c, c1);
    return r;
}

// dJ/d(state before each chunk but a sequence's first), from 0 behind it, and the
// chunk's summed step sizes.
template <class T, int L>
__global__ __launch_bounds__(kScanThreads) void k_scan_back(ScanArgs a) {
    constexpr int N = kStates * L, CB = ScanBlock<L>::CB;
    using Q = Quads<L>;
    __shared__ float in[kTile][CB][2];                  // s, p
    __shared__ __attribute__((aligned(16))) float sb[kTile][N], sc[kTile][N];
    const uint32_t block = block_index();
    const ScanBlock<L> where(a, (int)(block % a.blocks));
    const int64_t slot = block / a.blocks;
    if (slot >= a.chunks) return;
    const Seqs seqs{a.off, a.n, a.tokens};
    const ScanChunk chunk = scan_chunk_of(a, seqs, slot);
    if (chunk.seq < 0 || chunk.first) return;
    const int lane = threadIdx.x % L, mine = threadIdx.x / L, c = where.c0 + mine;
    const bool live = c < where.c1;
    const f32x4 decay = load_states(a, a.a, 0, c, lane * kStates, live) * kLog2e;
    f32x4 g = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    const int q0 = where.c0 + Q::channel();
    const bool there = q0 < where.c1 && Q::row(0) < kTile;
    float bias[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) bias[j] = there && q0 + j < where.c1 && a.dt_bias ? a.dt_bias[q0 + j] : 0.f;
    Raw<T> raw[Q::PER];
    TileBC<T, L> bc;
    const auto fetch = [&](int t0) {
        bc.load(a, where.group, chunk.begin + t0, chunk.len - t0);
        if (!there) return;
#pragma unroll
        for (int i = 0; i < Q::PER; ++i)
            raw[i] = load_raw<T>(a, chunk.begin + min(t0 + Q::row(i), chunk.len - 1), q0, where.c1);
    };
    const int last = (chunk.len - 1) / kTile * kTile;
    fetch(last);
    for (int t0 = last; t0 >= 0; t0 -= kTile) {
        __syncthreads();                                // the last tile has been read
        bc.store(a, chunk.len - t0, sb, sc);
#pragma unroll
        for (int i = 0; i < Q::PER; ++i) {
            const int t = Q::row(i);
            if (t >= kTile) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float s = 0.f, p = 0.f;
                if (there && t0 + t < chunk.len && q0 + j < where.c1) {
                    s = to_float(raw[i].dt.v[j]) + bias[j];
                    if (a.softplus) s = softplus(s);
                    p = to_float(raw[i].dout.v[j]);
                    if (a.z) p *= silu(to_float(raw[i].z.v[j]));
                }
                in[t][Q::channel() + j][0] = s;
                in[t][Q::channel() + j][1] = p;
            }
        }
        __syncthreads();
        if (t0 > 0) fetch(t0 - kTile);
#pragma unroll
        for (int t = kTile - 1; t >= 0; --t) {
            const float s = in[t][mine][0], p = in[t][mine][1];
            const f32x4 cc = *reinterpret_cast<const f32x4 *>(&sc[t][lane * kStates]);
#pragma unroll
            for (int i = 0; i < kStates; ++i) g[i] = __builtin_amdgcn_exp2f(s * decay[i]) * fmaf(cc[i], p, g[i]);
            total += s;
        }
    }
    store_own(a, a.ends, chunk.end, c, lane, live, g);
    if (live && lane == 0) a.sums[chunk.end * a.channels + c] = total;
}

template <class T, int L>
__global__ __launch_bounds__(kScanThreads, 2) void k_scan_bwd(ScanArgs a) {
    constexpr int N = kStates * L, CB = ScanBlock<L>::CB, WAVES = kScanThreads / 64;
    using Q = Quads<L>;
    // s, u and p of each token and channel; a channel's lanes, which are one wave's,
    // replace them by sum g a k, sum g b and sum c h when they are done with a token.
    __shared__ float io[kTile][3][CB];
    __shared__ __attribute__((aligned(16))) float sb[kTile][N], sc[kTile][N];
    __shared__ __attribute__((aligned(16))) float sums[WAVES][kTile][2][N];    // of db and dc, by wave
    const uint32_t block = block_index();
    const int cblock = (int)(block % a.blocks);
    const ScanBlock<L> where(a, cblock);
    const int64_t walker = block / a.blocks;
    if (walker >= a.walkers) return;
    const Seqs seqs{a.off, a.n, a.tokens};
    const int lane = threadIdx.x % L, mine = threadIdx.x / L, c = where.c0 + mine, wave = threadIdx.x / 64;
    const bool live = c < where.c1;
    const f32x4 decay = load_states(a, a.a, 0, c, lane * kStates, live) * kLog2e;
    f32x4 da = {0.f, 0.f, 0.f, 0.f};
    const int q0 = where.c0 + Q::channel();
    const bool there = q0 < where.c1 && Q::row(0) < kTile;
    float bias[4], d[4], dd[4], dbias[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool in = there && q0 + j < where.c1;
        bias[j] = in && a.dt_bias ? a.dt_bias[q0 + j] : 0.f;
        d[j] = in && a.d ? a.d[q0 + j] : 0.f;
        dd[j] = dbias[j] = 0.f;
    }
    for (int64_t slot = walker; slot < a.chunks; slot += a.walkers) {
        const ScanChunk chunk = scan_chunk_of(a, seqs, slot);
        if (chunk.seq < 0) continue;
        f32x4 g = chunk.alone() ? load_states(a, a.dfinal, chunk.seq, c, lane * kStates, live)
                                : load_own(a, a.ends, chunk.end, c, lane, live);
        const int64_t kept = scan_kept_slot(a, seqs, chunk);
        Raw<T> raw[Q::PER], next[Q::PER];
        TileBC<T, L> bc;
        f32x4 next_h;
        const auto fetch = [&](int t0) {
            bc.load(a, where.group, chunk.begin + t0, chunk.len - t0);
            next_h = load_own(a, a.kept, kept + t0 / kTile, c, lane, live);
            if (!there) return;
#pragma unroll
            for (int i = 0; i < Q::PER; ++i)
                next[i] = load_raw<T>(a, chunk.begin + min(t0 + Q::row(i), chunk.len - 1), q0, where.c1);
        };
        const int last = chunk.len > 0 ? (chunk.len - 1) / kTile * kTile : -1;
        if (last >= 0) fetch(last);
        for (int t0 = last; t0 >= 0; t0 -= kTile) {
            bc.store(a, chunk.len - t0, sb, sc);
#pragma unroll
            for (int i = 0; i < Q::PER; ++i) {
                raw[i] = next[i];
                const int t = Q::row(i);
                if (t >= kTile) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float s = 0.f, u = 0.f, p = 0.f;
                    if (there && t0 + t < chunk.len && q0 + j < where.c1) {
                        s = to_float(raw[i].dt.v[j]) + bias[j];
                        if (a.softplus) s = softplus(s);
                        u = to_float(raw[i].u.v[j]);
                        p = to_float(raw[i].dout.v[j]);
                        if (a.z) p *= silu(to_float(raw[i].z.v[j]));
                    }
                    io[t][0][Q::channel() + j] = s, io[t][1][Q::channel() + j] = u, io[t][2][Q::channel() + j] = p;
                }
            }
            f32x4 h[kTile + 1];                         // before each token, and after the last
            h[0] = next_h;
            __syncthreads();
            if (t0 > 0) fetch(t0 - kTile);
            float kept_y[kTile / L > 0 ? kTile / L : 1];
#pragma unroll
            for (int t = 0; t < kTile; ++t) {
                const float s = io[t][0][mine], x = s * io[t][1][mine];
                const f32x4 b = *reinterpret_cast<const f32x4 *>(&sb[t][lane * kStates]);
#pragma unroll
                for (int i = 0; i < kStates; ++i)
                    h[t + 1][i] = fmaf(x, b[i], __builtin_amdgcn_exp2f(s * decay[i]) * h[t][i]);
                if (a.z) {
                    const f32x4 cc = *reinterpret_cast<const f32x4 *>(&sc[t][lane * kStates]);
                    float y = 0.f;
#pragma unroll
                    for (int i = 0; i < kStates; ++i) y = fmaf(cc[i], h[t + 1][i], y);
                    y = over_states<L>(y);
                    kept_y[t / L] = t % L == 0 || lane == t % L ? y : kept_y[t / L];
                }
            }
#pragma unroll
            for (int t4 = kTile - 4; t4 >= 0; t4 -= 4) {
                float v[32];                            // [token][db, dc][state]
                float ak[4], gb[4];
#pragma unroll
                for (int t = t4 + 3; t >= t4; --t) {
                    const float s = io[t][0][mine], x = s * io[t][1][mine], p = io[t][2][mine];
                    const f32x4 b = *reinterpret_cast<const f32x4 *>(&sb[t][lane * kStates]);
                    const f32x4 cc = *reinterpret_cast<const f32x4 *>(&sc[t][lane * kStates]);
                    float *o = v + (t - t4) * 8;
                    float sum_ak = 0.f, sum_gb = 0.f;
#pragma unroll
                    for (int i = 0; i < kStates; ++i) {
                        const float e = __builtin_amdgcn_exp2f(s * decay[i]);
                        g[i] = fmaf(cc[i], p, g[i]);
                        const float gk = g[i] * (e * h[t][i]);
                        sum_ak = fmaf(gk, decay[i], sum_ak);
                        da[i] = fmaf(gk, s, da[i]);
                        sum_gb = fmaf(g[i], b[i], sum_gb);
                        o[i] = g[i] * x;
                        o[4 + i] = h[t + 1][i] * p;
                        g[i] *= e;
                    }
                    ak[t - t4] = over_states<L>(sum_ak), gb[t - t4] = over_states<L>(sum_gb);
                }
                sum_channels<L>(v);
                // Lane bits 5 and 4 are the token's where the channels have them (L <= 16).
                {
                    constexpr int R = L >= 2 ? L / 2 : 1;               // values a lane has now
                    const int at = ((threadIdx.x & 63) / (L > 2 ? L : 2)) * R;
                    float *to = &sums[wave][t4][0][0];
                    // Value at + i is [token][kind][state].
                    if constexpr (R >= 4) {
#pragma unroll
                        for (int i = 0; i < R; i += 4)
                            *reinterpret_cast<f32x4 *>(to + (at + i) / 4 * N + lane * kStates) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
                    } else {
#pragma unroll
                        for (int i = 0; i < R; ++i) to[(at + i) / 4 * N + lane * kStates + (at + i) % 4] = v[i];
                    }
                }
                // Lanes of a channel write the tokens' sums in turn, over what they have all read.
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (lane == t % L) {
                        io[t4 + t][0][mine] = ak[t] * kLn2;
                        io[t4 + t][1][mine] = gb[t];
                    }
            }
            if (a.z) {
#pragma unroll
                for (int i = 0; i < (kTile / L > 0 ? kTile / L : 1); ++i)
                    if (L <= kTile) io[i * L + lane][2][mine] = kept_y[i];
            }
            __syncthreads();
            if (there) {
#pragma unroll
                for (int i = 0; i < Q::PER; ++i) {
                    const int t = Q::row(i);
                    if (t >= kTile || t0 + t >= chunk.len) continue;
                    float du[4], ddt[4], dz[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float r = to_float(raw[i].dt.v[j]) + bias[j], s = a.softplus ? softplus(r) : r;
                        const float u = to_float(raw[i].u.v[j]), out = to_float(raw[i].dout.v[j]);
                        float p = out;
                        const float sum_gb = io[t][1][Q::channel() + j];
                        if (a.z) {
                            const float z = to_float(raw[i].z.v[j]);
                            dz[j] = out * fmaf(d[j], u, io[t][2][Q::channel() + j]) * silu_slope(z);
                            p *= silu(z);
                        }
                        du[j] = fmaf(s, sum_gb, d[j] * p);
                        ddt[j] = fmaf(u, sum_gb, io[t][0][Q::channel() + j]);
                        if (a.softplus) ddt[j] *= sigmoid(r);
                        if (q0 + j < where.c1) dd[j] = fmaf(p, u, dd[j]), dbias[j] += ddt[j];
                    }
                    const int64_t at = chunk.begin + t0 + t;
                    store_quad<T>(a, a.du, at, q0, where.c1, du);
                    store_quad<T>(a, a.ddt, at, q0, where.c1, ddt);
                    if (a.dz) store_quad<T>(a, a.dz, at, q0, where.c1, dz);
                }
            }
            for (int i = threadIdx.x; i < kTile * 2 * N; i += kScanThreads) {
                const int t = i / (2 * N), n = i % N;
                if (t0 + t >= chunk.len || n >= a.states) continue;
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) v += (&sums[w][0][0][0])[i];
                a.part_bc[(((int64_t)cblock * a.tokens + chunk.begin + t0 + t) * 2 + i / N % 2) * a.states + n] = v;
            }
        }
        if (chunk.first) store_states(a, a.dstate, chunk.seq, c, lane * kStates, live, g);
    }
    store_states(a, a.part_a, walker, c, lane * kStates, live, da);
    // dd and dbias: the quads of a channel are in threads ACROSS apart.
    float *last = &io[0][0][0];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (Q::row(0) < kTile) last[threadIdx.x * 8 + j] = dd[j], last[threadIdx.x * 8 + 4 + j] = dbias[j];
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * CB; i += kScanThreads) {
        const int ch = i % CB, kind = i / CB;
        if (where.c0 + ch >= where.c1) continue;
        float v = 0.f;
        for (int r = 0; r < (Q::ROWS < kTile ? Q::ROWS : kTile); ++r) v += last[(r * Q::ACROSS + ch / 4) * 8 + kind * 4 + ch % 4];
        a.part_d[(walker * 2 + kind) * a.channels + where.c0 + ch] = v;
    }
}

// db and dc of the blocks of a group's channels, in a fixed order.
template <class T>
__global__ __launch_bounds__(kScanThreads) void k_scan_bc(ScanArgs a) {
    const int64_t per = (int64_t)a.groups * a.states, i = (int64_t)block_index() * kScanThreads + threadIdx.x;
    if (i >= 2 * per * a.tokens) return;
    const int n = (int)(i % a.states), group = (int)(i / a.states % a.groups), kind = (int)(i / per % 2);
    const int64_t t = i / per / 2;
    const int64_t of = a.blocks / a.groups;
    const float *p = a.part_bc + ((group * of * a.tokens + t) * 2 + kind) * a.states + n;
    const int64_t on = a.tokens * 2 * a.states;
    float v = 0.f;
    for (int64_t k = 0; k < of; ++k) v += p[k * on];
    static_cast<T *>(kind ? a.dc : a.db)[t * per + group * a.states + n] = from_float<T>(v);
}

__global__ __launch_bounds__(1024) void k_scan_sum_a(ScanArgs a) {
    column_sums(a.part_a, (int64_t)a.channels * a.states, (int)a.walkers, [&](int64_t c, float v) { a.da[c] = v; });
}
__global__ __launch_bounds__(1024) void k_scan_sum_d(ScanArgs a) {
    column_sums(a.part_d, (int64_t)2 * a.channels, (int)a.walkers, [&](int64_t c, float v) {
        float *to = c < a.channels ? a.dd : a.ddt_bias;
        if (to) to[c < a.channels ? c : c - a.channels] = v;
    });
}

template <class T>
hipError_t backward(const ScanArgs &a, hipStream_t s) {
    for_lanes_of(a.states, [&](auto l) {
        constexpr int L = decltype(l)::value;
        if (a.parts) {
            k_scan_back<T, L><<<grid_of(a.blocks * a.chunks), kScanThreads, 0, s>>>(a);
            (void)launch_scan_join_back(a, s);
        }
        k_scan_bwd<T, L><<<grid_of(a.blocks * a.walkers), kScanThreads, 0, s>>>(a);
    });
    if (hipError_t e = hipGetLastError()) return e;
    if (a.tokens > 0)
        k_scan_bc<T><<<grid_of((2 * a.tokens * a.groups * a.states + kScanThreads - 1) / kScanThreads), kScanThreads, 0, s>>>(a);
    k_scan_sum_a<<<column_grid((int64_t)a.channels * a.states), 1024, 0, s>>>(a);
    if (a.dd || a.ddt_bias) k_scan_sum_d<<<column_grid((int64_t)2 * a.channels), 1024, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

// Blocks over the chunks, each of which has a part of da, dd and the bias' gradient.
int64_t scan_walkers(int64_t chunks, int64_t blocks) {
    const int64_t w = (2048 + blocks - 1) / blocks;
    return chunks < w ? (chunks > 0 ? chunks : 1) : w;
}

hipError_t launch_scan_backward(const ScanArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? backward<bf16_t>(a, s) : backward<float>(a, s);
}

}  // namespace rn
