// Sampling with temperature, top-k, min-p and top-p from given random numbers.
//
// With m a row's largest logit and c = log2(e) / temperature,
//   w_i = rint(2^31 2^((l_i - m) c)),
// whole numbers, so that sums over them are exact and do not depend on their
// order: parallel sums and histograms by atomics give the answer of the
// definition, bit by bit.  2^31 leaves room for 2^22 of them in a double's 53
// bits; the last bit of a weight is 2^-31 of the largest logit's share.  The
// filters keep a prefix of the logits in descending order (equal ones by
// index), so each is a threshold: a logit, and how many of its equals stay.
#include "rn_ops.hpp"

namespace rn {
namespace {

using namespace ops;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kOne = 0x1p31f;
constexpr float kInf = __builtin_huge_valf();

// A row's settings, resolved.
struct Row {
    bool greedy;
    float c, min_p, top_p;
    int top_k;                    // 0: all
};

__device__ inline Row row_settings(const rn_sample_params &p, uint32_t r) {
    Row q;
    const float t = p.dev_temperature ? p.dev_temperature[r] : p.temperature;
    q.c = kLog2e / t;
    q.greedy = !(t > 0.f) || !(q.c * 32.f < kInf);
    const int k = p.dev_top_k ? p.dev_top_k[r] : p.top_k;
    q.top_k = k > 0 ? k : 0;
    const float tp = p.dev_top_p ? p.dev_top_p[r] : p.top_p;
    q.top_p = tp > 0.f ? tp : 0.f;
    const float mp = p.dev_min_p ? p.dev_min_p[r] : p.min_p;
    q.min_p = mp > 0.f ? fminf(mp, 1.f) : 0.f;
    return q;
}

// NaN counts as -infinity, -0 as +0, so that order and equality are those of the key.
__device__ inline float canonical(float l) { return l == l ? l + 0.f : -kInf; }
// Bfloat16's keys have 16 bits, for their lower half would tell nothing.
template <class T>
__device__ inline uint32_t key_of(float l) {
    const uint32_t b = __float_as_uint(canonical(l));
    return (b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u)) >> (32 - 8 * sizeof(T));
}
template <class T>
__device__ inline float of_key(uint32_t k) {
    if (sizeof(T) == 2) k = k << 16 | (k & 0x8000u ? 0u : 0xffffu);
    return __uint_as_float(k ^ ((int32_t)k < 0 ? 0x80000000u : 0xffffffffu));
}

// log2 of the weight's share of the largest, exactly as rounded in float32.
// With a largest logit of +infinity its equals have share 1, the rest none.
__device__ inline float z_of(float l, float m, float c) {
    if (m == kInf) return l == kInf ? 0.f : -kInf;
    return (l - m) * c;
}
// Below z = -33 a weight rounds to 0 (and the hardware's exp2, exact in its
// normal range, would meet denormals).
__device__ inline uint32_t weight_of(float z, float min_p) {
    if (!(z > -33.f)) return 0;
    const float e = __builtin_amdgcn_exp2f(z);
    return e >= min_p ? (uint32_t)rintf(e * kOne) : 0;
}
__device__ inline float log_share(float z, uint64_t total) {
    return (z - log2f((float)((double)total * 0x1p-31))) * kLn2;
}
// floor(u total), below total.
__device__ inline uint64_t target_of(float u, uint64_t total) {
    const double t = (double)u * (double)total;
    if (!(t > 0.0)) return 0;
    return t < (double)total ? min((uint64_t)t, total - 1) : total - 1;
}

__device__ inline uint64_t shfl_up64(uint64_t v, int d) { return __shfl_up((unsigned long long)v, d); }
__device__ inline uint64_t shfl_xor64(uint64_t v, int d) { return __shfl_xor((unsigned long long)v, d); }
__device__ inline uint64_t shfl64(uint64_t v, int s) { return __shfl((unsigned long long)v, s); }
__device__ inline uint64_t wave_sum(uint64_t v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += shfl_xor64(v, d);
    return v;
}
__device__ inline uint32_t wave_scan32(uint32_t v) {    // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t t = __shfl_up(v, d);
        if (lane >= d) v += t;
    }
    return v;
}
__device__ inline uint64_t wave_scan(uint64_t v) {      // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t t = shfl_up64(v, d);
        if (lane >= d) v += t;
    }
    return v;
}

// ------------------------------------------------------------------ up to 64 choices

// One wave a row, one lane a choice.  Each lane counts the choices before its
// own in descending order and adds their weights in one walk over the row, whose
// keys and weights the wave broadcasts from its registers: no sort, no LDS.  Bound by
// that walk: 1024 rows of 18 in 4.9 us.
template <class T>
__global__ __launch_bounds__(256) void k_sample_wave(SampleArgs a) {
    const uint32_t r = block_index() * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (r >= (uint32_t)a.n) return;
    const Row q = row_settings(a.p, r);
    const bool live = lane < a.vocab;
    const float l = live ? to_float(static_cast<const T *>(a.logits)[r * a.stride + lane]) : -kInf;
    float m = l;
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    int token = -1;
    float logp = -kInf;
    if (m > -kInf) {
        if (q.greedy) {
            token = __ffsll((unsigned long long)__ballot(live && l == m)) - 1;
            logp = 0.f;
        } else {
            const float z = z_of(l, m, q.c);
            const uint32_t w = live ? weight_of(z, q.min_p) : 0, key = live ? key_of<T>(l) : 0;
            int rank = 0;
            uint64_t before = 0;
            for (int j = 0; j < a.vocab; ++j) {
                const uint32_t kj = __builtin_amdgcn_readlane(key, j), wj = __builtin_amdgcn_readlane(w, j);
                const bool ahead = kj > key || (kj == key && j < lane);
                rank += ahead;
                before += ahead ? wj : 0;
            }
            const bool in_k = q.top_k == 0 || rank < q.top_k;
            const double limit = (double)q.top_p * (double)wave_sum(in_k ? w : 0);
            const uint64_t mine = in_k && (rank == 0 || (double)before < limit) ? w : 0;
            const uint64_t upto = wave_scan(mine), total = shfl64(upto, 63);
            const uint64_t t = target_of(a.u[r], total);
            token = __ffsll((unsigned long long)__ballot(upto > t)) - 1;
            logp = log_share(__shfl(z, token), total);
        }
    }
    if (lane == 0) {
        a.tokens[r] = token;
        if (a.logprobs) a.logprobs[r] = logp;
    }
}

// ------------------------------------------------------------------ more choices

constexpr int kBins = 1024;

// One block of NT threads a row, which is streamed (from the caches after the first
// time) once for each question asked of it:
//   the largest logit;
//   the histogram of z in steps of 1/32 (counts for top-k and min-p, weights for
//     top-p), which gives the bin a threshold lies in.
// Where kPairs logits or fewer lie down to that bin they are put into a list, and
// each thread compares one of them with all others: no further reading.  (The
// list's order is that of an atomic counter and changes; nothing computed from it
// does.)  Otherwise
//   histograms of the keys within the bin, 1024 steps at a time, until a step is
//     one key: one or two more;
//   the weights that stay, by contiguous parts of the row, then of the part the
//     draw falls into, down to one wave's vector.
//
// One CU works on a row, so a reading is bound by what it has in flight: four
// vectors a thread are on their way while one is looked at (256 rows of 131072
// bfloat16: 12 us for the first reading without, 7
// with; with six the whole call is 4 us slower, for the registers it takes).  Those
// rows take 87 us, 0.8 TB/s: four readings from the caches where the list is too
// short, in the longest of them two LDS atomics an element.
constexpr int kPairs = 512;

template <class T, int VEC, int NT>
struct Block {
    static constexpr int NW = NT / 64, kAhead = 4;
    const T *x;
    int vocab;
    uint64_t (&hw)[kBins];
    uint32_t (&hc)[kBins];
    uint64_t (&part)[NW + 2];
    uint32_t (&ties)[NW + 2];
    int &bin;

    // f(index, logit) for the elements [lo, hi), thread by thread in vectors.  Logits
    // come as they are: NaN fails every comparison below, and has no weight.
    template <class F>
    __device__ __forceinline__ void each(int lo, int hi, int first, int step, F &&f) const {
        using P = Pack<T, VEC>;
        const int stride = step * VEC;
        int i = lo + first * VEC;
        P p[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u * stride + VEC <= hi) p[u] = *reinterpret_cast<const P *>(x + i + u * stride);
        for (; i + VEC <= hi; i += stride) {
            const P now = p[0];
#pragma unroll
            for (int u = 0; u + 1 < kAhead; ++u) p[u] = p[u + 1];
            if (i + kAhead * stride + VEC <= hi) p[kAhead - 1] = *reinterpret_cast<const P *>(x + i + kAhead * stride);
#pragma unroll
            for (int j = 0; j < VEC; ++j) f(i + j, to_float(now.v[j]));
        }
        for (; i < hi; ++i) f(i, to_float(x[i]));      // a last vector's part: one thread's
    }
    template <class F>
    __device__ __forceinline__ void all(F &&f) const { each(0, vocab, threadIdx.x, NT, f); }

    __device__ void clear() const {
        for (int i = threadIdx.x; i < kBins; i += NT) hw[i] = 0, hc[i] = 0;
        __syncthreads();
    }

    // The first bin at which `upto(before count, before weight, count, weight)`
    // holds of the bins in order, and what lies before it; kBins if there is none.
    struct Found {
        int bin;
        uint32_t count, in_count;
        uint64_t weight, in_weight;
    };
    template <class P>
    __device__ __forceinline__ Found find(P &&reached) const {
        constexpr int PER = kBins / NT;
        __syncthreads();
        uint64_t w = 0;
        uint32_t c = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) w += hw[threadIdx.x * PER + j], c += hc[threadIdx.x * PER + j];
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const uint64_t sw = wave_scan(w);
        const uint32_t sc = wave_scan32(c);
        if (lane == 63) part[wave] = sw, ties[wave] = sc;
        if (threadIdx.x == 0) bin = kBins;
        __syncthreads();
        uint64_t bw = sw - w;
        uint32_t bc = sc - c;
        for (int k = 0; k < wave; ++k) bw += part[k], bc += ties[k];
        // The conditions are monotone in the running sums: they turn true in one bin.
        for (int j = 0; j < PER; ++j) {
            const int b = threadIdx.x * PER + j;
            const uint64_t iw = hw[b];
            const uint32_t ic = hc[b];
            if (!reached(bc, bw) && reached(bc + ic, bw + iw))
                bin = b, part[NW] = bw, ties[NW] = bc, part[NW + 1] = iw, ties[NW + 1] = ic;
            bc += ic, bw += iw;
        }
        __syncthreads();
        const int low = bin;
        Found f{low, 0, 0, 0, 0};
        if (low < kBins) f = Found{low, ties[NW], ties[NW + 1], part[NW], part[NW + 1]};
        __syncthreads();
        return f;
    }
};

template <class T, int VEC, int NT>
__global__ __launch_bounds__(NT) void k_sample_block(SampleArgs a) {
    using B = Block<T, VEC, NT>;
    constexpr int NW = NT / 64;
    __shared__ uint64_t hw[kBins], part[NW + 2];
    __shared__ uint32_t hc[kBins], ties[NW + 2], bound[2];
    __shared__ uint32_t pair_key[kPairs], pair_weight[kPairs];
    __shared__ int pair_at[kPairs], found, listed;
    const uint32_t r = block_index();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (r >= (uint32_t)a.n) return;
    const Row q = row_settings(a.p, r);
    const B b{static_cast<const T *>(a.logits) + r * a.stride, a.vocab, hw, hc, part, ties, found};

    // the largest logit
    float m = -kInf;
    b.all([&](int, float l) { m = fmaxf(m, l); });
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (lane == 0) ties[wave] = __float_as_uint(m);
    __syncthreads();
    for (int k = 0; k < NW; ++k) m = fmaxf(m, __uint_as_float(ties[k]));
    __syncthreads();
    if (!(m > -kInf)) {                             // nothing to choose from
        if (threadIdx.x == 0) {
            a.tokens[r] = -1;
            if (a.logprobs) a.logprobs[r] = -kInf;
        }
        return;
    }
    if (q.greedy) {
        int at = a.vocab;
        b.all([&](int i, float l) { at = l == m ? min(at, i) : at; });
#pragma unroll
        for (int d = 32; d; d >>= 1) at = min(at, __shfl_xor(at, d));
        if (lane == 0) ties[wave] = at;
        __syncthreads();
        for (int k = 0; k < NW; ++k) at = min(at, (int)ties[k]);
        if (threadIdx.x == 0) {
            a.tokens[r] = at;
            if (a.logprobs) a.logprobs[r] = 0.f;
        }
        return;
    }

    // What stays: logits above `cut`, and the first `equals` of those equal to it.
    float cut = -kInf;
    uint32_t equals = 0, equal_weight = 0;
    const bool use_k = q.top_k > 0 && q.top_k < a.vocab, use_p = q.top_p < 1.f;
    uint64_t all_weights = 0;
    constexpr int PER = kBins / NT;
    if (use_k || use_p || q.min_p > 0.f) {
        b.clear();
        b.all([&](int, float l) {
            const float z = z_of(l, m, q.c);
            if (z > -32.f) {
                const int s = (int)(z * -32.f);
                atomicAdd(&hc[s], 1u);
                if (use_p) {
                    const uint32_t w = weight_of(z, q.min_p);
                    if (w) atomicAdd((unsigned long long *)&hw[s], (unsigned long long)w);
                }
            }
        });
        __syncthreads();
        // The last bin that anything may stay of: min-p's, and one more for rounding
        // (NaN and infinities of its logarithm do not occur, it is above 0 and at most 1) ...
        int last = kBins - 1;
        if (q.min_p > 0.f) last = min(last, (int)fminf(log2f(q.min_p) * -32.f, (float)kBins) + 1);
        // ... the k-th largest's, or the one in which top-p's share is reached.
        if (use_p) {
            uint64_t w = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) w += hw[threadIdx.x * PER + j];
            w = wave_sum(w);
            if (lane == 0) part[wave] = w;
            __syncthreads();
            for (int i = 0; i < NW; ++i) all_weights += part[i];
            __syncthreads();
        }
        if (use_k) last = min(last, b.find([&](uint32_t c, uint64_t) { return c >= (uint32_t)q.top_k; }).bin);
        else if (use_p) {
            const double limit = fmax((double)q.top_p * (double)all_weights, 0.5);
            last = min(last, b.find([&](uint32_t, uint64_t w) { return (double)w >= limit; }).bin);
        }
        uint32_t n = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if ((int)threadIdx.x * PER + j <= last) n += hc[threadIdx.x * PER + j];
        n = (uint32_t)wave_sum(n);
        if (lane == 0) ties[wave] = n;
        __syncthreads();
        n = 0;
        for (int i = 0; i < NW; ++i) n += ties[i];
        __syncthreads();
        if (n <= kPairs) {
            if (threadIdx.x == 0) listed = 0;
            for (int i = threadIdx.x; i < kPairs; i += NT) pair_key[i] = 0, pair_weight[i] = 0, pair_at[i] = INT32_MAX;
            __syncthreads();
            b.all([&](int i, float l) {
                const float z = z_of(l, m, q.c);
                if (z > -32.f && (int)(z * -32.f) <= last) {
                    const int place = atomicAdd(&listed, 1);
                    pair_key[place] = key_of<T>(l);
                    pair_weight[place] = weight_of(z, q.min_p);
                    pair_at[place] = i;
                }
            });
            __syncthreads();
            // As in k_sample_wave: what comes before each in descending order (equal ones
            // by index), then in index order.  Entries past n weigh nothing and rank last.
            constexpr int TWO = kPairs > NT ? kPairs / NT : 1;
            uint64_t kept[TWO], sum = 0;
            bool in_k[TWO];
            uint64_t before[TWO];
#pragma unroll
            for (int o = 0; o < TWO; ++o) {
                const uint32_t i = threadIdx.x + o * NT;
                before[o] = 0, in_k[o] = false, kept[o] = 0;
                if (i < n) {
                    const uint32_t key = pair_key[i];
                    const int mine = pair_at[i];
                    int rank = 0;
#pragma unroll 8
                    for (uint32_t t = 0; t < (n + 7) / 8 * 8; ++t) {
                        const uint32_t kt = pair_key[t], wt = pair_weight[t];
                        const bool ahead = (kt > key) | ((kt == key) & (pair_at[t] < mine));
                        rank += ahead;
                        before[o] += ahead ? wt : 0;
                    }
                    in_k[o] = !use_k || rank < q.top_k;
                    kept[o] = in_k[o] ? pair_weight[i] : 0;
                    sum += kept[o];
                }
            }
            uint64_t total = all_weights;
            if (use_k || !use_p) {                          // all that top-p takes its share of is in the list
                sum = wave_sum(sum);
                if (lane == 0) part[wave] = sum;
                __syncthreads();
                total = 0;
                for (int i = 0; i < NW; ++i) total += part[i];
            }
            const double limit = (double)q.top_p * (double)total;
            sum = 0;
#pragma unroll
            for (int o = 0; o < TWO; ++o) {
                if (use_p && !(before[o] == 0 || (double)before[o] < limit)) kept[o] = 0;
                sum += kept[o];
            }
            __syncthreads();                                // all have read the weights and the parts
#pragma unroll
            for (int o = 0; o < TWO; ++o)
                if (threadIdx.x + o * NT < n) pair_weight[threadIdx.x + o * NT] = (uint32_t)kept[o];
            sum = wave_sum(sum);
            if (lane == 0) part[wave] = sum;
            __syncthreads();
            total = 0;
            for (int i = 0; i < NW; ++i) total += part[i];
            const uint64_t target = target_of(a.u[r], total);
#pragma unroll
            for (int o = 0; o < TWO; ++o) {
                const uint32_t i = threadIdx.x + o * NT;
                if (i < n && kept[o]) {
                    const int mine = pair_at[i];
                    uint64_t run = 0;
#pragma unroll 8
                    for (uint32_t t = 0; t < (n + 7) / 8 * 8; ++t) {
                        const uint32_t wt = pair_weight[t];
                        run += pair_at[t] < mine ? wt : 0;
                    }
                    if (run <= target && run + kept[o] > target) {
                        a.tokens[r] = mine;
                        if (a.logprobs) a.logprobs[r] = log_share(z_of(of_key<T>(pair_key[i]), m, q.c), total);
                    }
                }
            }
            return;
        }
    }
    if (use_k || use_p) {
        const auto bin_of = [&](float l) {          // descending logits have ascending bins
            const float z = z_of(l, m, q.c);
            return z > -32.f ? (int)(z * -32.f) : kBins;   // kBins: no weight
        };
        // Narrows a bin down to one key: the first key, from the largest down, at
        // which the running count and weight satisfy `reached`.
        struct Cut {
            float logit;
            uint32_t count, in_count;               // before it, and of its equals
            uint64_t weight;
        };
        const auto narrow = [&](typename B::Found f, float above, auto &&reached) {
            // The keys of the bin: its two edges, each searched by one wave, 64 places at
            // once.  Wave 0: the least key with a bin up to this one; wave 1: the least with
            // a bin before it, whose neighbour below is the bin's greatest (m's for
            // bin 0).
            if (wave < 2) {
                uint32_t lo = key_of<T>(-kInf), hi = key_of<T>(m);
                const int most = f.bin - wave;
                if (most >= 0) {
                    while (lo < hi) {                      // the answer lies in [lo, hi]
                        const uint32_t width = (hi - lo + 63) / 64;
                        const uint32_t probe = lo + min(hi - lo, (uint32_t)lane * width);
                        const uint64_t yes = __ballot(bin_of(of_key<T>(probe)) <= most);
                        const int first = yes ? __ffsll((unsigned long long)yes) - 1 : 64;
                        if (first == 0) hi = lo;
                        else {
                            const uint32_t below = lo + min(hi - lo, (uint32_t)(first - 1) * width);
                            if (first < 64) hi = lo + min(hi - lo, (uint32_t)first * width);
                            lo = below + 1;
                        }
                    }
                }
                if (lane == 0) bound[wave] = wave == 0 ? lo : f.bin > 0 ? lo - 1 : key_of<T>(m);
            }
            __syncthreads();
            uint32_t lo = bound[0], hi = bound[1];
            uint32_t count = f.count;
            uint64_t weight = f.weight;
            for (;;) {
                int shift = 0;
                while (((hi - lo) >> shift) >= kBins) ++shift;
                b.clear();
                const float from = of_key<T>(lo), to = of_key<T>(hi);
                b.all([&](int, float l) {
                    if (l >= from && l <= to && l > above) {
                        const uint32_t key = key_of<T>(l);     // -0 and 0 compare equal, and have one key
                        if (key < lo || key > hi) return;
                        const int s = (int)((hi - key) >> shift);
                        atomicAdd(&hc[s], 1u);
                        const uint32_t w = weight_of(z_of(l, m, q.c), q.min_p);
                        if (w) atomicAdd((unsigned long long *)&hw[s], (unsigned long long)w);
                    }
                });
                const typename B::Found g = b.find([&](uint32_t c, uint64_t w) { return reached(count + c, weight + w); });
                count += g.count, weight += g.weight;
                hi -= (uint32_t)g.bin << shift;
                if (shift == 0) return Cut{of_key<T>(hi), count, g.in_count, weight};
                const uint32_t span = (1u << shift) - 1;
                lo = hi - lo > span ? hi - span : lo;
            }
        };

        // The histogram is needed again for top-p: its bins are kept in registers.
        uint64_t keep_w[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) keep_w[j] = hw[threadIdx.x * PER + j];
        uint64_t total = 0, above_weight = 0;       // of what stays, and of that above `cut`
        int k_bin = kBins;
        bool cut_by_k = false;
        if (use_k) {
            const typename B::Found f = b.find([&](uint32_t c, uint64_t) { return c >= (uint32_t)q.top_k; });
            if (f.bin < kBins) {
                const Cut k = narrow(f, -kInf, [&](uint32_t c, uint64_t) { return c >= (uint32_t)q.top_k; });
                cut = k.logit, equals = q.top_k - k.count, cut_by_k = true, k_bin = f.bin;
                equal_weight = weight_of(z_of(cut, m, q.c), q.min_p);
                above_weight = k.weight;
                total = above_weight + (uint64_t)equals * equal_weight;
            }
        }
        if (use_p) {
            __syncthreads();
            if (!cut_by_k) total = all_weights;
            // Elements before which less than `limit` lies stay; the first has nothing before it.
            const double limit = fmax((double)q.top_p * (double)total, 0.5);
            const auto fill = [&](float logit, uint32_t count, uint64_t before) {
                cut = logit, equal_weight = weight_of(z_of(cut, m, q.c), q.min_p);
                const double each = (double)equal_weight;
                uint32_t e = (uint32_t)fmin(ceil((limit - (double)before) / fmax(each, 1.0)), (double)count);
                while (e > 0 && (double)(before + (uint64_t)(e - 1) * equal_weight) >= limit) --e;
                while (e < count && (double)(before + (uint64_t)e * equal_weight) < limit) ++e;
                equals = e;
            };
            if (cut_by_k && (double)above_weight < limit) {
                fill(cut, equals, above_weight);    // it lies among the last of the top k
            } else {
                // The bins again, without those below the top k's last (whose bin's own
                // weight below the cut cannot be reached: above_weight >= limit).
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int s = threadIdx.x * PER + j;
                    hw[s] = s <= k_bin ? keep_w[j] : 0, hc[s] = 0;
                }
                const auto reached = [&](uint32_t, uint64_t w) { return (double)w >= limit; };
                const typename B::Found f = b.find(reached);
                const Cut p = narrow(f, cut, reached);
                fill(p.logit, p.in_count, p.weight);
            }
        }
    }

    // The draw.  Parts of the row in order: NW contiguous ones, then the part the
    // target falls into in the same way, until a part is one vector a lane.
    int lo = 0, hi = a.vocab;
    uint64_t before = 0, target = 0, total = 0;     // weight before lo
    uint32_t seen = 0;                              // equals before lo
    const auto stays = [&](uint32_t had, uint32_t n) { return min(had + n, equals) - min(had, equals); };
    for (bool first = true; first || hi - lo > 64 * VEC; first = false) {
        const int grain = 64 * VEC;
        const int step = ((hi - lo + NW - 1) / NW + grain - 1) / grain * grain;
        const int from = lo + wave * step, to = min(hi, from + step);
        uint64_t w = 0;
        uint32_t e = 0;
        b.each(from, to, lane, 64, [&](int, float l) {
            if (l > cut) w += weight_of(z_of(l, m, q.c), q.min_p);
            else if (l == cut) ++e;
        });
        w = wave_sum(w), e = (uint32_t)wave_sum(e);
        if (lane == 0) part[wave] = w, ties[wave] = e;
        __syncthreads();
        if (first) {
            uint32_t s = 0;
            for (int k = 0; k < NW; ++k) total += part[k] + (uint64_t)stays(s, ties[k]) * equal_weight, s += ties[k];
            target = target_of(a.u[r], total);
        }
        int k = 0;
        for (; k < NW - 1; ++k) {
            const uint64_t in = part[k] + (uint64_t)stays(seen, ties[k]) * equal_weight;
            if (before + in > target) break;
            before += in, seen += ties[k];
        }
        lo += k * step, hi = min(hi, lo + step);
        __syncthreads();
    }
    if (wave == 0) {
        uint64_t w = 0;
        uint32_t e = 0;
        b.each(lo, hi, lane, 64, [&](int, float l) {
            if (l > cut) w += weight_of(z_of(l, m, q.c), q.min_p);
            else if (l == cut) ++e;
        });
        const uint32_t had = seen + (uint32_t)wave_scan(e) - e;
        const uint64_t mine = w + (uint64_t)stays(had, e) * equal_weight;
        const uint64_t upto = before + wave_scan(mine);
        const int owner = __ffsll((unsigned long long)__ballot(upto > target)) - 1;
        if (lane == owner) {
            uint64_t run = upto - mine;
            uint32_t s = had;
            int token = -1;
            float z = 0.f;
            b.each(lo, hi, lane, 64, [&](int i, float l) {
                const float zi = z_of(l, m, q.c);
                if (l > cut) run += weight_of(zi, q.min_p);
                else if (l == cut) run += (uint64_t)stays(s++, 1) * equal_weight;
                if (token < 0 && run > target) token = i, z = zi;
            });
            a.tokens[r] = token;
            if (a.logprobs) a.logprobs[r] = log_share(z, total);
        }
    }
}

template <class T, int VEC>
void launch_block(const SampleArgs &a, hipStream_t s) {
    // A row of up to 4096 leaves most of 1024 threads without work; a longer one
    // is worth all the waves a CU takes.
    if (a.vocab <= 4096) k_sample_block<T, VEC, 256><<<grid_of(a.n), 256, 0, s>>>(a);
    else k_sample_block<T, VEC, 1024><<<grid_of(a.n), 1024, 0, s>>>(a);
}

template <class T>
hipError_t run(const SampleArgs &a, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(T);
    if (a.vocab <= 64) k_sample_wave<T><<<grid_of(((int64_t)a.n + 3) / 4), 256, 0, s>>>(a);
    else if (reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.stride % VEC == 0) launch_block<T, VEC>(a, s);
    else launch_block<T, 1>(a, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? run<bf16_t>(a, s) : run<float>(a, s);
}

}  // namespace rn
