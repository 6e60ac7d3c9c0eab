// Log-probabilities of given choices, entropy, the likeliest alternatives, and the
// gradient of the first two.
//
// With m a row's largest logit, c = log2(e) / temperature, z_i = (l_i - m) c:
//   s = sum 2^z_i, w = sum z_i 2^z_i,
//   log p_t = z_t ln 2 - log s,  entropy = log s - ln 2 w / s
// (both terms of the entropy are 0 or more: nothing cancels), in one pass: where a
// larger logit is met, by d in z, s becomes s 2^-d and w (w - d s) 2^-d.  Backward:
//   p_i = 2^z_i / s,  dl_i = (dlogp ([i = t] - p_i) - dent p_i (log p_i + entropy)) / temperature.
//
// Alternatives rank by key: the logit's bits in an order of whole numbers, then the
// lowest index, so that keys are distinct.  Each pair of threads knows the largest of
// its logits; the top-th largest of those is a bound below which no alternative lies,
// and only the pairs above it have any: their logits are read once more.  (Fours of
// threads: 4096 rows of 5000 with 20 alternatives 31 us and with 64 114, pairs 33 and
// 41, every thread by itself 46 and 50, for 256 keys are ranked against 256.)
//
// Bound by HBM: a logit is read once forward (a few are, twice) and once backward.
// 2048 rows of 131072 bfloat16, 537 MB: 135 us forward (4.0 TB/s), half as long again
// with 20 alternatives; 210 backward (5.1 TB/s).  4096 rows of 18: 3.5 and 2.8 us.
#include "rn_ops.hpp"

namespace rn {
namespace {

using namespace ops;

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();
constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kGroup = 2, kGroups = kThreads / kGroup;       // RN_LOGPROBS_MAX_TOP groups, or more
constexpr int kAhead = 2;         // vectors a thread has on their way at once
constexpr int kList = 1024;       // alternatives that are ranked at once
static_assert(kGroups >= RN_LOGPROBS_MAX_TOP);
// Smaller rows are in the registers of a wave or less (kWaveVocab / 64 logits a lane).
constexpr int kWaveVocab = 1024;

// NaN ranks as -infinity, -0 as +0.
__device__ inline uint64_t key_of(float l, uint32_t i) {
    const uint32_t b = __float_as_uint(l == l ? l + 0.f : -kInf);
    return (uint64_t)(b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (uint32_t)~i;
}
__device__ inline uint32_t index_of(uint64_t key) { return ~(uint32_t)key; }
__device__ inline float logit_of(uint64_t key) {
    const uint32_t k = (uint32_t)(key >> 32);
    return __uint_as_float(k ^ ((int32_t)k < 0 ? 0x80000000u : 0xffffffffu));
}

// m, s and w of some of a row's logits.  None, or only -infinity: m = -infinity, s = w = 0.
struct Sums {
    float m, s, w;
};
constexpr Sums kNone = {-kInf, 0.f, 0.f};

// Towards a largest logit m >= a.m.
__device__ inline Sums raised(const Sums &a, float m, float c) {
    if (a.m == m || a.m == -kInf) return {m, a.s, a.w};        // -infinity: s and w are 0
    const float d = (a.m - m) * c, f = __builtin_amdgcn_exp2f(d);
    return {m, a.s * f, fmaf(d > -1e30f ? d : -1e30f, a.s, a.w) * f};
}
__device__ inline Sums joined(const Sums &a, const Sums &b, float c) {
    const float m = fmaxf(a.m, b.m);
    const Sums x = raised(a, m, c), y = raised(b, m, c);
    return {m, x.s + y.s, x.w + y.w};
}
// One more logit, at most a.m.  NaN and infinities make s NaN.
__device__ inline void add(Sums &a, float base, float l, float c) {
    const float z = (l - base) * c, e = __builtin_amdgcn_exp2f(z);
    a.s += e;
    a.w = fmaf(fmaxf(z, -1e30f), e, a.w);                      // 0 (-infinity) is 0
}

template <int G>
__device__ inline Sums over_lanes(Sums a, float c) {
#pragma unroll
    for (int d = G / 2; d; d >>= 1) a = joined(a, {__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.w, d)}, c);
    return a;
}

// What is known of a row once its sums are.
struct Row {
    float m, log_s, inv_t;
    bool none;                    // nothing but -infinity
    __device__ Row(const Sums &a, float inv_t) : m(a.m), log_s(logf(a.s)), inv_t(inv_t), none(a.s == 0.f) {}
    // +infinity: NaN, as s is.
    __device__ float logp(float l) const { return none ? -kInf : (l == l ? (l - m) * inv_t - log_s : log_s); }
};

template <class T>
__device__ inline void finish(const LogpArgs &a, int64_t r, const Sums &x, const Row &row) {
    const float entropy = row.none ? 0.f : row.log_s - kLn2 * x.w / x.s;
    if (a.logprobs) {
        const int t = a.tokens[r];
        const bool in = t >= 0 && t < a.vocab;
        const float l = in ? to_float(static_cast<const T *>(a.logits)[r * a.stride + t]) : 0.f;
        a.logprobs[r] = in ? row.logp(l) : 0.f;
    }
    if (a.entropy) a.entropy[r] = entropy;
    if (a.stats) {
        float *st = a.stats + 4 * r;
        st[0] = x.m, st[1] = row.none ? 0.f : 1.f / x.s, st[2] = row.none ? 0.f : row.log_s, st[3] = entropy;
    }
}

__device__ inline void write_top(const LogpArgs &a, int64_t r, int place, uint64_t key, const Row &row, bool nan) {
    a.top_tokens[r * a.top + place] = (int32_t)index_of(key);
    a.top_logprobs[r * a.top + place] = nan ? row.log_s : row.logp(logit_of(key));
}

// ------------------------------------------------------------------ rows within a wave

// G lanes a row, ITEMS logits each: lane + G i.
template <class T, int G, int ITEMS>
__global__ __launch_bounds__(kThreads) void k_logp_rows(LogpArgs a) {
    const int lane = threadIdx.x % G;
    const int64_t r = (int64_t)block_index() * (kThreads / G) + threadIdx.x / G;
    if (r >= a.n) return;                                      // whole groups of lanes at once
    const T *x = static_cast<const T *>(a.logits) + r * a.stride;
    float l[ITEMS];
    float m = -kInf;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        l[i] = lane + G * i < a.vocab ? to_float(x[lane + G * i]) : -kInf;
        m = fmaxf(m, l[i]);
    }
#pragma unroll
    for (int d = G / 2; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    Sums s = {m, 0.f, 0.f};
    const float base = m == -kInf ? 0.f : m;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (lane + G * i < a.vocab) add(s, base, l[i], a.c);
#pragma unroll
    for (int d = G / 2; d; d >>= 1) s.s += __shfl_xor(s.s, d), s.w += __shfl_xor(s.w, d);
    const Row row(s, a.inv_t);
    if (lane == 0) finish<T>(a, r, s, row);
    if (!a.top) return;
    const bool nan = s.s != s.s;
    uint32_t left = (1u << ITEMS) - 1;
    for (int k = 0; k < a.top; ++k) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (lane + G * i < a.vocab && left >> i & 1) best = max(best, key_of(l[i], lane + G * i));
        const uint64_t mine = best;
#pragma unroll
        for (int d = G / 2; d; d >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, d));
        if (mine == best) left &= ~(1u << (index_of(best) / G));
        if (lane == 0) write_top(a, r, k, best, row, nan);
    }
}

// ------------------------------------------------------------------ long rows

// A row's logits in vectors that begin on 16 bytes: vector v holds elements
// v VEC - shift and on, the first and last vector some that are not the row's.
template <class T>
struct Vectors {
    static constexpr int VEC = 16 / sizeof(T);
    const T *x;
    int vocab, shift;
    __device__ Vectors(const T *x, int vocab)
        : x(x), vocab(vocab), shift((int)(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T))) {}
    __device__ int count() const { return (vocab + shift + VEC - 1) / VEC; }
    __device__ int first(int v) const { return v * VEC - shift; }
    __device__ bool whole(int v) const { return first(v) >= 0 && first(v) + VEC <= vocab; }
    __device__ bool has(int v, int j) const { return (unsigned)(first(v) + j) < (unsigned)vocab; }
    // What is not the row's reads as -infinity.
    __device__ void load(int v, float (&l)[VEC]) const {
        if (whole(v)) {
            const Pack<T, VEC> p = *reinterpret_cast<const Pack<T, VEC> *>(x + first(v));
#pragma unroll
            for (int j = 0; j < VEC; ++j) l[j] = to_float(p.v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) l[j] = has(v, j) ? to_float(x[first(v) + j]) : -kInf;
        }
    }
};

// Part `part` of a row, by one block: its sums (thread 0 has them), and its `top`
// largest keys in lds order (keys[], 0 where there are none).
template <class T>
struct Part {
    static constexpr int VEC = Vectors<T>::VEC;
    Vectors<T> vec;
    int lo, hi;                   // vectors of the part

    struct Lds {
        Sums sums[kWaves];
        uint64_t best[kGroups], list[kList], bound;
        int winner[RN_LOGPROBS_MAX_TOP], winners, count;
        uint64_t top[RN_LOGPROBS_MAX_TOP];
    };

    __device__ Part(const LogpArgs &a, int64_t r, int part)
        : vec(static_cast<const T *>(a.logits) + r * a.stride, a.vocab) {
        const int all = vec.count(), per = (all + a.parts - 1) / a.parts;
        lo = min(all, part * per), hi = min(all, lo + per);
    }

    __device__ uint64_t largest_of(int v, const float (&l)[VEC], uint64_t below) const {
        uint64_t best = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const uint64_t key = vec.has(v, j) ? key_of(l[j], vec.first(v) + j) : 0;
            if (key < below) best = max(best, key);
        }
        return best;
    }

    // TOP is no argument, for what it needs costs the other calls 30% (registers).
    template <bool TOP>
    __device__ Sums sums(Lds &lds, float c) const {
        Sums s = kNone;
        uint64_t best = 0;
        float best_logit = -kInf;
        const auto take = [&](int v, const float (&l)[VEC]) {
            float m = l[0];
#pragma unroll
            for (int j = 1; j < VEC; ++j) m = fmaxf(m, l[j]);
            if (m > s.m) s = raised(s, m, c);
            const float base = s.m == -kInf ? 0.f : s.m;
#pragma unroll
            for (int j = 0; j < VEC; ++j) add(s, base, l[j], c);
            // Equal ones later on rank behind: only a larger one, or the first, is looked at.
            if (TOP && (m > best_logit || best == 0)) {
                best = max(best, largest_of(v, l, ~0ull));
                best_logit = logit_of(best);
            }
        };
        const auto edge = [&](int v) {                  // the row's first or last vector, of which it has a part
            float l[VEC];
            vec.load(v, l);
            take(v, l);
        };
        int v = lo + threadIdx.x;
        int had = -1;
        if (v < hi && !vec.whole(v)) edge(v), had = v, v += kThreads;
        const int end = hi > lo && !vec.whole(hi - 1) ? hi - 1 : hi;
        if (v < end) {
            // The next vectors are on their way while these are worked on.
            Pack<T, VEC> next[kAhead];
            const auto fetch = [&](int v) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    next[u] = *reinterpret_cast<const Pack<T, VEC> *>(vec.x + vec.first(min(v + u * kThreads, end - 1)));
            };
            fetch(v);
            for (; v < end; v += kAhead * kThreads) {
                float l[kAhead][VEC];
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) l[u][j] = to_float(next[u].v[j]);
                fetch(v + kAhead * kThreads);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (v + u * kThreads < end) take(v + u * kThreads, l[u]);
            }
        }
        if (end < hi && end != had && (end - lo) % kThreads == threadIdx.x) edge(end);
        s = over_lanes<64>(s, c);
        if ((threadIdx.x & 63) == 0) lds.sums[threadIdx.x >> 6] = s;
        if constexpr (TOP) {
#pragma unroll
            for (int d = 1; d < kGroup; d *= 2) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, d));
            lds.best[threadIdx.x / kGroup] = best;
            if (threadIdx.x == 0) lds.winners = lds.count = 0, lds.bound = 1;
        }
        __syncthreads();
        s = lds.sums[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s = joined(s, lds.sums[w], c);
        return s;
    }

    // After sums(): the part's largest keys to lds.top.
    __device__ void top(Lds &lds, int k) const {
        if (threadIdx.x < kGroups) {
            const uint64_t mine = lds.best[threadIdx.x];
            int before = 0;
#pragma unroll 16
            for (int i = 0; i < kGroups; ++i) before += lds.best[i] > mine;
            if (mine && before < k) {
                lds.winner[before] = threadIdx.x;
                atomicAdd(&lds.winners, 1);
                if (before == k - 1) lds.bound = mine;
            }
        }
        if (threadIdx.x < k) lds.top[threadIdx.x] = 0;
        __syncthreads();
        const uint64_t bound = lds.bound;
        const int turns = (hi - lo + kThreads - 1) / kThreads, each = turns * kGroup, all = lds.winners * each;
        const auto vector_of = [&](int q) {
            return lo + lds.winner[q / each] * kGroup + q % kGroup + q % each / kGroup * kThreads;
        };
        for (int q = threadIdx.x; q < all; q += kThreads) {
            const int v = vector_of(q);
            if (v >= hi) continue;
            float l[VEC];
            vec.load(v, l);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const uint64_t key = vec.has(v, j) ? key_of(l[j], vec.first(v) + j) : 0;
                if (key >= bound) {
                    const int at = atomicAdd(&lds.count, 1);
                    if (at < kList) lds.list[at] = key;
                }
            }
        }
        __syncthreads();
        if (const int count = lds.count; count <= kList) {
            // The list is in no order, but keys are distinct: each has one place.
            for (int i = threadIdx.x; i < count; i += kThreads) {
                const uint64_t key = lds.list[i];
                int place = 0;
                for (int j = 0; j < count; ++j) place += lds.list[j] > key;
                if (place < k) lds.top[place] = key;
            }
        } else {
            // Few threads hold very many of the largest: one alternative a turn.
            uint64_t below = ~0ull;
            for (int i = 0; i < k; ++i) {
                uint64_t best = 0;
                for (int q = threadIdx.x; q < all; q += kThreads) {
                    const int v = vector_of(q);
                    if (v >= hi) continue;
                    float l[VEC];
                    vec.load(v, l);
                    best = max(best, largest_of(v, l, below));
                }
#pragma unroll
                for (int d = 32; d; d >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, d));
                __syncthreads();                               // the last turn's list[] has been read
                if ((threadIdx.x & 63) == 0) lds.list[threadIdx.x >> 6] = best;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kWaves; ++w) best = max(best, lds.list[w]);
                below = best;
                if (threadIdx.x == 0) lds.top[i] = best;
                if (best == 0) break;
            }
        }
        __syncthreads();
    }
};

// One block a row (parts = 1), or a part of one, whose sums and keys go to scratch.
template <class T, bool TOP>
__global__ __launch_bounds__(kThreads) void k_logp_part(LogpArgs a) {
    __shared__ typename Part<T>::Lds lds;
    const int64_t i = block_index(), r = i / a.parts;
    if (r >= a.n) return;
    const Part<T> part(a, r, (int)(i % a.parts));
    const Sums s = part.template sums<TOP>(lds, a.c);
    if constexpr (TOP) part.top(lds, a.top);
    if (a.parts > 1) {
        if (threadIdx.x == 0) a.part_sums[3 * i] = s.m, a.part_sums[3 * i + 1] = s.s, a.part_sums[3 * i + 2] = s.w;
        if ((int)threadIdx.x < a.top) a.part_keys[i * a.top + threadIdx.x] = lds.top[threadIdx.x];
        return;
    }
    const Row row(s, a.inv_t);
    if (threadIdx.x == 0) finish<T>(a, r, s, row);
    if ((int)threadIdx.x < a.top) write_top(a, r, threadIdx.x, lds.top[threadIdx.x], row, s.s != s.s);
}

// A row's parts, in their order.
template <class T>
__global__ __launch_bounds__(kThreads) void k_logp_join(LogpArgs a) {
    __shared__ uint64_t keys[kList];
    const int64_t r = block_index();
    if (r >= a.n) return;
    Sums s = kNone;
    if ((int)(threadIdx.x & 63) < a.parts) {
        const float *p = a.part_sums + 3 * (r * a.parts + (threadIdx.x & 63));
        s = {p[0], p[1], p[2]};
    }
    s = over_lanes<64>(s, a.c);
    const Row row(s, a.inv_t);
    if (threadIdx.x == 0) finish<T>(a, r, s, row);
    const int count = a.parts * a.top;                         // at most kList
    for (int i = threadIdx.x; i < count; i += kThreads) keys[i] = a.part_keys[r * count + i];
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += kThreads) {
        const uint64_t key = keys[i];
        int place = 0;
        for (int j = 0; j < count; ++j) place += keys[j] > key;
        if (key && place < a.top) write_top(a, r, place, key, row, s.s != s.s);
    }
}

// ------------------------------------------------------------------ gradient

struct Slope {
    float base, inv, log_s, entropy, c, inv_t, dlogp, dent;
    int token;
    __device__ Slope(const LogpArgs &a, int64_t r) : c(a.c), inv_t(a.inv_t) {
        const float *st = a.stats + 4 * r;
        base = st[0] == -kInf ? 0.f : st[0], inv = st[1], log_s = st[2], entropy = st[3];
        token = a.tokens[r];
        // Nothing to choose from, or no choice: no gradient of it.
        dlogp = a.dlogprobs && inv != 0.f && token >= 0 && token < a.vocab ? a.dlogprobs[r] : 0.f;
        dent = a.dentropy ? a.dentropy[r] : 0.f;
    }
    __device__ float operator()(float l, int i) const {
        const float z = (l - base) * c, p = __builtin_amdgcn_exp2f(z) * inv;
        float g = -dlogp * p;
        if (p != 0.f) g = fmaf(-dent * p, fmaf(z, kLn2, entropy - log_s), g);
        if (i == token) g += dlogp;
        return g * inv_t;
    }
};

// G lanes a row, for rows of up to kWaveVocab.
template <class T, int G>
__global__ __launch_bounds__(kThreads) void k_logp_bwd_rows(LogpArgs a) {
    const int64_t r = (int64_t)block_index() * (kThreads / G) + threadIdx.x / G;
    if (r >= a.n) return;
    const Slope slope(a, r);
    const T *x = static_cast<const T *>(a.logits) + r * a.stride;
    T *dx = static_cast<T *>(a.dlogits) + r * a.dstride;
    for (int i = threadIdx.x % G; i < a.vocab; i += G) dx[i] = from_float<T>(slope(to_float(x[i]), i));
}

constexpr int kTurns = 8;         // vectors a thread

// kTurns x 256 vectors of a row a block; single elements where the logits' rows and
// the gradient's are not on the same bytes of 16.
template <class T>
__global__ __launch_bounds__(kThreads) void k_logp_bwd(LogpArgs a, int pieces) {
    constexpr int VEC = 16 / sizeof(T);
    const int64_t i = block_index(), r = i / pieces;
    if (r >= a.n) return;
    const Slope slope(a, r);
    const Vectors<T> vec(static_cast<const T *>(a.logits) + r * a.stride, a.vocab);
    T *dx = static_cast<T *>(a.dlogits) + r * a.dstride;
    const bool same = (reinterpret_cast<uintptr_t>(dx) - reinterpret_cast<uintptr_t>(vec.x)) % 16 == 0;
    const int lo = (int)(i % pieces) * (kTurns * kThreads) + threadIdx.x, count = vec.count();
    float l[kTurns][VEC];
#pragma unroll
    for (int u = 0; u < kTurns; ++u)
        if (const int v = lo + u * kThreads; v < count) vec.load(v, l[u]);
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int v = lo + u * kThreads, first = vec.first(v);
        if (v >= count) break;
        Pack<T, VEC> p;
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.v[j] = from_float<T>(slope(l[u][j], first + j));
        if (same && vec.whole(v)) {
            *reinterpret_cast<Pack<T, VEC> *>(dx + first) = p;
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (vec.has(v, j)) dx[first + j] = p.v[j];
        }
    }
}

template <class F>
void for_lanes(int vocab, F &&f) {
    using std::integral_constant;
    const auto go = [&](auto g, auto i) { f(g, i); };
    if (vocab <= 8) go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (vocab <= 16) go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (vocab <= 32) go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (vocab <= 64) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (vocab <= 128) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (vocab <= 256) go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (vocab <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else go(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

template <class T>
hipError_t run_forward(const LogpArgs &a, hipStream_t s) {
    if (a.vocab <= kWaveVocab) {
        for_lanes(a.vocab, [&](auto g, auto i) {
            constexpr int G = decltype(g)::value, RPB = kThreads / G;
            k_logp_rows<T, G, decltype(i)::value><<<grid_of(((int64_t)a.n + RPB - 1) / RPB), kThreads, 0, s>>>(a);
        });
        return hipGetLastError();
    }
    const dim3 grid = grid_of((int64_t)a.n * a.parts);
    if (a.top) k_logp_part<T, true><<<grid, kThreads, 0, s>>>(a);
    else k_logp_part<T, false><<<grid, kThreads, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.parts > 1) k_logp_join<T><<<grid_of(a.n), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t run_backward(const LogpArgs &a, hipStream_t s) {
    if (a.vocab <= kWaveVocab) {
        for_lanes(a.vocab, [&](auto g, auto) {
            constexpr int G = decltype(g)::value, RPB = kThreads / G;
            k_logp_bwd_rows<T, G><<<grid_of(((int64_t)a.n + RPB - 1) / RPB), kThreads, 0, s>>>(a);
        });
        return hipGetLastError();
    }
    constexpr int VEC = 16 / sizeof(T), PER = kTurns * kThreads;
    // A row may begin inside a vector.  (Where none does and vocab is a multiple of PER
    // vectors, a block a row has nothing to do: one of 9 at 131072 bfloat16.)
    const int pieces = ((a.vocab + VEC - 1) / VEC + 1 + PER - 1) / PER;
    k_logp_bwd<T><<<grid_of((int64_t)a.n * pieces), kThreads, 0, s>>>(a, pieces);
    return hipGetLastError();
}

}  // namespace

// Blocks a row: rows are shared where there are too few to fill the GPU, as long as
// a part has four vectors a thread, its sums fit a wave and its keys the join's list.
// 64 rows of 131072 with 20 alternatives: in 512 blocks 18 us and the join 5.5, in 1024
// 21 and 12, in 2048 27 and 30.
int logp_parts(int n, int vocab, int top, bool bf16) {
    if (vocab <= kWaveVocab || n <= 0 || n >= 512) return 1;
    const int vectors = vocab / (bf16 ? 8 : 4), want = (512 + n - 1) / n;
    int p = vectors / (4 * kThreads);
    if (p > want) p = want;
    if (p > 32) p = 32;
    if (top > 0 && p > kList / top) p = kList / top;
    return p < 1 ? 1 : p;
}

hipError_t launch_logp(const LogpArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? run_forward<bf16_t>(a, s) : run_forward<float>(a, s);
}

hipError_t launch_logp_backward(const LogpArgs &a, bool bf16, hipStream_t s) {
    return bf16 ? run_backward<bf16_t>(a, s) : run_backward<float>(a, s);
}

}  // namespace rn
