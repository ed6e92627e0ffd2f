// trie_sample: one token a row from a batch of logits, by temperature, top-k,
// top-p, min-p and a grammar, with its log-probability.
//
// With x the allowed logits of a row (NaN counts as -inf), M the largest and
// w = exp((x - M) / T): order the tokens by (x descending, id ascending); keep
// the first k; of those each whose predecessors' weights sum to less than
// top_p times the weight of the first k; of those the ones with w >= min_p.
// The token is drawn in two steps, a group of kGroup consecutive ids and then
// a token of it, each by the largest of log(weight) + Gumbel noise, which draws
// with probabilities proportional to the weights (the maximum of variables
// shifted by log-weights is categorical). Noise number n of a row is
// -log(-log u), u from 23 bits of splitmix64(seed, n): number t for token t,
// 2^31 + j for group j. Two steps make the noise of an unfiltered row cost
// V / kGroup + kGroup numbers instead of V, and the draw does not depend on
// how a running sum over the vocabulary is rounded.
//
//  k_sample_groups  largest logit and sum of exp((x - largest) / T) of every
//                   group: the one pass over the logits.
//  k_sample_pick    one CTA per row: M and the total weight from the groups'
//                   values; then only groups that can matter are read again.
//                   The k-th largest group maximum bounds the k-th largest
//                   logit from below, so the first k (or a first guess at the
//                   top-p set) come from a few groups into a list in shared
//                   memory, which is sorted. A row whose kept set does not fit
//                   the list finds the last kept logit by a radix select over
//                   the groups, with weights summed in 40-bit fixed point (the
//                   order of atomic additions then does not matter).
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <cuda_runtime.h>

#include "logits.cuh"

namespace tmk {

namespace {

constexpr int kGroup = 256;
constexpr int kGroupThreads = 256;  // k_sample_groups
constexpr int kThreads = 512;       // k_sample_pick
constexpr int kWarps = kThreads / 32;
constexpr int kList = 2048;
constexpr int kListK = 1024;        // largest top-k that goes through the list
constexpr int kGuess = 64;          // groups of the first guess at a top-p set
constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kKeyNone = 0x007FFFFFu;  // order_key(-inf)
constexpr double kFixed = 1099511627776.0;  // 2^40

struct SampleArgs {
    const void *logits;
    int64_t stride;
    int32_t V;
    int32_t G;                // groups of a row
    const int64_t *seeds;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    Grammar g;
    float2 *stats;            // [B][G]
    int32_t *tokens;
    float *logprobs;
};

// How one row is sampled.
struct Way {
    float T;
    bool greedy;
    int32_t k;   // 0: off
    float p;     // 1: off
    float min_p; // 0: off
};

__device__ __forceinline__ Way row_way(const SampleArgs &a, int32_t b) {
    Way w;
    w.T = a.temperature ? __ldg(a.temperature + b) : 1.0f;
    w.greedy = !(w.T > 0.0f);
    if (w.greedy) w.T = 1.0f;
    w.k = a.top_k ? __ldg(a.top_k + b) : 0;
    if (w.k < 0 || w.k >= a.V) w.k = 0;
    w.p = a.top_p ? __ldg(a.top_p + b) : 1.0f;
    if (!(w.p < 1.0f)) w.p = 1.0f;
    w.min_p = a.min_p ? __ldg(a.min_p + b) : 0.0f;
    if (!(w.min_p > 0.0f)) w.min_p = 0.0f;
    return w;
}

// Unsigned order of floats: a > b as floats iff order_key(a) > order_key(b).
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// A logit as the sampler sees it: NaN is -inf, and -0 is +0 (they are equal).
__device__ __forceinline__ float clean(float x) { return x == x ? x + 0.0f : -INFINITY; }

template <typename T>
struct Row {
    const T *x;
    GrammarRow allow;
    int32_t V;
    __device__ __forceinline__ float operator()(int32_t v) const {
        return v < V && allow.allows(v) ? clean(to_f32(x[v])) : -INFINITY;
    }
};

template <typename T>
__device__ __forceinline__ Row<T> row_at(const SampleArgs &a, int32_t b) {
    Row<T> r;
    r.x = static_cast<const T *>(a.logits) + b * a.stride;
    r.allow = grammar_row(a.g, b);
    r.V = a.V;
    return r;
}

__device__ __forceinline__ float scaled(float x, float M, float T) { return x == M ? 0.0f : __fdiv_rn(x - M, T); }
__device__ __forceinline__ float weight(float x, float M, float T) {
    return x > -INFINITY ? exp2f(scaled(x, M, T) * kLog2e) : 0.0f;
}

__device__ __forceinline__ float gumbel(int64_t seed, uint64_t n) {
    uint64_t z = uint64_t(seed) + (n + 1) * 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    z ^= z >> 31;
    const float u = float(2u * uint32_t(z >> 41) + 1u) * 0x1p-24f;  // exact, in (0, 1)
    return -logf(-logf(u));
}

// ------------------------------------------------------------- reductions

// A score and what it belongs to; the larger score wins, then the smaller id.
struct Best {
    float score;
    int32_t id;
};
__device__ __forceinline__ Best better(Best a, Best b) {
    return b.score > a.score || (b.score == a.score && uint32_t(b.id) < uint32_t(a.id)) ? b : a;
}
__device__ __forceinline__ Best warp_best(Best x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        Best y;
        y.score = __shfl_xor_sync(~0u, x.score, d);
        y.id = __shfl_xor_sync(~0u, x.id, d);
        x = better(x, y);
    }
    return x;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

struct Shared {
    unsigned long long list[kList];     // order_key << 32 | ~id
    float before[kList];                // weights of the list before each entry; then groups' weights
    uint32_t count[256];
    unsigned long long mass[256];
    Best best[kWarps];
    float f[kWarps];
    int32_t n;
    uint32_t key;
    int32_t ties;
    unsigned long long above, total;
};

__device__ Best block_best(Shared &s, Best x) {
    x = warp_best(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.best[threadIdx.x >> 5] = x;
    __syncthreads();
    x = s.best[0];
    for (int i = 1; i < kWarps; i++) x = better(x, s.best[i]);
    return x;
}
__device__ float block_max(Shared &s, float x) {
    x = warp_max(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.f[threadIdx.x >> 5] = x;
    __syncthreads();
    x = s.f[0];
    for (int i = 1; i < kWarps; i++) x = fmaxf(x, s.f[i]);
    return x;
}
__device__ float block_sum(Shared &s, float x) {
    x = warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.f[threadIdx.x >> 5] = x;
    __syncthreads();
    x = s.f[0];
    for (int i = 1; i < kWarps; i++) x += s.f[i];
    return x;
}

// ------------------------------------------------------------ the one pass

template <typename T>
__global__ void __launch_bounds__(kGroupThreads) k_sample_groups(SampleArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int32_t b = blockIdx.y;
    const Way way = row_way(a, b);
    const Row<T> row = row_at<T>(a, b);
    const float c = __fdiv_rn(kLog2e, way.T);
    for (int32_t j = blockIdx.x * (kGroupThreads / 32) + (threadIdx.x >> 5); j < a.G;
         j += gridDim.x * (kGroupThreads / 32)) {
        float x[kGroup / 32], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < kGroup / 32; i++) {
            const int64_t v = int64_t(j) * kGroup + i * 32 + lane;
            x[i] = v < a.V ? row(int32_t(v)) : -INFINITY;
            m = fmaxf(m, x[i]);
        }
        m = warp_max(m);
        float sum = 0.0f;
        if (m > -INFINITY) {
#pragma unroll
            for (int i = 0; i < kGroup / 32; i++) sum += x[i] == m ? 1.0f : exp2f((x[i] - m) * c);
            sum = warp_sum(sum);
        }
        if (lane == 0) a.stats[int64_t(b) * a.G + j] = make_float2(m, sum);
    }
}

// ------------------------------------------------------------ one row's draw

// The m-th largest group maximum as a key (kKeyNone when there are fewer).
__device__ uint32_t nth_group(const float2 *stats, int32_t G, int32_t m) {
    uint32_t key = 0u;
    for (int bit = 31; bit >= 0; bit--) {
        const uint32_t tryit = key | (1u << bit);
        int32_t n = 0;
        for (int32_t j0 = 0; j0 < G; j0 += kThreads) {
            const int32_t j = j0 + int32_t(threadIdx.x);
            n += __syncthreads_count(j < G && order_key(stats[j].x) >= tryit);
        }
        if (n >= m) key = tryit;
    }
    return key > kKeyNone ? key : kKeyNone;
}

// Collects every allowed token with order_key >= key into s.list; returns how
// many there are (more than kList: only that many were stored).
template <typename T>
__device__ int32_t collect(Shared &s, const Row<T> &row, const float2 *stats, int32_t G, uint32_t key) {
    const int lane = threadIdx.x & 31;
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    for (int32_t j = threadIdx.x >> 5; j < G; j += kWarps) {
        if (order_key(stats[j].x) < key) continue;
        for (int i = 0; i < kGroup / 32; i++) {
            const int64_t v = int64_t(j) * kGroup + i * 32 + lane;
            const uint32_t k = v < row.V ? order_key(row(int32_t(v))) : 0u;
            const bool in = k >= key && k > kKeyNone;
            const uint32_t m = __ballot_sync(~0u, in);
            if (!m) continue;
            int32_t at = 0;
            if (lane == 0) at = atomicAdd(&s.n, __popc(m));
            at = __shfl_sync(~0u, at, 0) + __popc(m & ((1u << lane) - 1u));
            if (in && at < kList) s.list[at] = (uint64_t(k) << 32) | uint32_t(~uint32_t(v));
        }
    }
    __syncthreads();
    return s.n;
}

// Sorts s.list[0, n) in descending order (a bitonic network over the next power of two).
__device__ void sort_list(Shared &s, int32_t n) {
    int32_t size = 2;
    while (size < n) size <<= 1;
    for (int32_t i = n + int32_t(threadIdx.x); i < size; i += kThreads) s.list[i] = 0ull;
    for (int32_t k = 2; k <= size; k <<= 1) {
        for (int32_t d = k >> 1; d; d >>= 1) {
            __syncthreads();
            for (int32_t i = threadIdx.x; i < size / 2; i += kThreads) {
                const int32_t lo = (i / d) * 2 * d + i % d, hi = lo + d;
                const unsigned long long x = s.list[lo], y = s.list[hi];
                if (((lo & k) == 0) == (x < y)) {
                    s.list[lo] = y;
                    s.list[hi] = x;
                }
            }
        }
    }
    __syncthreads();
}

__device__ __forceinline__ int32_t list_id(unsigned long long e) { return int32_t(~uint32_t(e)); }
__device__ __forceinline__ float list_value(unsigned long long e) { return key_value(uint32_t(e >> 32)); }

// s.before[i] = weight of s.list[0, i); returns the whole list's weight. One
// thread's share is consecutive entries, so the sums' order is fixed.
__device__ float scan_list(Shared &s, int32_t n, float M, float T) {
    constexpr int kPer = kList / kThreads;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float w[kPer], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int32_t at = int32_t(threadIdx.x) * kPer + i;
        w[i] = at < n ? weight(list_value(s.list[at]), M, T) : 0.0f;
        sum += w[i];
    }
    float upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const float y = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += y;
    }
    __syncthreads();
    if (lane == 31) s.f[warp] = upto;
    __syncthreads();
    float base = 0.0f, total = 0.0f;
    for (int i = 0; i < kWarps; i++) {
        if (i < warp) base += s.f[i];
        total += s.f[i];
    }
    float at = base + (upto - sum);
    if (lane == 0) at = base;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int32_t p = int32_t(threadIdx.x) * kPer + i;
        if (p < n) s.before[p] = at;
        at += w[i];
    }
    __syncthreads();
    return total;
}

// Draws from the first n entries of the sorted list.
__device__ int32_t draw_list(Shared &s, int32_t n, float M, float T, int64_t seed) {
    for (int32_t i = threadIdx.x; i < n; i += kThreads) s.before[i] = weight(list_value(s.list[i]), M, T);
    __syncthreads();
    Best best = {-INFINITY, -1};
    for (int32_t i = threadIdx.x; i < n; i += kThreads) {
        const int32_t group = list_id(s.list[i]) / kGroup;
        float mass = 0.0f;
        for (int32_t j = 0; j < n; j++)
            if (list_id(s.list[j]) / kGroup == group) mass += s.before[j];
        best = better(best, {logf(mass) + gumbel(seed, 0x80000000ull + uint32_t(group)), group});
    }
    const int32_t group = block_best(s, best).id;
    best = {-INFINITY, -1};
    for (int32_t i = threadIdx.x; i < n; i += kThreads) {
        const int32_t v = list_id(s.list[i]);
        if (v / kGroup == group) best = better(best, {scaled(list_value(s.list[i]), M, T) + gumbel(seed, uint32_t(v)), v});
    }
    return block_best(s, best).id;
}

// The last kept token of a prefix of the order: every token above key is kept,
// and the first `ties` of those at key, by id.
struct Cut {
    uint32_t key;
    int32_t ties;
    float mass;  // of the prefix
};

// The shortest prefix with `count` tokens (by_mass false) or a weight of at
// least target / 2^40 (by_mass true); everything when there is none.
template <typename T>
__device__ Cut radix_cut(Shared &s, const Row<T> &row, const float2 *stats, int32_t G, float M, float T_, bool by_mass,
                         uint32_t count, unsigned long long target) {
    uint32_t key = 0u;
    unsigned long long above_n = 0ull, above_mass = 0ull;
    const int lane = threadIdx.x & 31;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += kThreads) {
            s.count[i] = 0u;
            s.mass[i] = 0ull;
        }
        __syncthreads();
        for (int32_t j = threadIdx.x >> 5; j < G; j += kWarps) {
            const uint32_t top = order_key(stats[j].x);
            if (top <= kKeyNone || top < key) continue;
            for (int i = 0; i < kGroup / 32; i++) {
                const int64_t v = int64_t(j) * kGroup + i * 32 + lane;
                const float x = v < row.V ? row(int32_t(v)) : -INFINITY;
                const uint32_t k = order_key(x);
                if (x > -INFINITY && (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8)))) {
                    atomicAdd(&s.count[(k >> shift) & 255u], 1u);
                    atomicAdd(&s.mass[(k >> shift) & 255u], (unsigned long long)(double(weight(x, M, T_)) * kFixed));
                }
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int last = -1, stop = -1;
            unsigned long long n = above_n, m = above_mass;
            for (int d = 255; d >= 0 && stop < 0; d--) {
                if (!s.count[d]) continue;
                last = d;
                if (by_mass ? m + s.mass[d] >= target : n + s.count[d] >= count) {
                    stop = d;
                } else {
                    n += s.count[d];
                    m += s.mass[d];
                }
            }
            if (stop < 0 && last >= 0) {  // fewer than asked for: up to the last one there is
                stop = last;
                n -= s.count[last];
                m -= s.mass[last];
            }
            s.key = key | (uint32_t(stop < 0 ? 0 : stop) << shift);
            s.above = n;
            s.total = m;
            s.ties = stop < 0 ? 0 : int32_t(s.count[stop]);
        }
        __syncthreads();
        key = s.key;
        above_n = s.above;
        above_mass = s.total;
    }
    Cut c;
    c.key = key;
    const int32_t there = s.ties;
    const unsigned long long each = (unsigned long long)(double(weight(key_value(key), M, T_)) * kFixed);
    int32_t ties = there;
    if (by_mass) {
        if (each && target > above_mass) {
            const unsigned long long need = (target - above_mass + each - 1) / each;
            if (need < (unsigned long long)(there)) ties = int32_t(need);
        } else if (target <= above_mass) {
            ties = 1;
        }
    } else if (count > above_n && count - above_n < (unsigned long long)(there)) {
        ties = int32_t(count - above_n);
    }
    c.ties = ties < 1 ? 1 : ties;
    c.mass = float((double(above_mass) + double(c.ties) * double(each)) / kFixed);
    __syncthreads();
    return c;
}

// The id of the cut.ties-th token at cut.key.
template <typename T>
__device__ int32_t last_tie(Shared &s, const Row<T> &row, float2 *stats, int32_t G, const Cut &cut) {
    const int lane = threadIdx.x & 31;
    for (int32_t j = threadIdx.x >> 5; j < G; j += kWarps) {
        int32_t n = 0;
        if (order_key(stats[j].x) >= cut.key)
            for (int i = 0; i < kGroup / 32; i++) {
                const int64_t v = int64_t(j) * kGroup + i * 32 + lane;
                n += __popc(__ballot_sync(~0u, v < row.V && order_key(row(int32_t(v))) == cut.key));
            }
        if (lane == 0) stats[j].y = __int_as_float(n);  // the sums of the groups are not needed any more
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int32_t left = cut.ties, group = G - 1;
        for (int32_t j0 = 0; j0 < G; j0 += 32) {
            const int32_t n = j0 + lane < G ? __float_as_int(stats[j0 + lane].y) : 0;
            int32_t upto = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int32_t y = __shfl_up_sync(~0u, upto, d);
                if (lane >= d) upto += y;
            }
            const uint32_t hit = __ballot_sync(~0u, upto >= left);
            if (hit) {
                const int at = __ffs(hit) - 1;
                group = j0 + at;
                left -= __shfl_sync(~0u, upto - n, at);
                break;
            }
            left -= __shfl_sync(~0u, upto, 31);
        }
        int32_t id = 0x7FFFFFFF;
        for (int i = 0; i < kGroup / 32 && left > 0; i++) {
            const int64_t v = int64_t(group) * kGroup + i * 32 + lane;
            const uint32_t m = __ballot_sync(~0u, v < row.V && order_key(row(int32_t(v))) == cut.key);
            const int32_t n = __popc(m);
            if (n >= left) {
                id = group * kGroup + i * 32 + int32_t(__fns(m, 0, left));
                break;
            }
            left -= n;
        }
        if (lane == 0) s.n = id;
    }
    __syncthreads();
    const int32_t id = s.n;
    __syncthreads();
    return id;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_sample_pick(SampleArgs a) {
    __shared__ Shared s;
    pdl_launch_dependents();
    pdl_wait();
    const int32_t b = blockIdx.x, G = a.G;
    const int lane = threadIdx.x & 31;
    const Way way = row_way(a, b);
    const Row<T> row = row_at<T>(a, b);
    float2 *stats = a.stats + int64_t(b) * G;
    const int64_t seed = a.seeds ? __ldg(a.seeds + b) : 0;
    float M = -INFINITY;
    for (int32_t j = threadIdx.x; j < G; j += kThreads) M = fmaxf(M, stats[j].x);
    M = block_max(s, M);
    if (M == -INFINITY) {
        if (threadIdx.x == 0) {
            a.tokens[b] = -1;
            if (a.logprobs) a.logprobs[b] = -INFINITY;
        }
        return;
    }
    float Z = 0.0f;
    for (int32_t j = threadIdx.x; j < G; j += kThreads) {
        const float2 g = stats[j];
        if (g.x > -INFINITY) Z += g.y * weight(g.x, M, way.T);
    }
    Z = block_sum(s, Z);

    int32_t token = -1;
    const bool by_k = !way.greedy && way.k > 0, by_p = !way.greedy && way.p < 1.0f;
    if ((by_k && way.k <= kListK) || (by_p && !by_k)) {
        const uint32_t from = nth_group(stats, G, by_k ? way.k : kGuess);
        const int32_t n = collect(s, row, stats, G, from);
        if (n <= kList) {
            sort_list(s, n);
            const float total = scan_list(s, n, M, way.T);
            const int32_t first = by_k ? min(way.k, n) : n;
            const float Zk = by_k ? (first < n ? s.before[first] : total) : Z;
            const float target = way.p * Zk;
            // without top-k the list has to hold the whole top-p set, or every token
            if (by_k || total >= target || from == kKeyNone) {
                if (threadIdx.x == 0) s.n = 1;
                __syncthreads();
                int32_t last = 0;
                for (int32_t i = threadIdx.x; i < first; i += kThreads)
                    if ((!by_p || s.before[i] < target) && weight(list_value(s.list[i]), M, way.T) >= way.min_p)
                        last = i + 1;
                atomicMax(&s.n, last);
                __syncthreads();
                const int32_t kept = s.n;
                token = draw_list(s, kept, M, way.T, seed);
            }
        }
    }
    if (token < 0) {
        Cut cut = {kKeyNone, 0, Z};
        int32_t last_id = 0x7FFFFFFF;
        if (by_k) cut = radix_cut(s, row, stats, G, M, way.T, false, uint32_t(way.k), 0ull);
        if (by_p) {
            const double target = double(way.p) * double(cut.mass) * kFixed;
            const Cut c = radix_cut(s, row, stats, G, M, way.T, true, 0u,
                                    target > 0.0 ? (unsigned long long)(target) : 0ull);
            if (!by_k || c.key > cut.key || (c.key == cut.key && c.ties < cut.ties)) cut = c;
        }
        const bool filtered = by_k || by_p || (!way.greedy && way.min_p > 0.0f);
        if (by_k || by_p) last_id = last_tie(s, row, stats, G, cut);
        Best best = {-INFINITY, -1};
        if (!filtered) {
            for (int32_t j = threadIdx.x; j < G; j += kThreads) {
                const float2 g = stats[j];
                if (!(g.x > -INFINITY)) continue;
                if (way.greedy) best = better(best, {g.x, j});
                else best = better(best, {logf(g.y) + scaled(g.x, M, way.T) + gumbel(seed, 0x80000000ull + uint32_t(j)), j});
            }
        } else {
            for (int32_t j = threadIdx.x >> 5; j < G; j += kWarps) {
                const uint32_t top = order_key(stats[j].x);
                if (top < cut.key || top <= kKeyNone || weight(stats[j].x, M, way.T) < way.min_p) continue;
                float mass = 0.0f;
                for (int i = 0; i < kGroup / 32; i++) {
                    const int64_t v = int64_t(j) * kGroup + i * 32 + lane;
                    const float x = v < a.V ? row(int32_t(v)) : -INFINITY;
                    const uint32_t k = order_key(x);
                    const float w = weight(x, M, way.T);
                    if (x > -INFINITY && (k > cut.key || (k == cut.key && v <= last_id)) && (x == M || w >= way.min_p)) mass += w;
                }
                mass = warp_sum(mass);
                if (mass > 0.0f) best = better(best, {logf(mass) + gumbel(seed, 0x80000000ull + uint32_t(j)), j});
            }
        }
        const int32_t group = block_best(s, best).id;
        best = {-INFINITY, -1};
        if (threadIdx.x < kGroup) {
            const int64_t v = int64_t(group) * kGroup + threadIdx.x;
            const float x = v < a.V ? row(int32_t(v)) : -INFINITY;
            const uint32_t k = order_key(x);
            if (x > -INFINITY) {
                if (way.greedy) best = {x, int32_t(v)};
                else if (!filtered || ((k > cut.key || (k == cut.key && v <= last_id)) &&
                                       (x == M || weight(x, M, way.T) >= way.min_p)))
                    best = {scaled(x, M, way.T) + gumbel(seed, uint32_t(v)), int32_t(v)};
            }
        }
        token = block_best(s, best).id;
    }
    if (threadIdx.x == 0) {
        a.tokens[b] = token;
        if (a.logprobs) a.logprobs[b] = scaled(row(token), M, way.T) - logf(Z);
    }
}

}  // namespace

}  // namespace tmk

extern "C" int64_t trie_sample_workspace(int32_t B, int32_t V) {
    if (B < 0 || V < 2 || V > tmk::kMaxV) return -1;
    return int64_t(B) * ((int64_t(V) + tmk::kGroup - 1) / tmk::kGroup) * int64_t(sizeof(float2));
}

extern "C" int trie_sample(const void *d_logits, int dtype, int64_t stride, int32_t B, int32_t V, const int64_t *d_seeds,
                           const float *d_temperature, const int32_t *d_top_k, const float *d_top_p,
                           const float *d_min_p, const uint32_t *d_mask, int32_t mask_rows, const int32_t *d_states,
                           void *d_workspace, int32_t *d_tokens, float *d_logprobs, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_logits(d_logits, dtype, stride, B, V);
    if (!*bad) bad = check_grammar(d_mask, mask_rows, d_states);
    if (!*bad && B > 65535) bad = "B must be <= 65535";
    if (!*bad && B > 0 && (!d_tokens || !d_workspace)) bad = "d_tokens / d_workspace is NULL";
    if (!*bad && (reinterpret_cast<uintptr_t>(d_workspace) & 7)) bad = "d_workspace is not aligned to 8 bytes";
    if (!*bad && B > 0 && !d_seeds) bad = "d_seeds is NULL";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (B == 0) return TRIE_OK;
    SampleArgs a;
    a.logits = d_logits;
    a.stride = stride;
    a.V = V;
    a.G = int32_t((int64_t(V) + kGroup - 1) / kGroup);
    a.seeds = d_seeds;
    a.temperature = d_temperature;
    a.top_k = d_top_k;
    a.top_p = d_top_p;
    a.min_p = d_min_p;
    a.g = make_grammar(d_mask, mask_rows, d_states, V);
    a.stats = static_cast<float2 *>(d_workspace);
    a.tokens = d_tokens;
    a.logprobs = d_logprobs;
    const dim3 grid((unsigned(a.G) + kGroupThreads / 32 - 1) / (kGroupThreads / 32), unsigned(B));
    const bool f32 = dtype == TRIE_DTYPE_F32;
    cudaError_t e = f32 ? launch_pdl_grid(k_sample_groups<float>, grid, kGroupThreads, 0, stream, a)
                        : launch_pdl_grid(k_sample_groups<__nv_bfloat16>, grid, kGroupThreads, 0, stream, a);
    if (e != cudaSuccess) return fail_launch(e, "sample groups launch");
    e = f32 ? launch_pdl(k_sample_pick<float>, B, kThreads, stream, a)
            : launch_pdl(k_sample_pick<__nv_bfloat16>, B, kThreads, stream, a);
    if (e != cudaSuccess) return fail_launch(e, "sample pick launch");
    return TRIE_OK;
}
