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
//                   group: the one pass over the logits. Rows whose top-k or
//                   top-p set may be large also get a histogram of their logits
//                   (kBins bins of 1/32, counts and weights in whole numbers so
//                   that the order of the atomics does not matter), each CTA's
//                   share stored by itself.
//  k_sample_pick    one CTA per row: M and the total weight from the groups'
//                   values, then only groups that can matter are read again.
//                   top_k <= kSmallK: the k-th largest group maximum bounds the
//                   k-th largest logit from below, so the first k are in a few
//                   groups. Otherwise the histogram tells the bin in which the
//                   kept set ends; one pass over the groups that reach that bin
//                   adds up what lies above it, exactly, and collects the bin.
//                   Either way a short list in shared memory is sorted and cut.
//                   A list that does not fit (many equal logits) and infinite
//                   logits leave the row to a radix select over all groups.
//
// What bounds it (times of calls that follow one another). One row of V 32,000:
// 11 us, two launches and the chain of block-wide steps of the pick. 256 rows of
// V 152,064 in bf16, top-k up to 64: 36 us, the pass 20 of it (78 MB at 3.9 TB/s;
// an exponent, a multiply-add and a sum for each logit are as much to issue), the
// pick 16. 64 rows of V 262,144 in f32, every kind of filter: 72 us; the pass is 25
// (the histograms' atomics), the pick 43: large kept sets are read a second time,
// and a row's steps between wait for one another. 200 rows of V 128,011, three
// quarters constrained: 70 us, bound by the free rows' pick.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <cuda_runtime.h>

#include "blackwell.cuh"
#include "logits.cuh"

namespace tmk {

namespace {

constexpr int kGroup = 256;
constexpr int kGroupThreads = 256;  // k_sample_groups
constexpr int kThreads = 512;       // k_sample_pick
constexpr int kMostCtas = 4;        // of a row in k_sample_pick
constexpr int kWarps = kThreads / 32;
constexpr int kList = 4096;
// A longer list is narrowed before it is sorted: 64 rows of V 262,144, mixed
// filters: 74 us, 95 when every list is sorted as it is.
constexpr int kNarrow = 128;
// Largest top-k that goes without a histogram: 256 rows of V 152,064, top-k up to
// 64: 37 us, with histograms 108; one row of V 32,000: 11 and 27.
constexpr int kSmallK = 64;
constexpr int kBins = 2048;
constexpr float kBinsPerUnit = 32.0f;
constexpr int kChunk = 256;         // most groups of a CTA of k_sample_groups: 2^16 tokens
constexpr int kQuad = 4;            // groups that a warp takes at a time
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr uint32_t kKeyNone = 0x007FFFFFu;  // order_key(-inf)

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
    float2 *stats;            // [B][G] largest logit (never -0), sum of weights (relative to it)
    float *bound;             // [B][G] what a group's score in the draw is not above
    uint32_t *hist;           // [B][parts][2][kBins] counts, weights
    int32_t chunk, parts;     // groups of a CTA, CTAs of a row in k_sample_groups
    int32_t ctas;             // of a row in k_sample_pick: a cluster
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
    // to where log2(e) / T is a number above 0: else 0 * inf would make NaNs of weights
    w.T = fminf(fmaxf(w.T, 0x1p-126f), 0x1.fffffep127f);
    w.k = a.top_k ? __ldg(a.top_k + b) : 0;
    if (w.k < 0 || w.k >= a.V) w.k = 0;
    w.p = a.top_p ? __ldg(a.top_p + b) : 1.0f;
    if (!(w.p < 1.0f)) w.p = 1.0f;
    w.min_p = a.min_p ? __ldg(a.min_p + b) : 0.0f;
    if (!(w.min_p > 0.0f)) w.min_p = 0.0f;
    if (w.min_p > 1.0f) w.k = 1, w.min_p = 0.0f;  // above every weight: only the first token, which is always kept
    return w;
}

// Rows that get a histogram: the k-th largest of G group maxima says little
// where k is large or there are fewer groups.
__device__ __forceinline__ bool wants_hist(const Way &w, int32_t G) {
    return !w.greedy && (w.k > min(kSmallK, G) || (w.p < 1.0f && w.k == 0));
}

// Bins of logits, the largest first: non-increasing in x, so a token of an
// earlier bin is above every token of a later one. The bins lie around the
// largest logit of the row's first group, which the row's largest is not below.
struct Bins {
    float top;
    __device__ __forceinline__ explicit Bins(float first) {
        top = (fabsf(first) <= 3.0e38f ? first : 0.0f) + float(kBins / 2) / kBinsPerUnit;
    }
    __device__ __forceinline__ float place(float x) const { return (top - x) * kBinsPerUnit; }
    __device__ __forceinline__ int32_t bin(float x) const {
        return int32_t(fminf(fmaxf(place(x), 0.0f), float(kBins - 1)));
    }
};

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

// Elementwise maximum of two pairs of bf16.
__device__ __forceinline__ uint32_t max2_bf16(uint32_t a, uint32_t b) {
    const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&m);
}

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
// (Floats in the order of signed whole numbers: the lower 31 bits of negative ones turned.)
__device__ __forceinline__ float warp_max(float x) {
    int32_t k = __float_as_int(x);
    k ^= (k >> 31) & 0x7FFFFFFF;
    k = __reduce_max_sync(~0u, k);
    return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF));
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

struct Shared {
    unsigned long long list[kList];     // order_key << 32 | ~id
    union {
        struct {
            float weight[kList];        // of the list's entries
            float before[kList];        // of those before each entry
        };
        unsigned long long sub[kList];  // a part of the list
        struct {
            uint32_t count[kBins];
            float mass[kBins];
        } hist;
        struct {
            uint32_t count[kThreads], mass[kThreads], rest[kThreads];
        } fine;
        struct {
            uint32_t count[256];
            unsigned long long mass[256];
        } radix;
    };
    Best best[kWarps];
    float f[kWarps], g[kWarps];
    int32_t i[kWarps];
    int32_t n;
    int32_t bin[2];
    uint32_t key;
    int32_t ties;
    unsigned long long above, total;
    // what the CTAs of a cluster are to do, and, of the first one's, what the others found
    float least, upper, largest;
    int32_t more;  // 0: nothing, 1: the list, 2: and the weight above it
    float mass[kMostCtas];
};

// Over the block: every warp reduces the warps' values once more, so that one
// barrier after they are written is enough (and one before, for the last use).
static_assert(kWarps == 16, "half a warp reads the warps' values");
__device__ __forceinline__ Best block_best(Shared &s, Best x) {
    x = warp_best(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.best[threadIdx.x >> 5] = x;
    __syncthreads();
    x = s.best[threadIdx.x & 15];
#pragma unroll
    for (int d = 8; d; d >>= 1) {
        Best y;
        y.score = __shfl_xor_sync(~0u, x.score, d);
        y.id = __shfl_xor_sync(~0u, x.id, d);
        x = better(x, y);
    }
    return x;
}
// The largest a and the smallest b.
__device__ __forceinline__ void block_range(Shared &s, float &a, float &b) {
    a = warp_max(a);
    b = -warp_max(-b);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.f[threadIdx.x >> 5] = a, s.g[threadIdx.x >> 5] = b;
    __syncthreads();
    a = s.f[threadIdx.x & 15];
    b = s.g[threadIdx.x & 15];
#pragma unroll
    for (int d = 8; d; d >>= 1) {
        a = fmaxf(a, __shfl_xor_sync(~0u, a, d));
        b = fminf(b, __shfl_xor_sync(~0u, b, d));
    }
}
__device__ __forceinline__ float block_sum(Shared &s, float x) {
    x = warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.f[threadIdx.x >> 5] = x;
    __syncthreads();
    x = s.f[threadIdx.x & 15];
#pragma unroll
    for (int d = 8; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}
// Sums over the threads before this one, of a count and a weight.
__device__ __forceinline__ void block_scan(Shared &s, int32_t &n, float &m) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t n0 = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t y = __shfl_up_sync(~0u, n, d);
        const float z = __shfl_up_sync(~0u, m, d);
        if (lane >= d) n += y, m += z;
    }
    __syncthreads();
    if (lane == 31) s.i[warp] = n, s.f[warp] = m;
    __syncthreads();
    int32_t nw = s.i[lane & 15];
    float mw = s.f[lane & 15];
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        const int32_t y = __shfl_up_sync(~0u, nw, d);
        const float z = __shfl_up_sync(~0u, mw, d);
        if ((lane & 15) >= d) nw += y, mw += z;
    }
    nw = __shfl_sync(~0u, nw, (warp + 15) & 15);
    mw = __shfl_sync(~0u, mw, (warp + 15) & 15);
    // before this thread within the warp, and the warps before
    n += (warp ? nw : 0) - n0;
    const float upto = __shfl_up_sync(~0u, m, 1);
    m = (lane ? upto : 0.0f) + (warp ? mw : 0.0f);
}

// The sums over the warp of two values, that of v[g] in lanes 16 g to 16 g + 15.
__device__ __forceinline__ float warp_sums(const float (&v)[2], int lane) {
    const bool high = lane & 16;
    float x = (high ? v[1] : v[0]) + __shfl_xor_sync(~0u, high ? v[0] : v[1], 16);
#pragma unroll
    for (int d = 8; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}
// The sums over the warp of four values, in six exchanges: that of v[g] in lanes
// 8 g to 8 g + 7.
__device__ __forceinline__ float warp_sums(const float (&v)[4], int lane) {
    const bool high = lane & 16, odd = lane & 8;
    const float a = (high ? v[2] : v[0]) + __shfl_xor_sync(~0u, high ? v[0] : v[2], 16);
    const float b = (high ? v[3] : v[1]) + __shfl_xor_sync(~0u, high ? v[1] : v[3], 16);
    float x = (odd ? b : a) + __shfl_xor_sync(~0u, odd ? a : b, 8);
#pragma unroll
    for (int d = 4; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

// A group's logits, eight a lane: token id(i) of the group in x[i], -inf where
// not allowed or past the end. Whole groups of rows without a grammar are read 16
// bytes at a time: as they lie where the row is on a 16-byte boundary (kWide);
// bf16 rows on any other boundary as the two aligned blocks that hold a lane's
// eight logits, shifted (kShifted: each block read holds a logit of the group,
// so no read leaves the 16-byte blocks of the row). The rest is read by elements.
enum : int { kByElement = 0, kWide = 1, kShifted = 2 };
// kAligned: every row of the batch is on a 16-byte boundary (256 such rows of V 152,064
// in bf16: 37 us, 39 by the general form).
template <typename T, bool kAligned = false>
struct GroupLoad {
    const T *x;
    GrammarRow allow;
    int32_t V;
    int mode;
    int shift;  // kShifted: elements from an aligned block's start to the row's
    __device__ __forceinline__ explicit GroupLoad(const Row<T> &row)
        : x(row.x), allow(row.allow), V(row.V), mode(kByElement), shift(int(reinterpret_cast<uintptr_t>(row.x) & 15) / int(sizeof(T))) {
        if (row.allow.kind == kAllowAll) mode = kAligned || shift == 0 ? kWide : sizeof(T) == 2 ? kShifted : kByElement;
    }
    __device__ __forceinline__ int32_t id(int i, int lane) const {
        if (mode == kByElement) return i * 32 + lane;
        return sizeof(T) == 2 ? lane * 8 + i : (i >> 2) * 128 + lane * 4 + (i & 3);
    }
    __device__ __forceinline__ bool whole(int32_t j) const { return mode != kByElement && int64_t(j + 1) * kGroup <= V; }
    // A whole group's blocks (kWide bf16 has one).
    __device__ __forceinline__ void read(int32_t j, int lane, uint4 (&q)[2]) const {
        const uint4 *p = reinterpret_cast<const uint4 *>(x + int64_t(j) * kGroup - (!kAligned && mode == kShifted ? shift : 0)) + lane;
        q[0] = __ldg(p);
        if (sizeof(T) == 4) q[1] = __ldg(p + 32);
        else if (!kAligned && mode == kShifted) q[1] = __ldg(p + 1);
    }
    // The lane's eight logits as they are stored: eight words, or four of two.
    __device__ __forceinline__ void words(const uint4 (&q)[2], uint32_t (&w)[8]) const {
        w[0] = q[0].x, w[1] = q[0].y, w[2] = q[0].z, w[3] = q[0].w, w[4] = q[1].x, w[5] = q[1].y, w[6] = q[1].z, w[7] = q[1].w;
        if (sizeof(T) == 2 && !kAligned && mode == kShifted) {
            if (shift & 4) {
#pragma unroll
                for (int i = 0; i < 6; i++) w[i] = w[i + 2];
            }
            if (shift & 2) {
#pragma unroll
                for (int i = 0; i < 5; i++) w[i] = w[i + 1];
            }
            if (shift & 1) {
#pragma unroll
                for (int i = 0; i < 4; i++) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
            }
        }
    }
    static __device__ __forceinline__ float value(const uint32_t (&w)[8], int i) {
        return __uint_as_float(sizeof(T) == 4 ? w[i] : i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ void decode(const uint4 (&q)[2], float (&f)[8]) const {
        uint32_t w[8];
        words(q, w);
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = fmaxf(value(w, i), -INFINITY);  // NaN counts as -inf
    }
    __device__ __forceinline__ void by_element(int32_t j, int lane, float (&f)[8]) const {
        const int64_t v0 = int64_t(j) * kGroup;
        if (allow.kind == kAllowAll) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const int64_t v = v0 + id(i, lane);
                f[i] = v < V ? to_f32(x[v]) : -INFINITY;
            }
        } else {
            const int32_t left = (V - int32_t(v0) + 31) >> 5;  // words of the mask from here on
            const uint32_t words = lane < 8 && lane < left ? allow.word(int32_t(v0 >> 5) + lane) : 0u;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t word = __shfl_sync(~0u, words, i);
                f[i] = -INFINITY;
                if (word) {  // the whole warp's
                    const int64_t v = v0 + i * 32 + lane;
                    if (((word >> lane) & 1u) && v < V) f[i] = to_f32(x[v]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = fmaxf(f[i], -INFINITY);
    }
    __device__ __forceinline__ void operator()(int32_t j, int lane, float (&f)[8]) const {
        if (whole(j)) {
            uint4 q[2] = {};
            read(j, lane, q);
            decode(q, f);
        } else {
            by_element(j, lane, f);
        }
    }
};

// ------------------------------------------------------------ the one pass

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Sum of exp((x - m) c') of a lane's eight logits, c' in powers of two; an
// infinite m is shared by the logits that are it.
__device__ __forceinline__ float lane_weight(const float (&x)[8], float m, float c) {
    float sum = 0.0f;
    if (fabsf(m) <= 3.0e38f) {
#pragma unroll
        for (int i = 0; i < 8; i++) sum += exp2_fast((x[i] - m) * c);
    } else if (m > -INFINITY) {
#pragma unroll
        for (int i = 0; i < 8; i++) sum += x[i] == m ? 1.0f : exp2_fast((x[i] - m) * c);
    }
    return sum;
}
__device__ __forceinline__ float lane_max(const float (&x)[8]) {
    return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}
// The same of words as they are stored (NaN does not show).
template <typename T>
__device__ __forceinline__ float words_max(const uint32_t (&w)[8]) {
    if (sizeof(T) == 4) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = __uint_as_float(w[i]);
        return fmaxf(lane_max(x), -INFINITY);
    }
    const uint32_t m = max2_bf16(max2_bf16(w[0], w[1]), max2_bf16(w[2], w[3]));
    return fmaxf(fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u)), -INFINITY);
}

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kGroupThreads, 3) k_sample_groups(SampleArgs a) {
    __shared__ __align__(16) uint32_t hist[2 * kBins];  // counts, weights
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t b = blockIdx.y;
    const GroupLoad<T, kAligned> load(row_at<T>(a, b));
    const int32_t j0 = int32_t(blockIdx.x) * a.chunk, j1 = min(a.G, j0 + a.chunk);
    // Some groups a warp at a time, those of the next turn asked for ahead: four where
    // they are one load each (aligned bf16: 256 rows of V 152,064 37 us, two: 39), else
    // two (four would leave room for two CTAs an SM: 200 unaligned rows 73 us and 69).
    constexpr int kTake = sizeof(T) == 2 && kAligned ? 4 : 2, kStep = kGroupThreads / 32 * kTake;
    uint4 q[kTake][2] = {};
    auto all_whole = [&](int32_t j) { return j + kTake <= j1 && load.whole(j + kTake - 1); };
    auto read = [&](int32_t j) {
        if (!all_whole(j)) return;
#pragma unroll
        for (int g = 0; g < kTake; g++) load.read(j + g, lane, q[g]);
    };
    read(j0 + warp * kTake);
    const Way way = row_way(a, b);
    const float c = __fdiv_rn(kLog2e, way.T);
    const bool binned = wants_hist(way, a.G);
    Bins bins(0.0f);
    if (binned) {
        for (int i = threadIdx.x; i < 2 * kBins; i += kGroupThreads) hist[i] = 0u;
        float x[8];
        load(0, lane, x);
        bins = Bins(warp_max(lane_max(x)));
        __syncthreads();
    }
    auto add_bins = [&](const float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (x[i] == -INFINITY) continue;
            const float place = bins.place(x[i]);
            const int32_t bin = bins.bin(x[i]);
            if (way.k) atomicAdd(&hist[bin], 1u);
            // the weight relative to the bin's upper end: below 2^16, at most 2^16 tokens a CTA
            if (way.p < 1.0f) {
                const float w = exp2_fast((float(bin) - place) * (c / kBinsPerUnit));
                atomicAdd(&hist[kBins + bin], uint32_t(fminf(w, 1.0f) * 65535.0f + 0.5f));
            }
        }
    };
    float2 *stats = a.stats + int64_t(b) * a.G;
    if (load.allow.kind != kAllowAll) {
        // most words of a mask are empty: a lane a word of four groups
        for (int32_t j = j0 + warp * 4; j < j1; j += kGroupThreads / 32 * 4) {
            const int64_t w = int64_t(j) * (kGroup / 32) + lane;
            const uint32_t any = __ballot_sync(~0u, w < a.g.W && load.allow.word(int32_t(w)));
            float2 mine = make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int g = 0; g < 4; g++) {
                if (!((any >> (8 * g)) & 255u) || j + g >= j1) continue;
                float x[8];
                load.by_element(j + g, lane, x);
                const float m = warp_max(lane_max(x));
                const float sum = warp_sum(lane_weight(x, m, c));
                if (lane == g) mine = make_float2(m + 0.0f, sum);
                if (binned) add_bins(x);
            }
            if (lane < 4 && j + lane < j1) stats[j + lane] = mine;
        }
    } else {
        for (int32_t j = j0 + warp * kTake; j < j1; j += kStep) {
            float m[kTake], sum[kTake];
            uint32_t w[kTake][8];
            const bool whole = all_whole(j);
            if (whole) {
#pragma unroll
                for (int g = 0; g < kTake; g++) load.words(q[g], w[g]);
                read(j + kStep);
                // exp((x - m) / T) as 2^(x c - m c): the product m c is rounded, which its
                // remainder, where small (its square is left out: 2^-23 of the sum at 2^-11),
                // makes good for the whole group. A larger one, NaN and infinities make the sum
                // NaN: it is then taken again with care.
#pragma unroll
                for (int g = 0; g < kTake; g++) {
                    m[g] = warp_max(words_max<T>(w[g]));
                    const float mc = m[g] > -INFINITY ? m[g] * c : 0.0f;
                    float part = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; i++) part += exp2_fast(fmaf(load.value(w[g], i), c, -mc));
                    const float rest = fmaf(m[g], c, -mc);
                    sum[g] = !(m[g] > -INFINITY) ? part : fabsf(rest) <= 0x1p-11f ? part - part * (rest * 0.6931471806f) : NAN;
                }
            } else {
                read(j + kStep);
#pragma unroll
                for (int g = 0; g < kTake; g++) sum[g] = NAN;
            }
            float total = warp_sums(sum, lane);
            const bool again = __any_sync(~0u, !(total >= 0.0f));
            if (again || binned) {
#pragma unroll
                for (int g = 0; g < kTake; g++) {
                    if (j + g >= j1) continue;
                    float x[8];
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < 8; i++) x[i] = fmaxf(load.value(w[g], i), -INFINITY);
                    } else {
                        load(j + g, lane, x);
                    }
                    if (again) {
                        m[g] = warp_max(lane_max(x));
                        sum[g] = lane_weight(x, m[g], c);
                    }
                    if (binned) add_bins(x);
                }
                if (again) total = warp_sums(sum, lane);
            }
            const int mine = lane / (32 / kTake);
            if (lane % (32 / kTake) == 0 && j + mine < j1) {
                const float largest = mine & 2 ? (mine & 1 ? m[kTake - 1] : m[kTake - 2]) : (mine & 1 ? m[1] : m[0]);
                stats[j + mine] = make_float2(largest + 0.0f, total);
            }
        }
    }
    if (binned) {
        __syncthreads();
        uint4 *to = reinterpret_cast<uint4 *>(a.hist + (int64_t(b) * a.parts + blockIdx.x) * 2 * kBins);
        for (int i = threadIdx.x; i < 2 * kBins / 4; i += kGroupThreads) to[i] = reinterpret_cast<uint4 *>(hist)[i];
    }
}

// ------------------------------------------------------------ one row's draw

// A lower bound, finite, of the m-th largest group maximum (m >= 1), and so of the
// m-th largest logit; of every logit when fewer groups have a token. `low`: the
// smallest maximum of those that have.
__device__ __forceinline__ float nth_group(Shared &s, const float2 *stats, int32_t G, int32_t m, float M, float low) {
    if (!(M <= 3.0e38f && low >= -3.0e38f) || M - low < 1e-30f) {  // no intervals between them: are there m at all?
        int32_t there = 0;
        for (int32_t j0 = 0; j0 < G && there < m; j0 += kThreads)
            there += __syncthreads_count(j0 + int32_t(threadIdx.x) < G && stats[j0 + threadIdx.x].x > -INFINITY);
        return there < m ? kLowest : fminf(low, -kLowest);
    }
    const float per = float(kThreads - 1) / (M - low);
    __syncthreads();
    s.fine.count[threadIdx.x] = 0u;
    if (threadIdx.x == 0) s.bin[0] = kThreads;
    __syncthreads();
    for (int32_t j = threadIdx.x; j < G; j += kThreads) {
        const float x = stats[j].x;
        if (x > -INFINITY) atomicAdd(&s.fine.count[min(kThreads - 1, int32_t((M - x) * per))], 1u);
    }
    __syncthreads();
    const int32_t mine = int32_t(s.fine.count[threadIdx.x]);
    int32_t before = mine;
    float none = 0.0f;
    block_scan(s, before, none);
    if (before < m && before + mine >= m) s.bin[0] = int32_t(threadIdx.x);
    __syncthreads();
    const int32_t bin = s.bin[0];
    if (bin >= kThreads) return kLowest;
    // every maximum of the bin or an earlier one is above this (a unit of rounding further down)
    const float edge = M - float(bin + 1) / per;
    return fmaxf(low, edge - 1e-6f * (fabsf(M) + fabsf(low)));
}

// Appends the ids of the tokens of the groups j whose bits of `in` are set (bits
// 8 g .. 8 g + 7: the lane's logits of group j[g]) to s.list; s.n counts on past
// kList.
template <typename T>
__device__ __forceinline__ void append(Shared &s, const GroupLoad<T> &load, const int32_t (&j)[kQuad], uint32_t in, int lane) {
    const int32_t mine = __popc(in);
    const uint32_t who = __ballot_sync(~0u, mine);
    if (!who) return;
    int32_t upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t y = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += y;
    }
    int32_t at = 0;
    if (lane == 31) at = atomicAdd(&s.n, upto);
    at = __shfl_sync(~0u, at, 31) + upto - mine;
    for (; in; in &= in - 1, at++) {
        const int bit = __ffs(in) - 1, g = bit >> 3;
        const int32_t group = g & 2 ? (g & 1 ? j[3] : j[2]) : (g & 1 ? j[1] : j[0]);
        if (at < kList) s.list[at] = uint32_t(group * kGroup + load.id(bit & 7, lane));
    }
}

// The ids in s.list to entries.
template <typename T>
__device__ __forceinline__ void fill_list(Shared &s, const Row<T> &row, int32_t n) {
    for (int32_t i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t id = uint32_t(s.list[i]);
        s.list[i] = (uint64_t(order_key(clean(to_f32(row.x[id])))) << 32) | uint32_t(~id);
    }
}

// The next four groups of a warp's `todo` (bit i: group j0 + stride i; -1 where
// there are no more) and their logits, all asked for before the first is used.
template <typename T>
__device__ __forceinline__ void take_quad(const GroupLoad<T> &load, uint32_t &todo, int32_t j0, int32_t stride, int lane,
                                          int32_t (&j)[kQuad], float (&x)[kQuad][8]) {
    uint4 q[kQuad][2] = {};
#pragma unroll
    for (int g = 0; g < kQuad; g++) {
        j[g] = todo ? j0 + (__ffs(todo) - 1) * stride : -1;
        todo &= todo - 1;
        if (j[g] >= 0 && load.whole(j[g])) load.read(j[g], lane, q[g]);
    }
#pragma unroll
    for (int g = 0; g < kQuad; g++) {
        if (j[g] >= 0 && !load.whole(j[g])) load.by_element(j[g], lane, x[g]);
        else load.decode(q[g], x[g]);
    }
}

// Collects every allowed token with a logit of at least `least` (finite) into
// s.list; returns how many there are (more than kList: only that many were stored).
template <typename T>
__device__ __forceinline__ int32_t collect(Shared &s, const GroupLoad<T> &load, const float2 *stats, int32_t G, float least) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    // a warp looks at 32 groups' maxima at a time, every 16th group so that crowds are shared
    for (int32_t j0 = 0; j0 < G; j0 += 32 * kWarps) {
        const int32_t mine = j0 + lane * kWarps + warp;
        uint32_t todo = __ballot_sync(~0u, mine < G && stats[mine].x >= least);
        while (todo) {
            int32_t j[kQuad];
            float x[kQuad][8];
            take_quad(load, todo, j0 + warp, kWarps, lane, j, x);
            uint32_t in = 0;
#pragma unroll
            for (int g = 0; g < kQuad; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) in |= uint32_t(j[g] >= 0 && x[g][i] >= least) << (8 * g + i);
            append(s, load, j, in, lane);
        }
    }
    __syncthreads();
    return s.n;
}

// Sorts s.list[0, n) in descending order: by each entry's rank where few, with
// up to 16 threads an entry, else by a bitonic network over the next power of two.
__device__ __forceinline__ void sort_list(Shared &s, int32_t n) {
    if (n <= kThreads) {
        int32_t each = 16;  // threads an entry
        while (each > 1 && n * each > kThreads) each >>= 1;
        const int32_t at = int32_t(threadIdx.x) / each, part = int32_t(threadIdx.x) & (each - 1);
        __syncthreads();
        const unsigned long long mine = at < n ? s.list[at] : 0ull;
        int32_t rank = 0;
        if (at < n)
            for (int32_t i = part; i < n; i += each) rank += s.list[i] > mine;
        for (int32_t d = each >> 1; d; d >>= 1) rank += __shfl_xor_sync(~0u, rank, d);
        __syncthreads();
        if (at < n && part == 0) s.list[rank] = mine;
        __syncthreads();
        return;
    }
    int32_t size = 2;
    while (size < n) size <<= 1;
    for (int32_t i = n + int32_t(threadIdx.x); i < size; i += kThreads) s.list[i] = 0ull;
    for (int32_t k = 2; k <= size; k <<= 1) {
        for (int32_t d = k >> 1; d; d >>= 1) {
            __syncthreads();
            for (int32_t i = threadIdx.x; i < size / 2; i += kThreads) {
                const int32_t lo = ((i & ~(d - 1)) << 1) | (i & (d - 1)), hi = lo + d;
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

// s.weight[i] = weight of s.list[i], s.before[i] = that of s.list[0, i); returns
// the whole list's weight. One thread's share is consecutive entries, so the
// sums' order is fixed.
__device__ __forceinline__ float scan_list(Shared &s, int32_t n, float M, float T) {
    for (int32_t i = threadIdx.x; i < n; i += kThreads) s.weight[i] = weight(list_value(s.list[i]), M, T);
    __syncthreads();
    const int32_t per = (n + kThreads - 1) / kThreads, first = int32_t(threadIdx.x) * per;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float sum = 0.0f;
    for (int32_t i = first; i < min(n, first + per); i++) sum += s.weight[i];
    float upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const float y = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += y;
    }
    float before = __shfl_up_sync(~0u, upto, 1);
    if (lane == 0) before = 0.0f;
    if (lane == 31) s.f[warp] = upto;
    __syncthreads();
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < kWarps; i++) {
        if (i == warp) before += total;
        total += s.f[i];
    }
    for (int32_t i = first; i < min(n, first + per); i++) {
        s.before[i] = before;
        before += s.weight[i];
    }
    __syncthreads();
    return total;
}

// How many of the first n entries of the sorted, scanned list are kept: those
// before which the weight, `above` included, is below target.
__device__ __forceinline__ int32_t cut_list(Shared &s, int32_t n, float above, float target) {
    __syncthreads();
    if (threadIdx.x == 0) s.n = 1;
    __syncthreads();
    int32_t last = 0;
    for (int32_t i = threadIdx.x; i < n; i += kThreads)
        if (above + s.before[i] < target) last = i + 1;
    if (last) atomicMax(&s.n, last);
    __syncthreads();
    n = s.n;
    __syncthreads();
    return n;
}

// The group drawn where only tokens with entry >= last (order_key << 32 | ~id) and
// w >= min_p are kept. A group's score is not above what it would be with all its
// tokens, so the kept weights of a few groups settle the draw: each warp looks at
// the best bounds of its groups until none is above the best score found.
template <typename T>
__device__ __forceinline__ int32_t draw_group(Shared &s, const GroupLoad<T> &load, const float2 *stats, float *bound, int32_t G,
                                              unsigned long long last, float min_p, float M, float T_, int64_t seed) {
    constexpr float kRounding = 2e-5f;  // of a score: sums of logarithms and noise below 64 in 24 bits
    const int lane = threadIdx.x & 31;
    const float c = __fdiv_rn(kLog2e, T_);
    for (int32_t j = threadIdx.x; j < G; j += kThreads) {
        const float2 g = stats[j];
        bound[j] = g.x > -INFINITY ? logf(g.y) + scaled(g.x, M, T_) + gumbel(seed, 0x80000000ull + uint32_t(j)) + kRounding
                                   : -INFINITY;
    }
    Best found = {-INFINITY, -1};
    for (;;) {
        Best next = {-INFINITY, -1};  // of this warp's groups: those of its threads
        for (int32_t j = threadIdx.x; j < G; j += kThreads) next = better(next, {bound[j], j});
        next = warp_best(next);
        const bool look = next.score > -INFINITY && next.score >= found.score;
        Best mine = {-INFINITY, -1};
        if (look) {
            float x[8], mass = 0.0f;
            load(next.id, lane, x);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const unsigned long long entry = (uint64_t(order_key(x[i] + 0.0f)) << 32) |
                                                 uint32_t(~uint32_t(next.id * kGroup + load.id(i, lane)));
                const float w = x[i] == M ? 1.0f : exp2_fast((x[i] - M) * c);
                if (x[i] > -INFINITY && entry >= last && w >= min_p) mass += w;
            }
            mass = warp_sum(mass);
            if (mass > 0.0f) mine = {logf(mass) + gumbel(seed, 0x80000000ull + uint32_t(next.id)), next.id};
            if ((next.id & 31) == lane) bound[next.id] = -INFINITY;  // its thread's own
        }
        found = better(found, block_best(s, mine));
        if (!__syncthreads_or(look)) return found.id;
    }
}

// Of the first n (at most kSmallK) entries of the sorted list, by one warp, an
// entry a lane and the next 32 in the lane's second place: top-p, min_p, the draw.
__device__ __forceinline__ int32_t draw_small(Shared &s, int32_t n, const Way &way, float M, int64_t seed, int lane) {
    float w[2], y[2], before[2];
    int32_t id[2], group[2];
    float total = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int32_t at = h * 32 + lane;
        const unsigned long long e = at < n ? s.list[at] : 0ull;
        id[h] = list_id(e);
        group[h] = at < n ? id[h] / kGroup : -1;
        y[h] = at < n ? scaled(list_value(e), M, way.T) : -INFINITY;
        w[h] = at < n ? exp2f(y[h] * kLog2e) : 0.0f;
        float upto = w[h];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const float z = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += z;
        }
        const float prev = __shfl_up_sync(~0u, upto, 1);
        before[h] = total + (lane ? prev : 0.0f);
        total += __shfl_sync(~0u, upto, 31);
    }
    const float target = way.p < 1.0f ? way.p * total : INFINITY;
    // what is kept is a prefix
    const uint32_t in0 = __ballot_sync(~0u, lane < n && before[0] < target && w[0] >= way.min_p);
    const uint32_t in1 = __ballot_sync(~0u, lane + 32 < n && before[1] < target && w[1] >= way.min_p);
    const int32_t kept = max(1, in1 ? 64 - __clz(in1) : 32 - __clz(in0));
    float mass[2] = {0.0f, 0.0f};
#pragma unroll
    for (int h = 0; h < 2; h++) {
        s.weight[h * 32 + lane] = w[h];
        s.before[h * 32 + lane] = __int_as_float(h * 32 + lane < kept ? group[h] : -2);
    }
    __syncwarp();
#pragma unroll 8
    for (int32_t i = 0; i < (kept + 7 & ~7); i++) {  // (a -2 is no entry's group)
        const float wi = s.weight[i];
        const int32_t gi = __float_as_int(s.before[i]);
        if (group[0] == gi) mass[0] += wi;
        if (group[1] == gi) mass[1] += wi;
    }
    Best best = {-INFINITY, -1};
#pragma unroll
    for (int h = 0; h < 2; h++)
        if (h * 32 + lane < kept)
            best = better(best, {logf(mass[h]) + gumbel(seed, 0x80000000ull + uint32_t(group[h])), group[h]});
    const int32_t drawn = warp_best(best).id;
    best = {-INFINITY, -1};
#pragma unroll
    for (int h = 0; h < 2; h++)
        if (h * 32 + lane < kept && group[h] == drawn) best = better(best, {y[h] + gumbel(seed, uint32_t(id[h])), id[h]});
    return warp_best(best).id;
}

// Where the list is long: its tokens from `least` to below `above` are counted and,
// where `weigh`, weighed (relative to `top`, the weight at `above`) by 512 equal
// intervals, and the one in which the kept set ends becomes the list; n_above and
// mass grow by what lies before it. By count, or by weight (count < 0). Returns the
// list's length. Weights are whole numbers of 2^-39 `top`, in two parts, so that the
// order of the atomics does not matter: of those down to kSpan powers of two below
// `top` that leaves 27 bits, more than a sum in 32 bits keeps.
// width > 0: the tokens are all equal, of weight `top`, and go by `width` ids.
constexpr float kSpan = 12.0f;
__device__ __forceinline__ int32_t narrow(Shared &s, int32_t n, float least, float above, float top, float c, bool weigh,
                                          int32_t count, float target, int32_t width, int32_t &n_above, float &mass) {
    const float per = float(kThreads) / (above - least);
    __syncthreads();
    s.fine.count[threadIdx.x] = s.fine.mass[threadIdx.x] = s.fine.rest[threadIdx.x] = 0u;
    if (threadIdx.x == 0) s.bin[0] = kThreads, s.ties = 0;
    __syncthreads();
    auto place = [&](unsigned long long e) {
        return width ? list_id(e) / width : max(0, min(kThreads - 1, int32_t((above - list_value(e)) * per)));
    };
    for (int32_t i = threadIdx.x; i < n; i += kThreads) {
        const float x = list_value(s.list[i]);
        const int32_t at = place(s.list[i]);
        atomicAdd(&s.fine.count[at], 1u);
        if (weigh && !width) {  // kList of either part fit
            const float w = fminf(exp2_fast((x - above) * c), 1.0f) * 0x1p19f;
            const uint32_t whole = uint32_t(w);
            atomicAdd(&s.fine.mass[at], whole);
            atomicAdd(&s.fine.rest[at], uint32_t((w - float(whole)) * 0x1p20f));
        }
    }
    __syncthreads();
    const int32_t mine = int32_t(s.fine.count[threadIdx.x]);
    const float weighed = (float(s.fine.mass[threadIdx.x]) + float(s.fine.rest[threadIdx.x]) * 0x1p-20f) * (top * 0x1p-19f);
    const float weighs = width ? float(mine) * top : weighed;
    int32_t n_before = mine;
    float m_before = weighs;
    block_scan(s, n_before, m_before);
    const bool reached = count >= 0 ? n_above + n_before + mine >= count : mass + (m_before + weighs) >= target;
    if (mine && reached) atomicMin(&s.bin[0], int32_t(threadIdx.x));
    if (mine) atomicMax(&s.ties, int32_t(threadIdx.x));
    __syncthreads();
    const int32_t bin = s.bin[0] < kThreads ? s.bin[0] : s.ties;
    if (int32_t(threadIdx.x) == bin) {
        s.i[0] = n_before;
        s.f[0] = m_before;
    }
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    n_above += s.i[0];
    mass += s.f[0];
    for (int32_t i = threadIdx.x; i < n; i += kThreads) {
        const unsigned long long e = s.list[i];
        if (place(e) == bin) s.sub[atomicAdd(&s.n, 1)] = e;
    }
    __syncthreads();
    n = s.n;
    for (int32_t i = threadIdx.x; i < n; i += kThreads) s.list[i] = s.sub[i];
    __syncthreads();
    return n;
}

// The smallest finite value whose bin is at most `last` (bin() does not increase
// with the value): comparing with it costs less than finding each value's bin.
__device__ __forceinline__ float bin_floor(const Bins &bins, int32_t last) {
    const uint32_t lowest = order_key(-3.4028234663852886e38f), highest = order_key(3.4028234663852886e38f);
    if (last >= kBins - 1) return key_value(lowest);
    if (last < 0) return INFINITY;
    uint32_t lo = lowest, hi = highest;  // bin(lo) > last, or lo is the answer; bin(hi) <= last
    if (bins.bin(key_value(lo)) <= last) return key_value(lo);
    // it is most likely where the arithmetic says, give or take its rounding
    const float about = bins.top - float(last + 1) / kBinsPerUnit, off = 4e-7f * (fabsf(bins.top) + fabsf(about));
    if (bins.bin(about - off) > last && bins.bin(about + off) <= last) lo = order_key(about - off), hi = order_key(about + off);
    const uint32_t lane = threadIdx.x & 31;
    while (hi - lo > 1) {  // 33 parts at a time, a lane a border
        const uint32_t step = max(1u, (hi - lo) / 33), at = min(hi, lo + step * (lane + 1));
        const uint32_t in = __ballot_sync(~0u, bins.bin(key_value(at)) <= last);
        const uint32_t first = in ? uint32_t(__ffs(in)) : 33u;  // the borders before it are not in
        if (first <= 32) hi = min(hi, lo + step * first);
        lo += step * (first - 1);
    }
    return key_value(hi);
}

// Bit i: x[i] is at least `least` (finite) and below `above` (not NaN). By the signs of the
// differences (a difference is zero only between equal numbers, and +inf - +inf has
// no sign bit): two instructions a comparison, where a flag turned into a bit takes three.
__device__ __forceinline__ uint32_t inside(const float (&x)[8], float least, float above) {
    uint32_t under = 0u, over = 0u;
#pragma unroll
    for (int i = 7; i >= 0; i--) {
        under = __funnelshift_l(__float_as_uint(__fsub_rn(x[i], least)), under, 1);
        over = __funnelshift_l(__float_as_uint(__fsub_rn(x[i], above)), over, 1);
    }
    return ~under & over & 255u;
}

// One pass over the groups that reach `least`, by CTA `rank` of `ctas`: s.list gets
// the ids of the tokens from `least` up to below `above`. Returns the weight of
// those at or above `above` (to thread 0), 0 when it is not asked for.
template <typename T>
__device__ __forceinline__ float split_at(Shared &s, Shared &first, const GroupLoad<T> &load, const float2 *stats, int32_t G,
                                          float least, float above, bool weigh, float M, float c, int rank, int ctas) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float sum = 0.0f;
    for (int32_t j0 = 0; j0 < G; j0 += ctas * 32 * kWarps) {
        const int32_t mine = j0 + (lane * kWarps + warp) * ctas + rank;
        uint32_t todo = __ballot_sync(~0u, mine < G && stats[mine].x >= least);
        while (todo) {
            int32_t j[kQuad];
            float x[kQuad][8];
            take_quad(load, todo, j0 + warp * ctas + rank, kWarps * ctas, lane, j, x);
            uint32_t in = 0;
#pragma unroll
            for (int g = 0; g < kQuad; g++) {
                if (j[g] < 0) continue;
                in |= inside(x[g], least, above) << (8 * g);
                if (weigh) {
                    float part = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const float w = exp2_fast((x[g][i] - M) * c);
                        part += x[g][i] >= above ? w : 0.0f;
                    }
                    sum += part;
                }
            }
            append(first, load, j, in, lane);
        }
    }
    return block_sum(s, sum);
}

// Adds up the row's histograms in s.hist, weights relative to M.
__device__ __forceinline__ void sum_hist(Shared &s, const uint32_t *hist, int32_t parts, const Bins &bins, const Way &way, float M) {
    constexpr int kPer = kBins / kThreads;
    static_assert(kPer == 4, "one 16-byte load a thread and part");
    const float c = __fdiv_rn(kLog2e, way.T);
    uint32_t count[kPer] = {};
    float mass[kPer] = {};
#pragma unroll 4
    for (int32_t p = 0; p < parts; p++) {
        const uint4 *at = reinterpret_cast<const uint4 *>(hist + int64_t(p) * 2 * kBins) + threadIdx.x;
        const uint4 n = __ldcg(at), w = __ldcg(at + kBins / 4);
        count[0] += n.x, count[1] += n.y, count[2] += n.z, count[3] += n.w;
        mass[0] += float(w.x), mass[1] += float(w.y), mass[2] += float(w.z), mass[3] += float(w.w);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int bin = int(threadIdx.x) * kPer + i;
        const float end = bins.top - float(bin) / kBinsPerUnit;
        s.hist.count[bin] = count[i];
        s.hist.mass[bin] = mass[i] > 0.0f ? mass[i] / 65535.0f * exp2_fast((end - M) * c) : 0.0f;
    }
    __syncthreads();
}

// The bins [s.bin[0], s.bin[1]] in which the kept set ends: by count exactly (and
// s.ties tokens are in the bins before), by weight to within the histogram's
// precision. kBins: none found.
__device__ __forceinline__ void find_bins(Shared &s, bool by_mass, int32_t count, float target) {
    constexpr int kPer = kBins / kThreads;
    constexpr float kSlack = 1e-4f;  // weights in the histogram are rounded to 2^-16
    int32_t n = 0;
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        n += int32_t(s.hist.count[threadIdx.x * kPer + i]);
        m += s.hist.mass[threadIdx.x * kPer + i];
    }
    if (threadIdx.x == 0) s.bin[0] = s.bin[1] = kBins;
    block_scan(s, n, m);
    int32_t lo = kBins, hi = kBins;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
        const int bin = int(threadIdx.x) * kPer + i;
        n += int32_t(s.hist.count[bin]);
        m += s.hist.mass[bin];
        if (by_mass) {
            if (lo == kBins && m * (1.0f + kSlack) >= target) lo = bin;
            if (hi == kBins && m * (1.0f - kSlack) >= target) hi = bin;
        } else if (lo == kBins && n >= count) {
            lo = hi = bin;
            if (n - int32_t(s.hist.count[bin]) < count) s.ties = n - int32_t(s.hist.count[bin]);
        }
    }
    lo = __reduce_min_sync(~0u, lo);
    hi = __reduce_min_sync(~0u, hi);
    if ((threadIdx.x & 31) == 0) {
        atomicMin(&s.bin[0], lo);
        atomicMin(&s.bin[1], hi);
    }
    __syncthreads();
}

// Weights (at most 1) as whole numbers of 2^-40, or more where so many as a row has
// tokens would not fit 64 bits: V of them stay below 2^63.
__device__ __forceinline__ double fixed_one(int32_t V) { return double(1ull << min(40, 31 + __clz(V))); }

// The last kept token of a prefix of the order: every token above key is kept,
// and the first `ties` of those at key, by id.
struct Cut {
    uint32_t key;
    int32_t ties;
    float mass;  // of the prefix
};

// The shortest prefix with `count` tokens (by_mass false) or a weight of at
// least target / fixed_one (by_mass true); everything when there is none.
template <typename T>
__device__ __noinline__ Cut radix_cut(Shared &s, const Row<T> &row, const float2 *stats, int32_t G, float M, float T_, bool by_mass,
                         uint32_t count, unsigned long long target) {
    const double one = fixed_one(row.V);
    uint32_t key = 0u;
    unsigned long long above_n = 0ull, above_mass = 0ull;
    const int lane = threadIdx.x & 31;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += kThreads) {
            s.radix.count[i] = 0u;
            s.radix.mass[i] = 0ull;
        }
        __syncthreads();
        for (int32_t j = threadIdx.x >> 5; j < G; j += kWarps) {
            const uint32_t top = order_key(stats[j].x);
            if (top <= kKeyNone || top < key) continue;
            for (int i = 0; i < kGroup / 32; i++) {
                const int64_t v = int64_t(j) * kGroup + i * 32 + lane;
                const float x = v < row.V ? row(int32_t(v)) : -INFINITY;
                const uint32_t k = order_key(x);
                const bool in = x > -INFINITY && (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8)));
                const uint32_t who = __ballot_sync(~0u, in);
                if (!who) continue;
                // the lanes that share the first one's digit add up in one go: equal logits come in crowds
                const uint32_t digit = (k >> shift) & 255u, of_first = __shfl_sync(~0u, digit, __ffs(who) - 1);
                const unsigned long long w = in ? (unsigned long long)(double(weight(x, M, T_)) * one) : 0ull;
                const bool same = in && digit == of_first;
                const uint32_t crowd = __ballot_sync(~0u, same);
                unsigned long long sum = same ? w : 0ull;
#pragma unroll
                for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
                if (lane == 0) {
                    atomicAdd(&s.radix.count[of_first], uint32_t(__popc(crowd)));
                    atomicAdd(&s.radix.mass[of_first], sum);
                }
                if (in && !same) {
                    atomicAdd(&s.radix.count[digit], 1u);
                    atomicAdd(&s.radix.mass[digit], w);
                }
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int last = -1, stop = -1;
            unsigned long long n = above_n, m = above_mass;
            for (int d = 255; d >= 0 && stop < 0; d--) {
                if (!s.radix.count[d]) continue;
                last = d;
                if (by_mass ? m + s.radix.mass[d] >= target : n + s.radix.count[d] >= count) {
                    stop = d;
                } else {
                    n += s.radix.count[d];
                    m += s.radix.mass[d];
                }
            }
            if (stop < 0 && last >= 0) {  // fewer than asked for: up to the last one there is
                stop = last;
                n -= s.radix.count[last];
                m -= s.radix.mass[last];
            }
            s.key = key | (uint32_t(stop < 0 ? 0 : stop) << shift);
            s.above = n;
            s.total = m;
            s.ties = stop < 0 ? 0 : int32_t(s.radix.count[stop]);
        }
        __syncthreads();
        key = s.key;
        above_n = s.above;
        above_mass = s.total;
    }
    Cut c;
    c.key = key;
    const int32_t there = s.ties;
    const unsigned long long each = (unsigned long long)(double(weight(key_value(key), M, T_)) * one);
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
    c.mass = float((double(above_mass) + double(c.ties) * double(each)) / one);
    __syncthreads();
    return c;
}

// The id of the cut.ties-th token at cut.key.
template <typename T>
__device__ __noinline__ int32_t last_tie(Shared &s, const Row<T> &row, const float2 *stats, float *scratch, int32_t G, const Cut &cut) {
    const int lane = threadIdx.x & 31;
    for (int32_t j = threadIdx.x >> 5; j < G; j += kWarps) {
        int32_t n = 0;
        if (order_key(stats[j].x) >= cut.key)
            for (int i = 0; i < kGroup / 32; i++) {
                const int64_t v = int64_t(j) * kGroup + i * 32 + lane;
                n += __popc(__ballot_sync(~0u, v < row.V && order_key(row(int32_t(v))) == cut.key));
            }
        if (lane == 0) scratch[j] = __int_as_float(n);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int32_t left = cut.ties, group = G - 1;
        for (int32_t j0 = 0; j0 < G; j0 += 32) {
            const int32_t n = j0 + lane < G ? __float_as_int(scratch[j0 + lane]) : 0;
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
__global__ void __launch_bounds__(kThreads, 2) k_sample_pick(SampleArgs a) {
    extern __shared__ __align__(16) unsigned char dynamic_smem[];
    Shared &s = *reinterpret_cast<Shared *>(dynamic_smem);
    const int ctas = a.ctas, rank = ctas > 1 ? int(cluster_rank()) : 0;
    // A CTA's shared memory may be written by the others only once it is known to run: the
    // cluster meets behind the wait for the pass, which takes longer.
    if (ctas > 1) cluster_arrive();
    pdl_launch_dependents();
    pdl_wait();
    if (ctas > 1) cluster_wait();
    const int32_t b = int32_t(blockIdx.x) / ctas, G = a.G;
    const int lane = threadIdx.x & 31;
    const float2 *stats = a.stats + int64_t(b) * G;
    const Way way = row_way(a, b);
    const Row<T> row = row_at<T>(a, b);
    const GroupLoad<T> load(row);
    const float c = __fdiv_rn(kLog2e, way.T);
    // rows whose kept set may be large have the cluster's CTAs share the pass over the groups
    const bool shared = ctas > 1 && wants_hist(way, G);
    if (rank > 0) {
        if (!shared) return;
        Shared &first = *cluster_object(&s, 0);
        for (;;) {
            cluster_sync();  // what is to be done is in this CTA's memory
            if (!s.more) return;
            const float mass = split_at(s, first, load, stats, G, s.least, s.upper, s.more > 1, s.largest, c, rank, ctas);
            if (threadIdx.x == 0) first.mass[rank] = mass;
            cluster_sync();  // and it is done
        }
    }
    auto tell = [&](int32_t more, float least, float above, float largest) {
        __syncthreads();
        if (threadIdx.x == 0) s.n = 0;
        if (shared) {
            if (int(threadIdx.x) < ctas) {
                Shared &other = *cluster_object(&s, threadIdx.x);
                other.least = least;
                other.upper = above;
                other.largest = largest;
                other.more = more;
            }
            cluster_sync();
        } else {
            __syncthreads();
        }
    };
    float M = -INFINITY, low = INFINITY;
    for (int32_t j = threadIdx.x; j < G; j += kThreads) {
        const float x = stats[j].x;
        M = fmaxf(M, x);
        if (x > -INFINITY) low = fminf(low, x);
    }
    const int64_t seed = __ldg(a.seeds + b);
    block_range(s, M, low);
    if (M == -INFINITY) {
        if (shared) tell(0, 0.0f, 0.0f, 0.0f);
        if (threadIdx.x == 0) {
            a.tokens[b] = -1;
            if (a.logprobs) a.logprobs[b] = -INFINITY;
        }
        return;
    }
    float Z = 0.0f;
    for (int32_t j = threadIdx.x; j < G; j += kThreads) {
        const float2 g = stats[j];
        if (g.x > -INFINITY) Z += g.y * (g.x == M ? 1.0f : exp2_fast((g.x - M) * c));
    }
    Z = block_sum(s, Z);

    const bool by_p = !way.greedy && way.p < 1.0f, by_min = !way.greedy && way.min_p > 0.0f;
    bool by_k = !way.greedy && way.k > 0;
    int32_t token = -1;
    unsigned long long last = 0ull;  // tokens below this entry (order_key << 32 | ~id) are not kept
    unsigned long long kth = 0ull;   // the last of the first top_k, once known
    const Bins bins(stats[0].x);
    enum { kSmall, kCount, kMass, kNone };  // how the kept set is found: few by count, by count, by weight
    float target = way.p * Z;
    int step = by_k ? (wants_hist(way, G) ? kCount : kSmall) : by_p ? kMass : kNone;
    while (step != kNone) {
        int32_t n = 0, n_above = 0;
        float mass = 0.0f, least = kLowest, above = INFINITY, top = 1.0f;
        if (step != kSmall && M > -kLowest) break;  // infinities have no bin's end above them
        if (step == kSmall) {
            n = collect(s, load, stats, G, nth_group(s, stats, G, way.k, M, low));
        } else {
            sum_hist(s, a.hist + int64_t(b) * a.parts * 2 * kBins, a.parts, bins, way, M);
            find_bins(s, step == kMass, way.k, target);
            const int32_t begin = s.bin[0], end = s.bin[1];
            if (end >= kBins) {
                if (step == kMass) break;
                by_k = false;  // fewer tokens than top_k: it keeps all
                step = by_p ? kMass : kNone;
                continue;
            }
            n_above = s.ties;  // by count; by weight it is not used
            least = bin_floor(bins, end);
            above = bin_floor(bins, begin - 1);
            if (above < M) top = exp2_fast((above - M) * c);
            tell(by_p ? 2 : 1, least, above, M);
            mass = split_at(s, s, load, stats, G, least, above, by_p, M, c, 0, ctas);
            if (shared) {
                cluster_sync();
                for (int r = 1; r < ctas; r++) mass += s.mass[r];
            } else {
                __syncthreads();
            }
            n = s.n;
        }
        if (n > kList) break;
        fill_list(s, row, n);
        // (a list whose weights are too far apart is sorted as it is)
        const bool by_value = above < M && (!by_p || (above - least) * c <= kSpan);
        for (int by_id = by_value ? 0 : 1; step != kSmall && by_id < 2 && n > kNarrow; by_id++) {
            if (by_id) {  // bf16 logits of one value come by the thousand
                __syncthreads();
                const uint32_t key = uint32_t(s.list[0] >> 32);
                bool same = true;
                for (int32_t i = threadIdx.x; i < n; i += kThreads) same &= uint32_t(s.list[i] >> 32) == key;
                if (!__syncthreads_and(same)) break;
                top = weight(key_value(key), M, way.T);
            }
            n = narrow(s, n, least, above, top, c, by_p, step == kCount ? way.k : -1, target,
                       by_id ? (a.V + kThreads - 1) / kThreads : 0, n_above, mass);
        }
        sort_list(s, n);
        if (step == kSmall) {
            if (__shfl_sync(~0u, threadIdx.x >> 5, 0)) return;  // one warp does the rest (such a row's cluster shares nothing)
            token = draw_small(s, min(way.k, n), way, M, seed, lane);
            break;
        }
        const int32_t wanted = min(n, way.k - n_above);
        if (step == kCount) kth = s.list[wanted - 1];
        if (step == kCount && !by_p) {
            last = kth;
            break;
        }
        const float total = scan_list(s, n, M, way.T);
        if (step == kCount) {
            target = way.p * (mass + (wanted < n ? s.before[wanted] : total));
            step = kMass;
            continue;
        }
        // (top_p next to 1 may let in more than the first top_k where the two lists' sums are rounded differently)
        if (mass < target && mass + total >= target) last = max(s.list[cut_list(s, n, mass, target) - 1], kth);
        break;
    }
    if (shared) tell(0, 0.0f, 0.0f, 0.0f);
    if (step != kSmall || token < 0) {
        const bool filtered = by_k || by_p || by_min;
        if ((by_k || by_p) && last == 0ull) {
            Cut cut = {kKeyNone, 0, Z};
            for (int by = 0; by < 2; by++) {
                if (by ? !by_p : !by_k) continue;
                const double to = double(way.p) * double(cut.mass) * fixed_one(a.V);
                const Cut found = radix_cut(s, row, stats, G, M, way.T, by == 1, uint32_t(way.k),
                                            to > 0.0 ? (unsigned long long)(to) : 0ull);
                if (by == 0 || !by_k || found.key > cut.key || (found.key == cut.key && found.ties < cut.ties)) cut = found;
            }
            last = (uint64_t(cut.key) << 32) | uint32_t(~uint32_t(last_tie(s, row, stats, a.bound + int64_t(b) * G, G, cut)));
        }
        int32_t group;
        if (filtered) {
            group = draw_group(s, load, stats, a.bound + int64_t(b) * G, G, last, way.min_p, M, way.T, seed);
        } else {
            Best best = {-INFINITY, -1};
            for (int32_t j = threadIdx.x; j < G; j += kThreads) {
                const float2 g = stats[j];
                if (!(g.x > -INFINITY)) continue;
                if (way.greedy) best = better(best, {g.x, j});
                else best = better(best, {logf(g.y) + scaled(g.x, M, way.T) + gumbel(seed, 0x80000000ull + uint32_t(j)), j});
            }
            group = block_best(s, best).id;
        }
        Best best = {-INFINITY, -1};
        if (threadIdx.x < kGroup) {
            const int64_t v = int64_t(group) * kGroup + threadIdx.x;
            const float x = v < a.V ? row(int32_t(v)) : -INFINITY;
            if (x > -INFINITY) {
                const unsigned long long entry = (uint64_t(order_key(x)) << 32) | uint32_t(~uint32_t(v));
                const bool kept = !filtered || (entry >= last && (x == M || exp2_fast((x - M) * c) >= way.min_p));
                if (way.greedy) best = {x, int32_t(v)};
                else if (kept) best = {scaled(x, M, way.T) + gumbel(seed, uint32_t(v)), int32_t(v)};
            }
        }
        token = block_best(s, best).id;
    }
    if (threadIdx.x == 0) {
        a.tokens[b] = token;
        if (a.logprobs) a.logprobs[b] = scaled(row(token), M, way.T) - logf(Z);
    }
}

// How a batch is cut and where its parts of the workspace lie. A row is cut into
// the fewest parts of at most kChunk groups (16 in a small batch) whose CTAs fill
// their rounds to nine tenths, some three an SM running at once.
struct Plan {
    int32_t G, chunk, parts;
    int64_t bound_at, hist_at, bytes;
    Plan(int32_t B, int32_t V) {
        G = int32_t((int64_t(V) + kGroup - 1) / kGroup);
        constexpr int64_t kRound = 3 * 152;
        const int32_t fewest = (G + kChunk - 1) / kChunk, most = (G + 15) / 16;
        parts = int64_t(B) * most <= kRound ? most : fewest;
        double best = 0.0;
        for (int32_t p = fewest; int64_t(B) * most > kRound && p <= most && p <= fewest + 16 + int32_t(2 * kRound / B); p++) {
            const int64_t ctas = int64_t(B) * p, rounds = (ctas + kRound - 1) / kRound;
            const double full = double(ctas) / double(rounds * kRound);
            if (full > best + 0.02) parts = p, best = full;
            if (best >= 0.9) break;
        }
        chunk = ((G + parts - 1) / parts + 3) / 4 * 4;
        parts = (G + chunk - 1) / chunk;
        bound_at = (int64_t(B) * G * int64_t(sizeof(float2)) + 255) / 256 * 256;
        hist_at = bound_at + (int64_t(B) * G * 4 + 255) / 256 * 256;
        bytes = hist_at + int64_t(B) * parts * 2 * kBins * 4;
    }
};

template <typename T>
cudaError_t launch_sample(const SampleArgs &a, int32_t B, cudaStream_t st) {
    const bool aligned = ((reinterpret_cast<uintptr_t>(a.logits) | uintptr_t(a.stride * int64_t(sizeof(T)))) & 15) == 0;
    const dim3 grid(unsigned(a.parts), unsigned(B));
    cudaError_t e = aligned ? launch_pdl_grid(k_sample_groups<T, true>, grid, kGroupThreads, 0, st, a)
                            : launch_pdl_grid(k_sample_groups<T, false>, grid, kGroupThreads, 0, st, a);
    if (e != cudaSuccess) return e;
    e = cudaFuncSetAttribute(k_sample_pick<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(sizeof(Shared)));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(B) * unsigned(a.ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Shared);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(a.ctas);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.ctas > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_sample_pick<T>, a);
}

}  // namespace

}  // namespace tmk

extern "C" int64_t trie_sample_workspace(int32_t B, int32_t V) {
    if (B < 0 || B > 65535 || V < 2 || V > tmk::kMaxV) return -1;
    return tmk::Plan(B, V).bytes;
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
    if (!*bad && (reinterpret_cast<uintptr_t>(d_workspace) & 15)) bad = "d_workspace is not aligned to 16 bytes";
    if (!*bad && B > 0 && !d_seeds) bad = "d_seeds is NULL";
    if (!*bad && (off_boundary(8, d_seeds) || off_boundary(4, d_temperature, d_top_k, d_top_p, d_min_p, d_tokens, d_logprobs)))
        bad = "an array is not aligned to its elements";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (B == 0) return TRIE_OK;
    SampleArgs a;
    a.logits = d_logits;
    a.stride = stride;
    a.V = V;
    const Plan plan(B, V);
    a.G = plan.G;
    a.chunk = plan.chunk;
    a.parts = plan.parts;
    // A cluster for each row while all of them run at once, two CTAs an SM, and for
    // twice that where a grammar leaves most rows little to do. CTAs a row 1, 2, 4:
    // 64 rows of V 262,144 99, 83, 74 us; 200 rows, three quarters constrained, 80, 69,
    // 68; 256 free rows of V 152,064 37, 49, 51; one row of V 32,000 12.4, 11.0, 11.0.
    const int round = 2 * sm_count();
    a.ctas = B * 4 <= round ? 4 : (B * 2 <= round || (d_mask && B <= round)) ? 2 : 1;
    a.seeds = d_seeds;
    a.temperature = d_temperature;
    a.top_k = d_top_k;
    a.top_p = d_top_p;
    a.min_p = d_min_p;
    a.g = make_grammar(d_mask, mask_rows, d_states, V);
    a.stats = static_cast<float2 *>(d_workspace);
    a.bound = reinterpret_cast<float *>(static_cast<unsigned char *>(d_workspace) + plan.bound_at);
    a.hist = reinterpret_cast<uint32_t *>(static_cast<unsigned char *>(d_workspace) + plan.hist_at);
    a.tokens = d_tokens;
    a.logprobs = d_logprobs;
    const cudaError_t e = dtype == TRIE_DTYPE_F32 ? launch_sample<float>(a, B, stream)
                                                  : launch_sample<__nv_bfloat16>(a, B, stream);
    if (e != cudaSuccess) return fail_launch(e, "sample launch");
    return TRIE_OK;
}
