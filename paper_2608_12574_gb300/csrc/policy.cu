// The clipped policy loss with a KL term of sampled tokens, and its gradient by
// their logits: trie_policy_loss.
//
// Of a row with logits x, token t, and the tokens that its state allows:
//   y = x / temperature,  lp = y[t] - log sum exp y
//   rho = exp(lp - old),  d = ref - lp
//   loss = weight (kl (exp(d) - d - 1) - min(rho A, clip(rho) A))
//   slope = dloss / dlp = weight (kl (1 - exp(d)) - [rho A <= clip(rho) A] rho A)
//   dloss / dx[v] = slope ([v = t] - exp(y[v] - log sum exp y)) / temperature
// A row is read once: its logits stay in shared memory between the pass that finds
// its largest and its sum, and the pass that writes its gradient.
//
//  k_policy_rows  rows of which three shares fit the shared memory of up to 16 CTAs.
//  k_policy       longer ones, and long ones without a gradient.
//
// What bounds it (times of calls that follow one another).
//   4,096 rows, V 152,064, bf16, with the gradient: 371 us, 6.7 TB/s: HBM. (A
//     CTA a row read twice: 2,210. Clusters with a row in registers, one row each:
//     1,389. The clusters staying, but with every warp making every row's slope: 885; a warp of its own
//     for it: 583; two logits an instruction and what a row needs of its scalars read ahead: 470; 15
//     working warps instead of 30, so that half as many instructions go into a row's own work: 393; less unrolled: 371.)
//     Without the gradient 225 us, 5.5 TB/s.
//   1,024 rows, V 128,011, half of them constrained: 86 us, 4.7 TB/s of zeros, gradients
//     and free rows' logits (all free 94, 5.6 TB/s: 28 rows a cluster, beside the first one's chain and
//     the last one's; all constrained 70): a constrained row waits for its mask's words and then for its tokens' logits,
//     behind what the workers store, and three rows of a cluster are on their way at a time. The next row's
//     words, asked for behind this row's logits, are 8 us of the 94 that it was.
//   288 rows, V 35,776, all constrained: 11 us. (Words gone through one after the other by the whole warp: 21.)
//   300 rows, V 262,144, f32: 109 us, 5.8 TB/s on the 112 SMs that clusters of 16 reach.
//   64 rows, V 32,000, f32, no gradient: 5 us, a chain of waits (row, masses, slope).
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include <cuda_runtime.h>

#include "blackwell.cuh"
#include "logits.cuh"
#include "two.cuh"

namespace tmk {

namespace {

constexpr int kSlots = 4;               // shares of rows in shared memory, at most
constexpr int kRowSmem = 228224;        // beside 4 KB that are declared
constexpr int kMaxCluster = 16;
constexpr int kRanks = 4;               // rows whose masses may be on their way
constexpr int kPolicyThreads = 256;     // of k_policy
constexpr int kMaxShare = kRowSmem / 3 / 128 * 128;  // bytes of a share of which three fit

struct PolicyArgs {
    const void *logits;
    int64_t stride;
    int32_t B, V;
    const int32_t *tokens;
    const float *old, *advantages, *ref, *weights, *temperature;
    float low, high, kl;  // the ratio is clipped to [low, high]
    Grammar g;
    float *losses, *logprobs;
    void *grad;
    int64_t grad_stride;
    int32_t ctas;         // of a row
    int32_t clusters;     // of k_policy_rows
    int32_t slots, slot_bytes;
};

__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The largest value seen and the sum of exp2((x - largest) c).
struct Mass {
    float top, sum;
    __device__ __forceinline__ void join(float other_top, float other_sum, float c) {
        const float t = fmaxf(top, other_top);
        if (t == -INFINITY) {  // nothing yet, or a NaN, which is in the sums
            sum += other_sum;
            return;
        }
        sum = sum * exp2_of((top - t) * c) + other_sum * exp2_of((other_top - t) * c);
        top = t;
    }
};

// Of a warp's masses, in all lanes.
__device__ __forceinline__ Mass warp_mass(const Mass &mine, float c) {
    Mass all;
    asm("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(all.top) : "f"(mine.top));
    const float off = all.top == -INFINITY ? 0.0f : all.top;
    all.sum = mine.sum * exp2_of((mine.top - off) * c);
#pragma unroll
    for (int d = 16; d; d >>= 1) all.sum += __shfl_xor_sync(~0u, all.sum, d);
    return all;
}

// exp2((x - top) c), with -top twice and c twice.
__device__ __forceinline__ Two exp2_of(Two x, Two minus_top, Two c) {
    const float2 y = apart(mul2(add2(x, minus_top), c));
    return two(exp2_of(y.x), exp2_of(y.y));
}

// 16 bytes of a row.
template <typename T>
struct Piece {
    static constexpr int kSize = 16 / int(sizeof(T));
    uint32_t w[4];
    __device__ __forceinline__ void set(const uint4 &v) { w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w; }
    __device__ __forceinline__ uint4 raw() const { return make_uint4(w[0], w[1], w[2], w[3]); }
    __device__ __forceinline__ void clear() {
        const uint32_t none = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;  // -inf
        set(make_uint4(none, none, none, none));
    }
    // -inf where the element's bit is 0
    __device__ __forceinline__ void keep(uint32_t bits) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if (sizeof(T) == 2) {
                if (!(bits >> (2 * i) & 1)) w[i] = (w[i] & 0xFFFF0000u) | 0xFF80u;
                if (!(bits >> (2 * i) & 2)) w[i] = (w[i] & 0xFFFFu) | 0xFF800000u;
            } else if (!(bits >> i & 1)) {
                w[i] = 0xFF800000u;
            }
        }
    }
    // elements 2 i and 2 i + 1
    __device__ __forceinline__ Two pair(int i) const {
        if (sizeof(T) == 2) return two(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
        return two(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    }
    __device__ __forceinline__ void set_pair(int i, Two x) {
        const float2 v = apart(x);
        if (sizeof(T) == 2) {
            const __nv_bfloat162 both = __floats2bfloat162_rn(v.x, v.y);
            w[i] = *reinterpret_cast<const uint32_t *>(&both);
        } else {
            w[2 * i] = __float_as_uint(v.x), w[2 * i + 1] = __float_as_uint(v.y);
        }
    }
    __device__ __forceinline__ T element(int i) const {
        if (sizeof(T) == 2) return from_f32<T>(__uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16));
        return from_f32<T>(__uint_as_float(w[i]));
    }
};
// The bits of the tokens from v on.
__device__ __forceinline__ uint32_t bits_from(const GrammarRow &row, int32_t v, int32_t words) {
    const int32_t w = v >> 5;
    const uint32_t next = w + 1 < words ? row.word(w + 1) : 0u;
    return __funnelshift_r(row.word(w), next, v & 31);
}
// Adds up kCount pieces. A NaN does not show in the largest value but in the sum.
template <typename T, int kCount>
__device__ __forceinline__ void add_pieces(Mass &all, const Piece<T> (&p)[kCount], float c) {
    float top = all.top;
    if (sizeof(T) == 2) {
        __nv_bfloat162 most = *reinterpret_cast<const __nv_bfloat162 *>(&p[0].w[0]);
#pragma unroll
        for (int i = 0; i < kCount; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) most = __hmax2(most, *reinterpret_cast<const __nv_bfloat162 *>(&p[i].w[j]));
        top = fmaxf(top, fmaxf(__low2float(most), __high2float(most)));
    } else {
#pragma unroll
        for (int i = 0; i < kCount; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) top = fmaxf(top, __uint_as_float(p[i].w[j]));
    }
    const float off = top == -INFINITY ? 0.0f : top;
    all.sum *= exp2_of((all.top - off) * c);
    all.top = top;
    const Two minus_top = two(-off, -off), cc = two(c, c);
    Two sum[2] = {two(0.0f, 0.0f), two(0.0f, 0.0f)};
#pragma unroll
    for (int i = 0; i < kCount; i++)
#pragma unroll
        for (int j = 0; j < Piece<T>::kSize / 2; j++) sum[j & 1] = add2(sum[j & 1], exp2_of(p[i].pair(j), minus_top, cc));
    const float2 s = apart(add2(sum[0], sum[1]));
    all.sum += s.x + s.y;
}
__device__ __forceinline__ float temperature_of(const PolicyArgs &a, int32_t b) {
    const float given = a.temperature ? __ldg(a.temperature + b) : 1.0f;
    return given > 0.0f ? fminf(fmaxf(given, 1.17549435e-38f), 3.40282347e38f) : 1.0f;
}

struct RowValues {
    int32_t token, state;
    float old, advantage, ref, weight, temperature;
    __device__ RowValues(const PolicyArgs &a, int32_t b)
        : token(__ldg(a.tokens + b)), state(a.g.mask ? __ldg(a.g.states + b) : TRIE_STATE_FREE), old(__ldg(a.old + b)),
          advantage(__ldg(a.advantages + b)), ref(a.ref ? __ldg(a.ref + b) : 0.0f),
          weight(a.weights ? __ldg(a.weights + b) : 1.0f), temperature(temperature_of(a, b)) {}
};

// What the gradient of a row needs of it, and its loss (written by one thread).
struct Slope {
    float top, c;      // exp2((x - top) c) ..
    float f;           // .. times this: the gradient of a token
    float at_token;    // of the row's own
    int32_t token;     // -1: the gradient is 0 everywhere
};
__device__ __forceinline__ Slope finish(const PolicyArgs &a, int32_t b, const Mass &all, float xt, const RowValues &v, bool writes) {
    float lp = (xt - all.top) / v.temperature - logf(all.sum);
    if (all.top == INFINITY) lp = __int_as_float(0x7FC00000);
    if (xt == -INFINITY) lp = -INFINITY;
    float loss = 0.0f, slope = 0.0f;
    if (lp != -INFINITY && v.weight != 0.0f) {
        const float rho = expf(lp - v.old);
        // no advantage, no surrogate, if the ratio is infinite too
        const float free = v.advantage == 0.0f && rho == INFINITY ? 0.0f : rho * v.advantage, held = fminf(fmaxf(rho, a.low), a.high) * v.advantage;
        loss = -(free > held ? held : free);  // a NaN stays one
        slope = free > held ? 0.0f : -free;
        if (a.ref) {
            const float d = v.ref - lp, e = expm1f(d);
            loss += a.kl * (e - d);
            slope -= a.kl * e;
        }
        loss *= v.weight;
        slope *= v.weight;
    }
    if (writes) {
        a.losses[b] = loss;
        a.logprobs[b] = lp;
    }
    const float per = 1.0f / v.temperature, others = -expm1f(lp);
    return {all.top, 1.44269504f / v.temperature, -slope / all.sum * per, others == 0.0f && slope == slope ? 0.0f : slope * others * per,
            slope == 0.0f ? -1 : v.token};
}
// Of a token that is not allowed 0, whatever f is, and of one whose probability is 0 in 32 bits, unless f is a NaN.
__device__ __forceinline__ float slope_of(const Slope &s, float x) {
    const float e = exp2_of((x - s.top) * s.c);
    return x == -INFINITY || (e == 0.0f && s.f == s.f) ? 0.0f : s.f * e;
}

// Of a piece. f exp2() is 0 where x is -inf, unless f is not a number of its own.
template <typename T>
__device__ __forceinline__ Piece<T> slope_of(const Slope &s, const Piece<T> &p) {
    Piece<T> g;
    if (fabsf(s.f) <= 3.40282347e38f) {
        const Two minus_top = two(-s.top, -s.top), c = two(s.c, s.c), f = two(s.f, s.f);
#pragma unroll
        for (int j = 0; j < Piece<T>::kSize / 2; j++) g.set_pair(j, mul2(f, exp2_of(p.pair(j), minus_top, c)));
    } else {
#pragma unroll
        for (int j = 0; j < Piece<T>::kSize / 2; j++) {
            const float2 x = apart(p.pair(j));
            g.set_pair(j, two(slope_of(s, x.x), slope_of(s, x.y)));
        }
    }
    return g;
}

// Where the 16-byte pieces of row b lie, and the share of a CTA: pieces [first,
// last), tokens [lo, hi): what is before the first piece belongs to the first
// CTA of the row, what is behind the last to the last.
template <typename T>
struct Share {
    const T *x;
    T *grad;
    int32_t head, first, last, lo, hi;
    bool same;  // the gradient's pieces lie as the logits'
    Share() = default;
    __device__ Share(const PolicyArgs &a, int32_t b, int32_t rank) {
        constexpr int kSize = Piece<T>::kSize;
        x = static_cast<const T *>(a.logits) + b * a.stride;
        grad = a.grad ? static_cast<T *>(a.grad) + b * a.grad_stride : nullptr;
        head = min(int32_t((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / int32_t(sizeof(T)), a.V);
        const int32_t pieces = (a.V - head) / kSize, share = (pieces + a.ctas - 1) / a.ctas;
        first = min(pieces, rank * share);
        last = min(pieces, first + share);
        lo = rank == 0 ? 0 : head + first * kSize;
        hi = rank == a.ctas - 1 ? a.V : head + last * kSize;
        same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(grad)) & 15) == 0;
    }
    __device__ __forceinline__ const uint4 *pieces() const { return reinterpret_cast<const uint4 *>(x + head); }
    // the token of thread i among those outside pieces, -1 for none
    __device__ __forceinline__ int32_t edge(int32_t i) const {
        const int32_t from = head + first * Piece<T>::kSize, to = head + last * Piece<T>::kSize, before = from - lo;
        const int32_t v = i < before ? lo + i : to + i - before;
        return v < hi ? v : -1;
    }
    __device__ __forceinline__ void store(int32_t i, const Piece<T> &g) const {
        constexpr int kSize = Piece<T>::kSize;
        if (same) {
            reinterpret_cast<uint4 *>(grad + head)[i] = g.raw();
        } else {
#pragma unroll
            for (int e = 0; e < kSize; e++) grad[head + i * kSize + e] = g.element(e);
        }
    }
};

// Rows of which three shares fit a CTA's shared memory: clusters of CTAs stay and
// go over the rows, a cluster a row, a share of it a CTA. Warps with a part of their own:
//   bringers    one for each slot: a free row's share comes to the slot by a bulk copy; of a
//               constrained row the allowed tokens are listed from its mask, with
//               their logits, or, if they are many, the share comes as well
//   workers     the mass of a row's share, then the gradient of the row before, whose
//               slope has had that long to arrive
//   the sender  a CTA's mass of a row to all CTAs of the cluster
//   the finisher  the row's loss and slope from these
// The gradient of a constrained row is zeros with the listed tokens' put in.
// A warp whose wait gives up (no wait of a correct program does) goes no further, so that nothing is
// taken for there that is not, and stays until all other warps of the cluster have ended or given up too:
// these may still write to its CTA's shared memory. What it has not finished becomes NaN: the workers' gradients and the
// finisher's losses, from that row on.
constexpr int kWorkerWarps = 15;
constexpr int kWorkers = 32 * kWorkerWarps;
constexpr int kSender = kWorkerWarps, kFinisher = kSender + 1, kFirstBringer = kFinisher + 1;
constexpr int kRowThreads = 32 * (kFirstBringer + kSlots);
constexpr int kListed = 128;  // allowed tokens of a share that are listed, at most
constexpr int kWordsAhead = 38;  // words of the mask that a lane reads: 38,912 tokens, more than a share of bf16 logits
constexpr int kWordsTogether = 8;  // of these, how many are gone through if one of them is not 0
static_assert(kMaxShare / 2 + 16 + 2 * 32 <= kWordsAhead * 32 * 32, "a share's words");
constexpr int kTogether = 5;  // pieces that a worker adds up at a time

// What the workers need to know of a row.
template <typename T>
struct RowIn {
    Share<T> share;
    GrammarRow row;
    int32_t listed;   // >= 0: so many allowed tokens are listed in the slot; -1: the share is there
    Mass mass;        // of the listed tokens
    float c;          // log2(e) / temperature
    float edge[16];   // logits outside the pieces
};
struct List {
    int32_t token[kListed];
    float x[kListed];
};

__device__ __forceinline__ void first_logits_sync() { asm volatile("barrier.cta.sync 2, 64;" ::: "memory"); }

// Calls, so that they take no room among the instructions of the rows' loop, and without an address of the kernel's own
// variables, which it would keep on a stack then (1,024 rows of 128,011, all of them constrained, 69.6 us, and 70.8 inlined;
// 4,096 rows of 152,064 370 us, and 380 with a stack): a warp's waits that are hardly ever ones; and a CTA's share of a row's
// gradient as NaN, by a warp: all of it, as the tokens of the warp's part of a list lie in other warps' pieces.
__device__ __noinline__ void copies_end(uint32_t bar, uint32_t parity) {
    int none = 0;
    bar_wait(bar, parity, &none);
    __syncwarp();
}
__device__ __noinline__ bool ended_apart(uint32_t bar, uint32_t parity, int *gave_up) {
    return __all_sync(~0u, bar_wait(bar, parity, gave_up));
}
template <typename T>
__device__ __noinline__ void no_gradient(const PolicyArgs &a, int32_t b, int32_t rank) {
    const Share<T> s(a, b, rank);
    const T nan = from_f32<T>(__int_as_float(0x7FC00000));
    for (int32_t v = s.lo + int32_t(threadIdx.x & 31); v < s.hi; v += 32) s.grad[v] = nan;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 1) k_policy_rows(const PolicyArgs a) {
    constexpr int kSize = Piece<T>::kSize;
    extern __shared__ __align__(128) unsigned char slots[];
    __shared__ uint64_t bars[2 * kSlots + kRanks + 5];
    __shared__ Mass parts[2][32];
    __shared__ Mass ranks[kRanks][kMaxCluster];
    __shared__ __align__(16) unsigned char in_bytes[kSlots * sizeof(RowIn<T>)];
    RowIn<T> *const in = reinterpret_cast<RowIn<T> *>(in_bytes);
    __shared__ int32_t found[kSlots][kListed];  // a bringer's own
    __shared__ Slope slopes[2];
    __shared__ int gave_up;
    const uint32_t full = smem_addr(bars), freed = full + 8 * kSlots;  // of a slot
    const uint32_t masses = freed + 8 * kSlots;                         // of a row, of all its CTAs
    const uint32_t summed = masses + 8 * kRanks, sloped = summed + 8 * 2, filled = sloped + 8 * 2;
    const int lane = threadIdx.x & 31, warp = __shfl_sync(~0u, int(threadIdx.x >> 5), 0);
    const int32_t cluster = int32_t(blockIdx.x) / a.ctas, rank = int32_t(blockIdx.x) % a.ctas, V = a.V;
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int i = 0; i < kSlots; i++) {
            bar_init(full + 8 * i, 1);
            bar_init(freed + 8 * i, kWorkerWarps);
        }
        for (int i = 0; i < kRanks; i++) bar_init(masses + 8 * i, a.ctas);
        for (int i = 0; i < 2; i++) {
            bar_init(summed + 8 * i, kWorkerWarps);
            bar_init(sloped + 8 * i, 1);
        }
        bar_init(filled, kWorkerWarps);
        bar_init_fence();
    }
    pdl_launch_dependents();
    if (a.ctas > 1) cluster_sync();  // every CTA's barriers are there
    else __syncthreads();
    pdl_wait();

    const int32_t rows = (a.B - cluster + a.clusters - 1) / a.clusters;
    // A wait by a warp; and what it does once that is false. (The hardware's barrier takes warps that have ended for arrived.)
    auto ended = [&](uint32_t bar, uint32_t parity) { return __all_sync(~0u, bar_wait(bar, parity, &gave_up)) != 0; };
    auto leave = [&] {
        if (a.ctas > 1) cluster_sync();
    };
    if (warp >= kFirstBringer) {
        // Brings every a.slots-th row into its slot: what there is to know of it, and its share or the list of its
        // allowed tokens. What does not need the slot comes before the wait for it, and the next row's mask is on its
        // way while this row's logits are waited for.
        const int slot = warp - kFirstBringer;
        if (slot >= a.slots) return;
        RowIn<T> &i = in[slot];
        bool ok = true;
        uint32_t phase = 1, word[kWordsAhead];
        auto state_of = [&](int32_t r) { return a.g.mask && r < rows ? __ldg(a.g.states + cluster + r * a.clusters) : TRIE_STATE_FREE; };
        auto c_of = [&](int32_t r) { return 1.44269504f / temperature_of(a, cluster + min(r, rows - 1) * a.clusters); };
        auto share_of = [&](int32_t r) { return Share<T>(a, cluster + min(r, rows - 1) * a.clusters, rank); };
        auto read_words = [&](const Share<T> &s, const GrammarRow &row) {
            if (row.kind != kAllowRow) return;
            const int32_t w = (s.lo >> 5) + lane, n = ((s.hi + 31) >> 5) - w;
#pragma unroll
            for (int k = 0; k < kWordsAhead; k++) word[k] = 32 * k < n ? __ldg(row.words + w + 32 * k) : 0u;
        };
        int32_t state = state_of(slot), state_next = state_of(slot + a.slots);
        float c_next = c_of(slot);
        read_words(share_of(slot), grammar_state(a.g, state));
        for (int32_t r = slot; r < rows; r += a.slots, phase ^= 1) {
            const Share<T> s = share_of(r);
            const GrammarRow row = grammar_state(a.g, state);
            const float c = c_next;
            c_next = c_of(r + a.slots);
            int32_t listed = row.kind == kAllowAll ? -1 : 0;
            if (row.kind == kAllowRow) {
                // every lane's words' tokens, one lane after the other
                const int32_t v = ((s.lo >> 5) + lane) * 32, left = s.hi - v;  // left: tokens from its first word on
                if (v < s.lo) word[0] &= ~0u << (s.lo - v);
                int32_t mine = 0;
#pragma unroll
                for (int k = 0; k < kWordsAhead; k++) {
                    const int32_t n = left - 1024 * k;
                    if (n > 0 && n < 32) word[k] &= (1u << n) - 1u;
                    mine += __popc(word[k]);
                }
                int32_t upto = mine;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const int32_t before = __shfl_up_sync(~0u, upto, d);
                    if (lane >= d) upto += before;
                }
                listed = __shfl_sync(~0u, upto, 31);
                if (listed > kListed) {
                    listed = -1;
                } else if (mine) {
                    int32_t *to = found[slot] + upto - mine;
#pragma unroll
                    for (int k0 = 0; k0 < kWordsAhead; k0 += kWordsTogether) {
                        uint32_t any = 0;
#pragma unroll
                        for (int k = k0; k < min(k0 + kWordsTogether, kWordsAhead); k++) any |= word[k];
                        if (!any) continue;
#pragma unroll
                        for (int k = k0; k < min(k0 + kWordsTogether, kWordsAhead); k++)
                            for (uint32_t bits = word[k]; bits; bits &= bits - 1) *to++ = v + 1024 * k + __ffs(bits) - 1;
                    }
                }
            } else if (row.kind == kAllowEos && s.lo < s.hi && s.hi == V) {
                listed = 1;
                if (lane == 0) found[slot][0] = V - 1;
            }
            __syncwarp();
            float at_edge = -INFINITY;
            if (listed < 0) {
                const int32_t edge = lane < 16 ? s.edge(lane) : -1;
                if (edge >= 0 && row.allows(edge)) at_edge = to_f32(s.x[edge]);
            }
            int32_t token[kListed / 32];
            float x[kListed / 32];
            Mass mass = {-INFINITY, 0.0f};
#pragma unroll
            for (int k = 0; k < kListed / 32; k++) {
                token[k] = lane + 32 * k < listed ? found[slot][lane + 32 * k] : 0;
                x[k] = lane + 32 * k < listed ? to_f32(s.x[token[k]]) : -INFINITY;
            }
            state = state_next;
            state_next = state_of(r + 2 * a.slots);
            read_words(share_of(r + a.slots), grammar_state(a.g, state));
#pragma unroll
            for (int k = 0; k < kListed / 32; k++) mass.top = fmaxf(mass.top, x[k]);
            const float off = mass.top == -INFINITY ? 0.0f : mass.top;
#pragma unroll
            for (int k = 0; k < kListed / 32; k++) mass.sum += exp2_of((x[k] - off) * c);
            mass = warp_mass(mass, c);
            if (!(ok = ended(freed + 8 * slot, phase))) break;
            if (lane == 0 && listed < 0) {  // first: 4,096 rows 383 us, and 390 with the row's values before it
                const uint32_t bytes = uint32_t(s.last - s.first) * 16u;
                bar_expect_bytes(full + 8 * slot, bytes);
                if (bytes) bulk_load(smem_addr(slots + slot * a.slot_bytes), s.pieces() + s.first, bytes, full + 8 * slot);
            }
            if (lane < 16) i.edge[lane] = at_edge;
            if (listed >= 0) {
                List &list = *reinterpret_cast<List *>(slots + slot * a.slot_bytes);
#pragma unroll
                for (int k = 0; k < kListed / 32; k++) {
                    list.token[lane + 32 * k] = token[k];
                    list.x[lane + 32 * k] = x[k];
                }
                async_fence();  // a copy may write there next
            }
            if (lane == 0) {
                i.share = s;
                i.row = row;
                i.listed = listed;
                i.mass = mass;
                i.c = c;
            }
            __syncwarp();
            if (lane == 0) bar_arrive(full + 8 * slot);
        }
        if (slot < rows) copies_end(full + 8 * slot, phase);  // before the CTA does
        if (!ok) leave();
        return;
    }
    if (warp == kSender) {
        // The CTA's mass of a row, to all CTAs of the cluster; the first once the finisher has its tokens' logits.
        first_logits_sync();
        for (int32_t r = 0; r < rows; r++) {
            const float c = 1.44269504f / temperature_of(a, cluster + r * a.clusters);
            if (!ended(summed + 8 * (r & 1), (r >> 1) & 1)) {
                leave();
                return;
            }
            Mass all = {-INFINITY, 0.0f};
            if (lane < kWorkerWarps) all = parts[r & 1][lane];
            all = warp_mass(all, c);
            if (lane < a.ctas) {
                *cluster_object(&ranks[r % kRanks][rank], lane) = all;
                bar_arrive_cluster(cluster_addr(masses + 8 * (r % kRanks), lane));
            }
        }
        return;
    }
    if (warp == kFinisher) {
        // A row's slope from all its CTAs' masses. What it needs of a row is read ahead so that it waits for none:
        // the row's values four rows, the mask's word with its token three, the token's logit two, and the
        // latter is there before the slope of two rows earlier is, and so before any CTA writes the row's gradient.
        auto values = [&](int32_t r) { return RowValues(a, cluster + min(r, rows - 1) * a.clusters); };
        auto mask_word = [&](const RowValues &v) {
            const GrammarRow row = grammar_state(a.g, v.state);
            if (v.token < 0 || v.token >= V) return 0u;
            return row.kind == kAllowRow ? __ldg(row.words + (v.token >> 5)) : row.word(v.token >> 5);
        };
        auto token_logit = [&](int32_t r, const RowValues &v, uint32_t word) {
            return (word >> (v.token & 31)) & 1u ? to_f32(Share<T>(a, cluster + min(r, rows - 1) * a.clusters, rank).x[v.token]) : -INFINITY;
        };
        RowValues v0 = values(0), v1 = values(1), v2 = values(2), v3 = values(3);
        float x0 = token_logit(0, v0, mask_word(v0)), x1 = token_logit(1, v1, mask_word(v1));
        uint32_t word2 = mask_word(v2);
        x0 = __shfl_sync(~0u, x0, 0), x1 = __shfl_sync(~0u, x1, 0);
        first_logits_sync();
        for (int32_t r = 0; r < rows; r++) {
            float x2 = token_logit(r + 2, v2, word2);
            const uint32_t word3 = mask_word(v3);
            const RowValues v4 = values(r + 4);
            const float c = 1.44269504f / v0.temperature;
            if (!__all_sync(~0u, bar_wait_cluster(masses + 8 * (r % kRanks), (r / kRanks) & 1, &gave_up))) {
                for (int32_t q = r + lane; rank == 0 && q < rows; q += 32)
                    a.losses[cluster + q * a.clusters] = a.logprobs[cluster + q * a.clusters] = __int_as_float(0x7FC00000);
                __syncwarp();
                leave();
                return;
            }
            Mass all = {-INFINITY, 0.0f};
            if (lane < a.ctas) all = ranks[r % kRanks][lane];
            all = warp_mass(all, c);
            const Slope slope = finish(a, cluster + r * a.clusters, all, x0, v0, rank == 0 && lane == 0);
            x2 = __shfl_sync(~0u, x2, 0);  // it is there
            if (lane == 0) {
                slopes[r & 1] = slope;
                bar_arrive(sloped + 8 * (r & 1));
            }
            v0 = v1, v1 = v2, v2 = v3, v3 = v4, x0 = x1, x1 = x2, word2 = word3;
        }
        return;
    }

    const int32_t worker = threadIdx.x, words = int32_t(a.g.W);
    const bool in_place = a.grad == a.logits;
    uint32_t filled_phase = 0;
    auto fill = [&](const Share<T> &s) {  // with zeros
        const int32_t edge = worker < 16 ? s.edge(worker) : -1;
        if (edge >= 0) s.grad[edge] = from_f32<T>(0.0f);
        Piece<T> g;
        g.set(make_uint4(0u, 0u, 0u, 0u));
        for (int32_t j = s.first + worker; j < s.last; j += kWorkers) s.store(j, g);
    };
    // Both are false where a wait gave up.
    auto first_pass = [&](int32_t r, int slot, uint32_t phase) {
        if (!ended(full + 8 * slot, phase)) return false;
        const RowIn<T> &i = in[slot];
        const float c = i.c;
        Mass all = {-INFINITY, 0.0f};
        if (i.listed < 0) {
            if (worker < 16) {
                const float x = i.edge[worker];
                all.top = fmaxf(all.top, x);
                all.sum = exp2_of((x - (all.top == -INFINITY ? 0.0f : all.top)) * c);
            }
            uint4 *held = reinterpret_cast<uint4 *>(slots + slot * a.slot_bytes) + worker;
            const bool masked = i.row.kind != kAllowAll;
            int32_t v = i.share.head + (i.share.first + worker) * kSize;
            for (int32_t left = i.share.last - i.share.first - worker; left > 0; left -= kTogether * kWorkers) {
                Piece<T> p[kTogether];
#pragma unroll
                for (int k = 0; k < kTogether; k++) {
                    p[k].clear();
                    if (left > k * kWorkers) p[k].set(held[k * kWorkers]);
                }
                if (masked) {  // for the second pass too
#pragma unroll
                    for (int k = 0; k < kTogether; k++)
                        if (left > k * kWorkers) {
                            p[k].keep(bits_from(i.row, v + k * kWorkers * kSize, words));
                            held[k * kWorkers] = p[k].raw();
                        }
                    async_fence();  // a copy writes there next
                }
                add_pieces(all, p, c);
                held += kTogether * kWorkers;
                v += kTogether * kWorkers * kSize;
            }
        } else {
            if (worker == 0) all = i.mass;
            if (a.grad && !in_place) fill(i.share);
        }
        all = warp_mass(all, c);
        __syncwarp();  // the zeros are written, too
        if (lane == 0) {
            parts[r & 1][warp] = all;
            bar_arrive(summed + 8 * (r & 1));
        }
        return true;
    };
    auto second_pass = [&](int32_t r, int slot) {
        if (!ended(sloped + 8 * (r & 1), (r >> 1) & 1)) return false;
        if (!a.grad) return true;
        const Slope slope = slopes[r & 1];
        const Share<T> s = in[slot].share;
        const int32_t n = s.last - s.first;
        const unsigned char *const held = slots + slot * a.slot_bytes;
        const int32_t edge = worker < 16 ? s.edge(worker) : -1;
        if (in[slot].listed < 0 && slope.token >= 0) {
            if (edge >= 0) s.grad[edge] = from_f32<T>(edge == slope.token ? slope.at_token : slope_of(slope, in[slot].edge[worker]));
            const uint4 *from = reinterpret_cast<const uint4 *>(held);
            const int32_t at = slope.token < s.head ? -1 : (slope.token - s.head) / kSize - s.first;  // the token's piece
#pragma unroll 4  // 4,096 rows, V 152,064, bf16 371 us; 5: 392, 10: 485
            for (int32_t j = worker; j < n; j += kWorkers) {
                Piece<T> p;
                p.set(from[j]);
                s.store(s.first + j, slope_of(slope, p));
                if (j == at) s.grad[slope.token] = from_f32<T>(slope.at_token);
            }
            return true;
        }
        if (in_place || in[slot].listed < 0) fill(s);
        const int32_t listed = slope.token >= 0 ? in[slot].listed : 0;
        if (in_place && listed > 0) {
            __syncwarp();
            if (lane == 0) bar_arrive(filled);
            if (!ended_apart(filled, filled_phase, &gave_up)) return false;
            filled_phase ^= 1;
        }
        if (worker < listed) {
            const List &list = *reinterpret_cast<const List *>(held);
            const int32_t v = list.token[worker];
            s.grad[v] = from_f32<T>(v == slope.token ? slope.at_token : slope_of(slope, list.x[worker]));
        }
        return true;
    };
    int slot = 0, slot_next = 0;
    uint32_t phase = 0;  // of slot_next
    auto step = [&] {
        if (++slot_next == a.slots) slot_next = 0, phase ^= 1;
    };
    int32_t r = -1;
#pragma unroll 1
    for (; r < rows; r++) {
        if (r + 1 < rows && !first_pass(r + 1, slot_next, phase)) break;
        if (r >= 0) {
            if (!second_pass(r, slot)) break;
            __syncwarp();
            if (lane == 0) bar_arrive(freed + 8 * slot);
        }
        slot = slot_next;
        step();
    }
    if (r == rows) return;
    __syncwarp();
    leave();
    if (!a.grad) return;
    for (r = max(r, 0); r < rows; r++) no_gradient<T>(a, cluster + r * a.clusters, rank);
}

// Longer rows: a cluster of CTAs a row, a share of its 16-byte pieces each, which
// the second pass reads again (from L2, as far as it holds the rows at work).
template <typename T>
__global__ void __launch_bounds__(kPolicyThreads) k_policy(const PolicyArgs a) {
    constexpr int kSize = Piece<T>::kSize;
    __shared__ Mass parts[kPolicyThreads / 32];
    __shared__ Mass ranks[kMaxCluster];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t b = int32_t(blockIdx.x) / a.ctas, rank = int32_t(blockIdx.x) % a.ctas, V = a.V;
    if (a.ctas > 1) cluster_arrive();
    const Share<T> s(a, b, rank);
    const GrammarRow row = grammar_row(a.g, b);
    const bool masked = row.kind != kAllowAll;
    const int32_t words = int32_t(a.g.W);
    const float c = 1.44269504f / temperature_of(a, b);
    const int32_t edge = s.edge(threadIdx.x);

    // piece i, -inf where it is not there or a token is not allowed
    auto load = [&](int32_t i, Piece<T> &p) {
        const uint32_t bits = i >= s.last ? 0u : masked ? bits_from(row, s.head + i * kSize, words) : ~0u;
        p.clear();
        if (bits & ((1u << kSize) - 1u)) p.set(s.pieces()[i]);
        if (masked) p.keep(bits);
    };
    auto load_edge = [&]() { return edge >= 0 && row.allows(edge) ? to_f32(s.x[edge]) : -INFINITY; };

    Mass all = {load_edge(), 0.0f};
    if (!(all.top == all.top)) all.top = -INFINITY;  // a NaN shows in the sum
    all.sum = exp2_of((load_edge() - (all.top == -INFINITY ? 0.0f : all.top)) * c);
    constexpr int kBatch = 4;
    for (int32_t i0 = s.first + int32_t(threadIdx.x); i0 < s.last; i0 += kBatch * kPolicyThreads) {
        Piece<T> p[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; i++) load(i0 + i * kPolicyThreads, p[i]);
        add_pieces(all, p, c);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) all.join(__shfl_xor_sync(~0u, all.top, d), __shfl_xor_sync(~0u, all.sum, d), c);
    if (lane == 0) parts[warp] = all;
    const RowValues values(a, b);
    const int32_t t = values.token;
    const float xt = t >= 0 && t < V && row.allows(t) ? to_f32(s.x[t]) : -INFINITY;
    __syncthreads();
    all = parts[0];
#pragma unroll
    for (int i = 1; i < kPolicyThreads / 32; i++) all.join(parts[i].top, parts[i].sum, c);
    if (a.ctas > 1) {
        cluster_wait();  // all CTAs of the row are there
        if (int32_t(threadIdx.x) < a.ctas) *cluster_object(&ranks[rank], threadIdx.x) = all;
        cluster_sync();
        all = ranks[0];
        for (int i = 1; i < a.ctas; i++) all.join(ranks[i].top, ranks[i].sum, c);
    }
    const Slope slope = finish(a, b, all, xt, values, rank == 0 && threadIdx.x == 0);
    if (!a.grad) return;
    const bool zero = slope.token < 0;
    if (edge >= 0) s.grad[edge] = from_f32<T>(zero ? 0.0f : slope_of(slope, load_edge()));
    for (int32_t i = s.first + int32_t(threadIdx.x); i < s.last; i += kPolicyThreads) {
        Piece<T> p;
        if (zero) {
            p.set(make_uint4(0u, 0u, 0u, 0u));
        } else {
            load(i, p);
            p = slope_of(slope, p);
        }
        s.store(i, p);
    }
    if (zero || t < s.lo || t >= s.hi) return;
    __syncthreads();
    if (threadIdx.x == 0) s.grad[t] = from_f32<T>(slope.at_token);
}

// Launches `kernel` with clusters of a.ctas CTAs.
template <typename K>
cudaError_t launch_policy(K kernel, const PolicyArgs &a, int64_t ctas, int threads, int smem, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ctas));
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = size_t(smem);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(a.ctas);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.ctas > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

// Clusters of k_policy_rows<T> of so many CTAs that the current device runs at once.
template <typename T>
int active_clusters(int ctas) {
    static std::atomic<int> known[16][kMaxCluster + 1];
    int dev = 0, n = 0;
    const bool listed = cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < 16;  // else asked every time
    if (listed && (n = known[dev][ctas].load(std::memory_order_relaxed))) return n;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ctas));
    cfg.blockDim = dim3(kRowThreads);
    cfg.dynamicSmemBytes = size_t(kRowSmem);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(ctas);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(k_policy_rows<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaFuncSetAttribute(k_policy_rows<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, k_policy_rows<T>, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 0;
    }
    if (listed) known[dev][ctas].store(n, std::memory_order_relaxed);
    return n;
}

template <typename T>
cudaError_t run_policy(PolicyArgs a, cudaStream_t st) {
    const int64_t pieces = int64_t(a.V) * int64_t(sizeof(T)) / 16;
    auto share = [&] { return (pieces + a.ctas - 1) / a.ctas * 16; };
    // The fewest CTAs a row of which three shares fit, in even numbers: clusters of 5 reach more SMs than of 6 (140, and
    // 138 of 152), but not all of them fit at once while the call before still holds SMs (1,085 rows of 152,296 in
    // bf16 119 to 159 us, and 134; 168 by clusters of 8), and of 9 instead of 8 are no gain (500 rows of 150,000
    // in 32 bits 109 us, and 99). Beyond 10 the largest, 7 of which reach 112 SMs (8 of 12 96): 300 rows of
    // 220,000 in 32 bits 102 us, and 106.
    while (a.ctas < kMaxCluster && share() > kMaxShare) a.ctas = a.ctas == 10 ? kMaxCluster : (a.ctas + 2) / 2 * 2;
    a.clusters = 0;
    // Without a gradient a row that takes more than 8 is read by k_policy, in one pass (300 rows of 200,000 in 32
    // bits 65 us, and 75 by clusters of 16; with the gradient 138 and 98).
    if (share() <= kMaxShare && (a.grad || a.ctas <= kMaxCluster / 2)) {
        // More where the rows are few (8 rows of 32,000 in 32 bits with the gradient 5.1 us, and 6.3 with the fewest;
        // 1 row 4.2 and 4.6).
        while (a.ctas <= kMaxCluster / 4 && int64_t(a.B) * a.ctas * 2 <= sm_count() && share() > 16 * kRowThreads) a.ctas *= 2;
        a.clusters = std::min(a.B, active_clusters<T>(a.ctas));
    }
    if (a.clusters) {
        const int rows = (a.B + a.clusters - 1) / a.clusters;
        a.slot_bytes = std::max(int(sizeof(List)), int((share() + 127) / 128 * 128));
        a.slots = std::min(std::min(kSlots, rows), kRowSmem / a.slot_bytes);
        return launch_policy(k_policy_rows<T>, a, int64_t(a.clusters) * a.ctas, kRowThreads, a.slots * a.slot_bytes, st);
    }
    a.ctas = 8;
    if (int64_t(a.B) * a.ctas > 0x7FFFFFFF) return cudaErrorInvalidValue;
    return launch_policy(k_policy<T>, a, int64_t(a.B) * a.ctas, kPolicyThreads, 0, st);
}

}  // namespace

}  // namespace tmk

extern "C" int trie_policy_loss(const void *d_logits, int dtype, int64_t stride, int32_t B, int32_t V, const int32_t *d_tokens,
                                const float *d_old_logprobs, const float *d_advantages, const float *d_ref_logprobs,
                                const float *d_weights, const float *d_temperature, float clip_low, float clip_high, float kl,
                                const uint32_t *d_mask, int32_t mask_rows, const int32_t *d_states, float *d_losses,
                                float *d_logprobs, void *d_grad, int64_t grad_stride, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_logits(d_logits, dtype, stride, B, V);
    if (!*bad) bad = check_grammar(d_mask, mask_rows, d_states);
    if (!*bad && B > 0 && (!d_tokens || !d_old_logprobs || !d_advantages || !d_losses || !d_logprobs)) bad = "NULL pointer";
    if (!*bad && B > (1 << 30)) bad = "B must be <= 2^30";
    if (!*bad && off_boundary(4, d_tokens, d_old_logprobs, d_advantages, d_ref_logprobs, d_weights, d_temperature, d_losses, d_logprobs))
        bad = "an array of the rows is not aligned to 4 bytes";
    if (!*bad && !(clip_low >= 0.0f && clip_low <= 1.0f && clip_high >= 0.0f && clip_high <= 3e38f))
        bad = "clip_low must be in [0, 1] and clip_high >= 0";
    if (!*bad && !(kl >= 0.0f && kl <= 3e38f)) bad = "kl must be >= 0";
    if (!*bad && d_grad && grad_stride < V) bad = "the gradient's row stride must be >= V";
    if (!*bad && d_grad && off_boundary(dtype == TRIE_DTYPE_F32 ? 4 : 2, static_cast<const char *>(d_grad)))
        bad = "d_grad is not aligned to its element size";
    if (!*bad && d_grad == d_logits && d_grad && grad_stride != stride && B > 1) bad = "a gradient in place needs the logits' stride";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (B == 0) return TRIE_OK;
    PolicyArgs a = {d_logits, stride, B, V, d_tokens, d_old_logprobs, d_advantages, kl > 0.0f ? d_ref_logprobs : nullptr, d_weights,
                    d_temperature, 1.0f - clip_low, 1.0f + clip_high, kl, make_grammar(d_mask, mask_rows, d_states, V),
                    d_losses, d_logprobs, d_grad, grad_stride, 1, 0, 0, 0};
    const cudaError_t e = dtype == TRIE_DTYPE_F32 ? run_policy<float>(a, stream) : run_policy<__nv_bfloat16>(a, stream);
    if (e != cudaSuccess) return fail_launch(e, "policy loss launch");
    return TRIE_OK;
}
