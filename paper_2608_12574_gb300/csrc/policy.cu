// The clipped policy loss with a KL term of sampled tokens, and its gradient by
// their logits: trie_policy_loss.
//
// Of a row with logits x, token t, and the tokens that its state allows:
//   y = x / temperature,  lp = y[t] - log sum exp y
//   rho = exp(lp - old),  d = ref - lp
//   loss = weight (kl (exp(d) - d - 1) - min(rho A, clip(rho) A))
//   slope = dloss / dlp = weight (kl (1 - exp(d)) - [rho A <= clip(rho) A] rho A)
//   dloss / dx[v] = slope ([v = t] - exp(y[v] - log sum exp y)) / temperature
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include <cuda_runtime.h>

#include "blackwell.cuh"
#include "logits.cuh"

namespace tmk {

namespace {

constexpr int kSlots = 4;               // shares of rows in shared memory, at most
constexpr int kRowSmem = 224 * 1024;
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

// Two numbers at a time.
using Two = unsigned long long;
__device__ __forceinline__ Two two(float x, float y) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 apart(Two x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ Two add2(Two x, Two y) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ Two mul2(Two x, Two y) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
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
        : token(__ldg(a.tokens + b)), state(a.g.mask ? __ldg(a.g.states + b) : TRIE_STATE_FREE), old(__ldg(a.old + b)), advantage(__ldg(a.advantages + b)), ref(a.ref ? __ldg(a.ref + b) : 0.0f),
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
        const float free = rho * v.advantage, held = fminf(fmaxf(rho, a.low), a.high) * v.advantage;
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
    const float per = 1.0f / v.temperature;
    return {all.top, 1.44269504f / v.temperature, -slope / all.sum * per, slope * -expm1f(lp) * per, slope == 0.0f ? -1 : v.token};
}
// Of a token that is not allowed (or has no probability, for which it is the same) 0, whatever f is.
__device__ __forceinline__ float slope_of(const Slope &s, float x) { return x == -INFINITY ? 0.0f : s.f * exp2_of((x - s.top) * s.c); }

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
// go over the rows, a cluster a row. One warp of a CTA, the clerk, asks for a
// free row's shares by bulk copies rows ahead, reads what else a row has, sends
// the CTA's mass of a row to the others and makes its slope; the other
// warps take the masses of a row and then write the gradient of the row before,
// whose slope has had that long to arrive. Of a constrained row only allowed
// tokens are read, word by word of its mask, and its gradient is zeros with
// these put in.
constexpr int kWorkerWarps = 15;
constexpr int kWorkers = 32 * kWorkerWarps;
constexpr int kRowThreads = kWorkers + 64;
constexpr int kTogether = 5;  // pieces that a worker adds up at a time

// What the workers need to know of a row.
template <typename T>
struct RowIn {
    Share<T> share;
    GrammarRow row;
    int32_t listed;   // of a constrained row: its allowed tokens in this share, whose ids and logits are in the slot
    float c;          // log2(e) / temperature
    float edge[16];   // logits outside the pieces
};
struct Listed {
    int32_t token;
    float x;
};

__device__ __forceinline__ void workers_sync() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(kWorkers) : "memory"); }

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 1) k_policy_rows(const PolicyArgs a) {
    constexpr int kSize = Piece<T>::kSize;
    extern __shared__ __align__(128) unsigned char slots[];
    __shared__ uint64_t bars[2 * kSlots + kRanks + 4];
    __shared__ Mass parts[2][32];
    __shared__ Mass ranks[kRanks][kMaxCluster];
    __shared__ __align__(16) unsigned char in_bytes[kSlots * sizeof(RowIn<T>)];
    RowIn<T> *const in = reinterpret_cast<RowIn<T> *>(in_bytes);
    __shared__ Slope slopes[2];
    __shared__ int gave_up;
    const uint32_t full = smem_addr(bars), freed = full + 8 * kSlots;  // of a slot
    const uint32_t masses = freed + 8 * kSlots;                         // of a row, of all its CTAs
    const uint32_t summed = masses + 8 * kRanks, sloped = summed + 8 * 2;
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
        bar_init_fence();
    }
    pdl_launch_dependents();
    if (a.ctas > 1) cluster_sync();  // every CTA's barriers are there
    else __syncthreads();
    pdl_wait();

    const int32_t rows = (a.B - cluster + a.clusters - 1) / a.clusters;
    if (warp == kWorkerWarps) {
        // What there is to know of a row, then its share. What does not need the slot comes before the wait for it.
        for (int32_t r = 0; r < rows; r++) {
            const int32_t b = cluster + r * a.clusters, slot = r % a.slots;
            const Share<T> s(a, b, rank);
            const int32_t state = a.g.mask ? __ldg(a.g.states + b) : TRIE_STATE_FREE;
            const GrammarRow row = grammar_state(a.g, state);
            const float c = 1.44269504f / temperature_of(a, b);
            const int32_t edge = lane < 16 ? s.edge(lane) : -1;
            const float at_edge = edge >= 0 && row.allows(edge) ? to_f32(s.x[edge]) : -INFINITY;
            if (r >= a.slots && !__all_sync(~0u, bar_wait(freed + 8 * slot, (r / a.slots - 1) & 1, &gave_up))) break;
            if (lane < 16) in[slot].edge[lane] = at_edge;
            if (lane == 0) {
                in[slot].share = s;
                in[slot].row = row;
                in[slot].listed = 0;
                in[slot].c = c;
            }
            __syncwarp();
            if (lane == 0) {
                const uint32_t bytes = row.kind == kAllowAll ? uint32_t(s.last - s.first) * 16u : 0u;
                bar_expect(full + 8 * slot, bytes);
                if (bytes) bulk_load(smem_addr(slots + slot * a.slot_bytes), s.pieces() + s.first, bytes, full + 8 * slot);
            }
        }
        return;
    }
    if (warp > kWorkerWarps) {
        // The clerk. It reads a row's values two rows ahead, and its token's logit one, so that it waits for none.
        auto token_logit = [&](int32_t r, const RowValues &v) {
            const int32_t b = cluster + r * a.clusters;
            return v.token >= 0 && v.token < V && grammar_state(a.g, v.state).allows(v.token) ? to_f32(Share<T>(a, b, rank).x[v.token]) : -INFINITY;
        };
        auto values = [&](int32_t r) { return RowValues(a, cluster + min(r, rows - 1) * a.clusters); };
        RowValues next = values(0), after = values(1);
        float xt_next = token_logit(0, next);
        for (int32_t r = 0; r < rows; r++) {
            const int32_t b = cluster + r * a.clusters;
            const RowValues v = next;
            const float xt = xt_next;
            next = after;
            if (r + 1 < rows) xt_next = token_logit(r + 1, next);
            after = values(r + 2);
            const float c = 1.44269504f / v.temperature;
            bool ok = bar_wait(summed + 8 * (r & 1), (r >> 1) & 1, &gave_up);
            Mass all = {-INFINITY, 0.0f};
            if (lane < kWorkerWarps) all = parts[r & 1][lane];
            all = warp_mass(all, c);
            if (a.ctas > 1) {
                if (lane < a.ctas) {
                    *cluster_object(&ranks[r % kRanks][rank], lane) = all;
                    bar_arrive_cluster(cluster_addr(masses + 8 * (r % kRanks), lane));
                }
                __syncwarp();
                ok = bar_wait_cluster(masses + 8 * (r % kRanks), (r / kRanks) & 1, &gave_up) && ok;
                all = {-INFINITY, 0.0f};
                if (lane < a.ctas) all = ranks[r % kRanks][lane];
                all = warp_mass(all, c);
            }
            if (!__all_sync(~0u, ok)) all.sum = __int_as_float(0x7FC00000);  // gave up waiting: no result
            const Slope slope = finish(a, b, all, xt, v, rank == 0 && lane == 0);
            if (lane == 0) {
                slopes[r & 1] = slope;
                bar_arrive(sloped + 8 * (r & 1));
            }
        }
        return;
    }

    const int32_t worker = threadIdx.x, most = a.slot_bytes / int32_t(sizeof(Listed));
    auto first_pass = [&](int32_t r, int slot, uint32_t phase) {
        const bool there = bar_wait(full + 8 * slot, phase, &gave_up);
        RowIn<T> &i = in[slot];
        const float c = i.c;
        unsigned char *const held = slots + slot * a.slot_bytes;
        Mass all = {-INFINITY, 0.0f};
        if (i.row.kind == kAllowAll) {
            if (worker < 16) {
                const float x = i.edge[worker];
                all.top = fmaxf(all.top, x);
                all.sum = exp2_of((x - (all.top == -INFINITY ? 0.0f : all.top)) * c);
            }
            const uint4 *from = reinterpret_cast<const uint4 *>(held) + worker;
            for (int32_t left = i.share.last - i.share.first - worker; left > 0; left -= kTogether * kWorkers) {
                Piece<T> p[kTogether];
#pragma unroll
                for (int k = 0; k < kTogether; k++) {
                    p[k].clear();
                    if (left > k * kWorkers) p[k].set(from[k * kWorkers]);
                }
                add_pieces(all, p, c);
                from += kTogether * kWorkers;
            }
        } else {
            Listed *list = reinterpret_cast<Listed *>(held);
            const Share<T> s = i.share;
            const GrammarRow row = i.row;
            for (int32_t w = (s.lo >> 5) + worker; w * 32 < s.hi; w += kWorkers) {
                for (uint32_t bits = row.word(w); bits; bits &= bits - 1) {
                    const int32_t v = w * 32 + __ffs(bits) - 1;
                    if (v < s.lo || v >= s.hi) continue;
                    const float x = to_f32(s.x[v]), top = fmaxf(all.top, x), off = top == -INFINITY ? 0.0f : top;
                    all.sum = all.sum * exp2_of((all.top - off) * c) + exp2_of((x - off) * c);
                    all.top = top;
                    const int32_t at = atomicAdd(&i.listed, 1);
                    if (at < most) list[at] = {v, x};
                }
            }
        }
        if (!there) all.sum = __int_as_float(0x7FC00000);
        all = warp_mass(all, c);
        if (lane == 0) {
            parts[r & 1][warp] = all;
            bar_arrive(summed + 8 * (r & 1));
        }
    };
    auto second_pass = [&](int32_t r, int slot) {
        bar_wait(sloped + 8 * (r & 1), (r >> 1) & 1, &gave_up);
        if (!a.grad) return;
        const Slope slope = slopes[r & 1];
        const Share<T> s = in[slot].share;
        const int32_t n = s.last - s.first;
        const unsigned char *const held = slots + slot * a.slot_bytes;
        const int32_t edge = worker < 16 ? s.edge(worker) : -1;
        if (in[slot].row.kind == kAllowAll && slope.token >= 0) {
            if (edge >= 0) s.grad[edge] = from_f32<T>(edge == slope.token ? slope.at_token : slope_of(slope, in[slot].edge[worker]));
            const uint4 *from = reinterpret_cast<const uint4 *>(held);
            const int32_t at = slope.token < s.head ? -1 : (slope.token - s.head) / kSize - s.first;  // the token's piece
#pragma unroll 5
            for (int32_t j = worker; j < n; j += kWorkers) {
                Piece<T> p;
                p.set(from[j]);
                s.store(s.first + j, slope_of(slope, p));
                if (j == at) s.grad[slope.token] = from_f32<T>(slope.at_token);
            }
            return;
        }
        const int32_t listed = slope.token >= 0 ? in[slot].listed : 0;
        if (listed <= most) {
            Piece<T> g;
            g.set(make_uint4(0u, 0u, 0u, 0u));
            if (edge >= 0) s.grad[edge] = from_f32<T>(0.0f);
            for (int32_t j = worker; j < n; j += kWorkers) s.store(s.first + j, g);
            workers_sync();
            const Listed *list = reinterpret_cast<const Listed *>(held);
            for (int32_t j = worker; j < listed; j += kWorkers) {
                const Listed one = list[j];
                s.grad[one.token] = from_f32<T>(one.token == slope.token ? slope.at_token : slope_of(slope, one.x));
            }
        } else {
            const GrammarRow row = in[slot].row;
            for (int32_t v = s.lo + worker; v < s.hi; v += kWorkers)
                s.grad[v] = from_f32<T>(!row.allows(v) ? 0.0f : v == slope.token ? slope.at_token : slope_of(slope, to_f32(s.x[v])));
        }
    };
    int slot = 0, slot_next = 0;
    uint32_t phase = 0;  // of slot_next
    auto step = [&] {
        if (++slot_next == a.slots) slot_next = 0, phase ^= 1;
    };
    first_pass(0, 0, 0);
    step();
    for (int32_t r = 0; r < rows; r++) {
        if (r + 1 < rows) first_pass(r + 1, slot_next, phase);
        second_pass(r, slot);
        __syncwarp();
        if (lane == 0) bar_arrive(freed + 8 * slot);
        slot = slot_next;
        step();
    }
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

// Clusters of k_policy_rows<T> of 1 << log_ctas CTAs that the current device runs at once.
template <typename T>
int active_clusters(int log_ctas) {
    static std::atomic<int> known[16][5];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 16) return 1;
    if ((n = known[dev][log_ctas].load(std::memory_order_relaxed))) return n;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1u << log_ctas);
    cfg.blockDim = dim3(kRowThreads);
    cfg.dynamicSmemBytes = size_t(kRowSmem);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1u << log_ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(k_policy_rows<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaFuncSetAttribute(k_policy_rows<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, k_policy_rows<T>, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 0;
    }
    known[dev][log_ctas].store(n, std::memory_order_relaxed);
    return n;
}

template <typename T>
cudaError_t run_policy(PolicyArgs a, cudaStream_t st) {
    // The fewest CTAs a row of which three shares fit; more where the rows are few.
    const int64_t pieces = int64_t(a.V) * int64_t(sizeof(T)) / 16;
    auto share = [&] { return (pieces + a.ctas - 1) / a.ctas * 16; };
    int log_ctas = 0;
    while (a.ctas < kMaxCluster && (share() > kMaxShare || (a.ctas < 8 && int64_t(a.B) * a.ctas * 2 <= sm_count() && share() > 16 * kRowThreads))) {
        a.ctas *= 2;
        log_ctas++;
    }
    a.clusters = share() <= kMaxShare ? std::min(a.B, active_clusters<T>(log_ctas)) : 0;
    if (a.clusters) {
        const int rows = (a.B + a.clusters - 1) / a.clusters;
        a.slot_bytes = std::max(128, int((share() + 127) / 128 * 128));
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
