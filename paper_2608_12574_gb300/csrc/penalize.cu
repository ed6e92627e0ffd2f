// trie_penalize: repetition, presence and frequency penalties, biases and the
// grammar mask on a batch of logits, in place.
//
// With seen(t) and c(t) from the row's history (t anywhere in it; occurrences
// of t after the prompt):
//   l <- l > 0 ? l / r : l * r   where seen(t)
//   l <- (l - f c) - p           where c(t) > 0
//   l <- l + bias(t)
//   l <- -inf                    where the row's state does not allow t
// in 32 bits, each operation rounded to nearest, with one rounding to bf16 at
// the end. Logits that nothing applies to keep their bits and are not read.
//
// k_penalize does two kinds of work, which touch different logits (allowed and
// not allowed ones) and so need no order among them:
//   edits  the row's history and biases are entered into a hash table in shared
//          memory (integer atomics: their order does not matter; a token listed
//          twice among the biases is added up in list order when it is written),
//          then each entry's logit is read and written: what is moved is the
//          history and the touched logits, not the row. A long history is split
//          over several CTAs by a hash of the token, each of which reads all of
//          it and keeps its own. Where a table fills up (long bias lists), the
//          CTA goes over the vocabulary in windows of the table's size instead.
//   fills  -inf into the constrained rows, 16 bytes at a time where nothing is
//          allowed; allowed logits are neither read nor written. Every CTA takes
//          a part, those with a row to edit after it.
//
// What bounds it. One row of 300 tokens: 5.5 us, the chain of waits (length,
// history, table, logit) and the launch. 256 rows of V 152,064 in bf16, 2,000
// tokens, half of them constrained: 22 us, of which the fills alone are 10 (39 MB
// at 4 TB/s) and the edits alone 11; together they move 39 MB in full lines and
// 230,000 logits that lie in a 32-byte sector each. 48 rows with 32,768 tokens:
// 31 us; half of that is the 460,000 touched logits, about 55 sectors a clock
// from L2, and half the history: a CTA reads all of its row's (three read it
// each) and enters a third.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include <cuda_runtime.h>

#include "logits.cuh"

namespace tmk {

namespace {

// History tokens of an edit CTA (at most 0.73 of its table when all differ), and
// its threads: two CTAs an SM with tables of up to 96 KB while a row's history
// fits one of them, else one of 192 KB, because each of a row's CTAs reads all of
// the history. 48 rows with 32,768 tokens: 31 us on three large CTAs, 36 on six
// small ones. 256 rows with 2,000: 22 us on small ones; large ones would take
// two rounds of the SMs.
constexpr int kShare = 6000, kMostShare = 12000;
constexpr int kThreads = 512, kMostThreads = 1024;
constexpr int kTableBits = 14;           // most entries of an edit CTA's table
constexpr int kLeastBits = 10;           // fewest: room for some hundred biases
constexpr int kProbes = 128;             // past this the table counts as full
constexpr int kAhead = 4;                // 16-byte reads of the history in flight a thread
constexpr int kWrites = 4;               // logits in flight a thread
constexpr int kQueue = 31 + (kWrites + 1) * 32;  // of a warp: less than a batch of writes, and two slots a lane
static_assert(kQueue >= 31 + 4 * 32, "or what was left, and four tokens a lane");
constexpr int kSegment = 1024;           // tokens of a row that a warp fills at a time (2,048: 10 -> 12 us for 39 MB)
// A table's key: a token, and whether it is in the prompt.
constexpr uint32_t kNoToken = 0xFFFFFFFFu;
constexpr uint32_t kPrompt = 0x80000000u;
// Beside the count of a key's occurrences in the output:
constexpr uint32_t kBiased = 0x40000000u;  // it has a bias
constexpr uint32_t kAgain = 0x20000000u;   // it has several
constexpr uint32_t kCount = 0x1FFFFFFFu;

struct PenalizeArgs {
    void *logits;
    int64_t stride;
    int32_t V;
    const int32_t *history;  // [B] rows of history_stride, of which H may be used
    int64_t history_stride;
    int32_t H;
    const int32_t *length;
    const int32_t *prompt;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_offsets, *bias_tokens;
    const float *bias_values;
    int32_t B, shards;       // edit CTAs of a row
    int32_t bits;            // of the table's size
    Grammar g;
};

struct Table {
    uint32_t *key, *entry;
    float *bias;
    int bits, size;
    __device__ Table(unsigned char *smem, int bits_) : bits(bits_), size(1 << bits_) {
        key = reinterpret_cast<uint32_t *>(smem);
        entry = key + size;
        bias = reinterpret_cast<float *>(entry + size);
    }
};

__device__ __forceinline__ uint32_t mix(uint32_t t) {
    t *= 0x9E3779B1u;
    return t ^ (t >> 15);
}
__device__ __forceinline__ bool in_shard(const PenalizeArgs &a, uint32_t t, uint32_t shard) {
    return a.shards == 1 || __umulhi(t * 0x85EBCA6Bu, uint32_t(a.shards)) == shard;
}

// Enters a key (kNoToken: none) into the hash table, or (base >= 0) into the window
// of tokens base .. base + table.size - 1. Its slot; -1: none, not in the window,
// or the table is full, which also clears `fits`. A slot never changes its token,
// so a frequent token costs a read, not an atomic that all lanes queue for.
__device__ __forceinline__ int32_t enter_key(const Table &table, int64_t base, uint32_t key, bool &fits) {
    const uint32_t t = key & ~kPrompt;
    if (key == kNoToken || (base >= 0 && (int64_t(t) < base || int64_t(t) >= base + table.size))) return -1;
    int32_t at = base < 0 ? int32_t((mix(t) * 0xC2B2AE35u) >> (32 - table.bits)) : int32_t(int64_t(t) - base);
    for (int n = 0; n < kProbes; n++) {
        uint32_t old = *static_cast<volatile uint32_t *>(table.key + at);
        if (old == kNoToken) old = atomicCAS(table.key + at, kNoToken, key);
        if (old == kNoToken || old == key) return at;
        if (((old ^ key) & ~kPrompt) == 0u) {
            if (key & kPrompt) atomicOr(table.key + at, kPrompt);
            return at;
        }
        at = (at + 1) & (table.size - 1);
    }
    fits = false;
    return -1;
}

// Enters the row's history and biases, those of this CTA's shard. Of a row on
// several CTAs a warp first gathers the tokens that are this CTA's in a queue and
// enters 32 at a time: of those that its lanes read only one in `shards` is.
__device__ __forceinline__ bool enter(const PenalizeArgs &a, const Table &table, uint32_t *queue, int32_t b, uint32_t shard, int64_t base) {
    bool fits = true;
    const int lane = threadIdx.x & 31, threads = blockDim.x;
    if (a.history) {
        const int32_t *h = a.history + b * a.history_stride;
        // to a 16-byte boundary, by fours, and the rest: of max_length, so that the first
        // reads go out together with that of the length
        const int32_t head = min(a.H, int32_t((16 - (reinterpret_cast<uintptr_t>(h) & 15)) & 15) / 4);
        const int32_t fours = (a.H - head) / 4, tail = head + fours * 4;
        const int4 *q = reinterpret_cast<const int4 *>(h + head);
        int4 x[kAhead];
        auto read = [&](int32_t i) {
#pragma unroll
            for (int n = 0; n < kAhead; n++)
                x[n] = i + n * threads < fours ? __ldg(q + i + n * threads) : make_int4(-1, -1, -1, -1);
        };
        read(int32_t(threadIdx.x));
        int32_t odd_at = lane < 4 ? lane : tail + lane - 4;  // of warp 0: the head, and the rest
        if (threadIdx.x >= 8 || (lane < 4 ? odd_at >= head : odd_at >= a.H)) odd_at = -1;
        const uint32_t odd = odd_at >= 0 ? uint32_t(__ldg(h + odd_at)) : kNoToken;
        const int32_t len = max(0, min(__ldg(a.length + b), a.H));
        const int32_t prompt = a.prompt ? max(0, __ldg(a.prompt + b)) : 0;
        auto key_of = [&](int32_t i, uint32_t t) { return i >= len || t >= uint32_t(a.V) ? kNoToken : i < prompt ? t | kPrompt : t; };
        auto say = [&](uint32_t key) {
            const int32_t at = enter_key(table, base, key, fits);
            if (at >= 0 && key < kPrompt) atomicAdd(table.entry + at, 1u);
        };
        int32_t queued = 0;  // the warp's
        auto push = [&](uint32_t key) {
            const bool mine = key != kNoToken && in_shard(a, key & ~kPrompt, shard);
            const uint32_t all = __ballot_sync(~0u, mine);
            if (mine) queue[queued + __popc(all & ((1u << lane) - 1u))] = key;
            queued += __popc(all);
        };
        push(key_of(odd_at, odd));
        const int32_t end = min(fours, (len - head + 3) / 4);
        int32_t i0 = int32_t(threadIdx.x) - lane, n = 0;
        while (true) {
            const bool more = i0 + n * threads < end && __all_sync(~0u, fits);
            if (more) {  // four tokens a lane
                const int4 y = n == 0 ? x[0] : n == 1 ? x[1] : n == 2 ? x[2] : x[3];
                const int32_t i = head + 4 * (i0 + lane + n * threads);
                if (++n == kAhead) {
                    i0 += kAhead * threads, n = 0;
                    read(i0 + lane);
                }
                const uint32_t k0 = key_of(i, uint32_t(y.x)), k1 = key_of(i + 1, uint32_t(y.y));
                const uint32_t k2 = key_of(i + 2, uint32_t(y.z)), k3 = key_of(i + 3, uint32_t(y.w));
                if (a.shards == 1) {
                    say(k0), say(k1), say(k2), say(k3);
                    continue;
                }
                push(k0), push(k1), push(k2), push(k3);
            }
            __syncwarp();
            while (queued >= 32 || (!more && queued > 0)) {
                queued -= 32;
                say(queued + lane >= 0 ? queue[queued + lane] : kNoToken);
            }
            __syncwarp();
            if (!more) break;
        }
    }
    if (a.bias_offsets) {
        const int32_t lo = __ldg(a.bias_offsets + b), hi = __ldg(a.bias_offsets + b + 1);
        for (int32_t i = lo + int32_t(threadIdx.x); i < hi && fits; i += threads) {
            const uint32_t t = uint32_t(__ldg(a.bias_tokens + i));
            const float value = __ldg(a.bias_values + i);
            const int32_t at = t >= uint32_t(a.V) || !in_shard(a, t, shard) ? -1 : enter_key(table, base, t, fits);
            if (at < 0) continue;
            if (atomicOr(table.entry + at, kBiased) & kBiased) atomicOr(table.entry + at, kAgain);
            else table.bias[at] = value;
        }
    }
    return fits;
}

__device__ __forceinline__ float bias_sum(const PenalizeArgs &a, int32_t b, int32_t t) {
    const int32_t lo = __ldg(a.bias_offsets + b), hi = __ldg(a.bias_offsets + b + 1);
    float sum = 0.0f;
    bool first = true;
    for (int32_t i = lo; i < hi; i++)
        if (__ldg(a.bias_tokens + i) == t) {
            sum = first ? __ldg(a.bias_values + i) : __fadd_rn(sum, __ldg(a.bias_values + i));
            first = false;
        }
    return sum;
}

struct Rates {
    float r, p, f;
};

__device__ __forceinline__ float penalized(float x, bool in_prompt, uint32_t entry, const Rates &k, float bias) {
    const uint32_t c = entry & kCount;
    if (c || in_prompt) x = x > 0.0f ? __fdiv_rn(x, k.r) : __fmul_rn(x, k.r);
    if (c) x = __fsub_rn(__fsub_rn(x, __fmul_rn(k.f, float(c))), k.p);
    if (entry & kBiased) x = __fadd_rn(x, bias);
    return x;
}

// Writes the logits of the table's entries (base >= 0: a window's) and clears it.
template <typename T>
__device__ __forceinline__ void write_entries(const PenalizeArgs &a, const Table &table, uint32_t *queue, int32_t b, const Rates &k,
                                              const GrammarRow &row, T *logits) {
    const int lane = threadIdx.x & 31, threads = blockDim.x;
    // the first n slots of the queue
    auto write = [&](int n) {
        __syncwarp();
        int32_t slot[kWrites], t[kWrites];
        uint32_t key[kWrites], entry[kWrites];
        float x[kWrites];
#pragma unroll
        for (int i = 0; i < kWrites; i++) {
            const bool there = lane + 32 * i < n;
            slot[i] = there ? int32_t(queue[lane + 32 * i]) : 0;
            key[i] = there ? table.key[slot[i]] : kNoToken;
            entry[i] = there ? table.entry[slot[i]] : 0u;
        }
#pragma unroll
        for (int i = 0; i < kWrites; i++) {
            t[i] = int32_t(key[i] & ~kPrompt);
            if (key[i] != kNoToken && !row.allows(t[i])) key[i] = kNoToken;
        }
#pragma unroll
        for (int i = 0; i < kWrites; i++) x[i] = key[i] != kNoToken ? to_f32(logits[t[i]]) : 0.0f;
#pragma unroll
        for (int i = 0; i < kWrites; i++) {
            if (key[i] == kNoToken) continue;
            const float bias = entry[i] & kAgain ? bias_sum(a, b, t[i]) : table.bias[slot[i]];
            logits[t[i]] = from_f32<T>(penalized(x[i], key[i] & kPrompt, entry[i], k, bias));
        }
        __syncwarp();
    };
    int queued = 0;
    for (int s = 2 * threadIdx.x;; s += 2 * threads) {  // two slots a lane
        const bool more = s - 2 * int(threadIdx.x) < table.size;  // the whole block's
        if (more) {
            const uint2 k2 = *reinterpret_cast<const uint2 *>(table.key + s);
            const uint32_t first = __ballot_sync(~0u, k2.x != kNoToken), second = __ballot_sync(~0u, k2.y != kNoToken);
            if (k2.x != kNoToken) queue[queued + __popc(first & ((1u << lane) - 1u))] = uint32_t(s);
            queued += __popc(first);
            if (k2.y != kNoToken) queue[queued + __popc(second & ((1u << lane) - 1u))] = uint32_t(s + 1);
            queued += __popc(second);
        }
        if (queued >= kWrites * 32 || (!more && queued)) {
            write(min(queued, kWrites * 32));
            queued = max(queued - kWrites * 32, 0);  // fewer than 64 are left
            const uint32_t rest = lane < queued ? queue[kWrites * 32 + lane] : 0u;
            const uint32_t more_rest = lane + 32 < queued ? queue[kWrites * 32 + 32 + lane] : 0u;
            __syncwarp();
            queue[lane] = rest, queue[lane + 32] = more_rest;
            __syncwarp();  // before other lanes enter theirs at these places
        }
        if (!more) break;
    }
}

__device__ __forceinline__ void clear(const Table &table) {
    for (int i = threadIdx.x; i < table.size / 4; i += int(blockDim.x)) {
        reinterpret_cast<uint4 *>(table.key)[i] = make_uint4(kNoToken, kNoToken, kNoToken, kNoToken);
        reinterpret_cast<uint4 *>(table.entry)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
}

template <typename T>
__device__ __forceinline__ void edit_row(const PenalizeArgs &a, const Table &table, int32_t b, uint32_t shard) {
    uint32_t *const queue = reinterpret_cast<uint32_t *>(table.bias + table.size) + (threadIdx.x >> 5) * kQueue;
    T *logits = static_cast<T *>(a.logits) + b * a.stride;
    Rates k;
    k.r = a.repetition ? __ldg(a.repetition + b) : 1.0f;
    k.p = a.presence ? __ldg(a.presence + b) : 0.0f;
    k.f = a.frequency ? __ldg(a.frequency + b) : 0.0f;
    const GrammarRow row = grammar_row(a.g, b);
    int64_t base = -1;
    while (true) {
        const bool fits = enter(a, table, queue, b, shard, base);
        if (__syncthreads_and(fits)) {
            write_entries(a, table, queue, b, k, row, logits);
            if (base < 0) return;
            base += table.size;
        } else {  // by windows from here on: they always fit
            base = 0;
        }
        if (base >= a.V) return;
        __syncthreads();
        clear(table);
        __syncthreads();
    }
}

// -inf into the tokens v0 .. v1 - 1 of a row that are not allowed, by one warp.
template <typename T>
__device__ __forceinline__ void fill_segment(const GrammarRow &row, T *logits, int32_t V, int32_t v0, int32_t v1, int lane) {
    constexpr int kVec = 16 / sizeof(T), kSteps = kSegment / kVec / 32;
    const T none = from_f32<T>(-INFINITY);
    const uint32_t pair = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    const uint4 fill = make_uint4(pair, pair, pair, pair);
    const int32_t last = (V - 1) >> 5;
    // chunks of 16 bytes by address; the first may begin before v0, the last end past v1
    const int32_t ahead = int32_t((reinterpret_cast<uintptr_t>(logits + v0) & 15) / sizeof(T));
    uint32_t bits[kSteps + 1];
#pragma unroll
    for (int i = 0; i <= kSteps; i++) {
        const int32_t t = v0 - ahead + (lane + 32 * i) * kVec, w = t >> 5;  // the chunk's first token
        const bool there = t < v1;
        const uint32_t lo = there && w >= 0 ? row.word(w) : 0u;
        const uint32_t hi = there && (t & 31) > 32 - kVec && w < last ? row.word(w + 1) : 0u;
        bits[i] = __funnelshift_r(lo, hi, t & 31) & ((1u << kVec) - 1u);
        if (i == kSteps - 1 && ahead == 0) break;  // no chunk more than a segment has
    }
#pragma unroll
    for (int i = 0; i <= kSteps; i++) {
        const int32_t t = v0 - ahead + (lane + 32 * i) * kVec;
        if (t >= v1) break;
        if (bits[i] == 0u && t >= v0 && t + kVec <= v1) {
            *reinterpret_cast<uint4 *>(logits + t) = fill;
        } else {
#pragma unroll
            for (int n = 0; n < kVec; n++)
                if (!((bits[i] >> n) & 1u) && t + n >= v0 && t + n < v1) logits[t + n] = none;
        }
    }
}

// This CTA's part of the fills: `shares` of `all` equal parts of the constrained
// rows' segments, from part `share` on. Which rows are constrained is counted
// first, for a row a thread at a time: half of a batch that is free would
// otherwise leave some CTAs with twice the work of others.
template <typename T>
__device__ __forceinline__ void fill_part(const PenalizeArgs &a, int2 *rows, uint32_t share, uint32_t shares, uint32_t all) {
    __shared__ int32_t counts[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, threads = blockDim.x;
    const int32_t segments = (a.V + kSegment - 1) / kSegment;
    for (int32_t b0 = 0; b0 < a.B; b0 += threads) {
        const int32_t b = b0 + int32_t(threadIdx.x);
        const int32_t state = b < a.B ? __ldg(a.g.states + b) : TRIE_STATE_FREE;
        const bool mine = state != TRIE_STATE_FREE;
        const uint32_t found = __ballot_sync(~0u, mine);
        __syncthreads();
        if (lane == 0) counts[warp] = __popc(found);
        __syncthreads();
        const int32_t n = lane < threads / 32 ? counts[lane] : 0;
        const int32_t before = __reduce_add_sync(~0u, lane < warp ? n : 0), total = __reduce_add_sync(~0u, n);
        if (mine) rows[before + __popc(found & ((1u << lane) - 1u))] = make_int2(b, state);
        __syncthreads();
        const uint64_t work = uint64_t(total) * uint32_t(segments);
        const uint64_t from = work * share / all, to = work * (share + shares) / all;
        for (uint64_t i = from + uint32_t(warp); i < to; i += threads / 32) {
            const int2 r = rows[i / uint32_t(segments)];
            const int32_t v0 = int32_t(i % uint32_t(segments)) * kSegment;
            fill_segment<T>(grammar_state(a.g, r.y), static_cast<T *>(a.logits) + r.x * a.stride, a.V, v0, v0 + min(kSegment, a.V - v0), lane);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kMostThreads) k_penalize(PenalizeArgs a) {
    extern __shared__ __align__(16) unsigned char dynamic_smem[];
    const Table table(dynamic_smem, a.bits);
    const uint32_t edits = uint32_t(a.B) * uint32_t(a.shards);
    if (blockIdx.x < edits) {
        clear(table);
        __syncthreads();
    }
    pdl_launch_dependents();
    pdl_wait();
    if (blockIdx.x < edits) {
        edit_row<T>(a, table, int32_t(blockIdx.x / uint32_t(a.shards)), blockIdx.x % uint32_t(a.shards));
    }
    if (!a.g.mask) return;
    if (blockIdx.x < edits) __syncthreads();  // the table is read no more
    // one part for an edit CTA, which comes to them late, and two for a fill CTA
    const uint32_t all = 2 * gridDim.x - edits, extra = blockIdx.x < edits ? 0 : blockIdx.x - edits;
    fill_part<T>(a, reinterpret_cast<int2 *>(dynamic_smem), blockIdx.x + extra, blockIdx.x < edits ? 1 : 2, all);
}

template <typename T>
cudaError_t launch_penalize(const PenalizeArgs &a, int64_t grid, int threads, cudaStream_t st) {
    constexpr size_t queue = sizeof(uint32_t) * kQueue;
    const cudaError_t e = cudaFuncSetAttribute(k_penalize<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               int((12 << kTableBits) + kMostThreads / 32 * queue));
    if (e != cudaSuccess) return e;
    return launch_pdl_smem(k_penalize<T>, grid, threads, (size_t(12) << a.bits) + threads / 32 * queue, st, a);
}

}  // namespace

}  // namespace tmk

extern "C" int trie_penalize(void *d_logits, int dtype, int64_t stride, int32_t B, int32_t V,
                             const int32_t *d_history, int64_t history_stride, int32_t max_length,
                             const int32_t *d_length, const int32_t *d_prompt, const float *d_repetition,
                             const float *d_presence, const float *d_frequency, const int32_t *d_bias_offsets,
                             const int32_t *d_bias_tokens, const float *d_bias_values, const uint32_t *d_mask,
                             int32_t mask_rows, const int32_t *d_states, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_logits(d_logits, dtype, stride, B, V);
    if (!*bad) bad = check_grammar(d_mask, mask_rows, d_states);
    if (!d_history) max_length = 0;  // of no history
    if (!*bad && d_history) {
        if (!d_length) bad = "d_history without d_length";
        else if (max_length < 0 || max_length > (1 << 28)) bad = "max_length must be in [0, 2^28]";
        else if (history_stride < max_length) bad = "history_stride must be >= max_length";
    }
    if (!*bad && d_bias_offsets && (!d_bias_tokens || !d_bias_values))
        bad = "d_bias_offsets without d_bias_tokens and d_bias_values";
    if (!*bad && off_boundary(4, d_history, d_length, d_prompt, d_repetition, d_presence, d_frequency, d_bias_offsets,
                              d_bias_tokens, d_bias_values))
        bad = "an array is not aligned to 4 bytes";
    if (!*bad && B > 65535) bad = "B must be <= 65535";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (B == 0) return TRIE_OK;
    PenalizeArgs a;
    a.logits = d_logits;
    a.stride = stride;
    a.V = V;
    a.history = d_history;
    a.history_stride = history_stride;
    a.H = max_length;
    a.length = d_length;
    a.prompt = d_prompt;
    a.repetition = d_repetition;
    a.presence = d_presence;
    a.frequency = d_frequency;
    a.bias_offsets = d_bias_offsets;
    a.bias_tokens = d_bias_tokens;
    a.bias_values = d_bias_values;
    a.g = make_grammar(d_mask, mask_rows, d_states, V);
    const bool any = (d_history && max_length > 0) || d_bias_offsets;
    a.B = B;
    const int threads = max_length > kShare ? kMostThreads : kThreads;
    a.shards = !any ? 0 : max_length > kMostShare ? (max_length + kMostShare - 1) / kMostShare : 1;
    a.bits = kLeastBits;
    while (a.bits < kTableBits && (3 << a.bits) / 4 < max_length) a.bits++;
    const int64_t edits = int64_t(B) * a.shards;
    // fill CTAs take the places that the edits leave of one round of CTAs, if there is work for them:
    // 2^14 tokens at least
    const int64_t round = int64_t(sm_count()) * (kMostThreads / threads);
    const int64_t parts = d_mask ? (int64_t(B) * V + (1 << 14) - 1) >> 14 : 0;
    const int64_t fills = std::min(parts, std::max(int64_t(edits ? 0 : 1), round - edits));
    if (edits + fills == 0) return TRIE_OK;  // nothing applies
    if (edits + fills > 0x7FFFFFFF) return set_error(TRIE_EINVAL, "B times max_length is too large");
    const cudaError_t e = dtype == TRIE_DTYPE_F32 ? launch_penalize<float>(a, edits + fills, threads, stream)
                                                  : launch_penalize<__nv_bfloat16>(a, edits + fills, threads, stream);
    if (e != cudaSuccess) return fail_launch(e, "penalize launch");
    return TRIE_OK;
}
