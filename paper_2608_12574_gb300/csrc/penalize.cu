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
// k_penalize has CTAs of two kinds, which touch different logits (allowed and
// not allowed ones) and so need no order among them:
//   edits  the row's history and biases are entered into a hash table in shared
//          memory (integer atomics: their order does not matter; a token listed
//          twice among the biases is added up in list order when it is written),
//          then each entry's logit is read and written: what is moved is the
//          history and the touched logits, not the row. A long history is split
//          over several CTAs by a hash of the token, each of which reads all of
//          it and keeps its own. Where a table fills up (long bias lists), the
//          CTA goes over the vocabulary in windows of the table's size instead.
//   fills  -inf into a segment of a constrained row, 16 bytes at a time where
//          nothing is allowed; allowed logits are neither read nor written.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include <cuda_runtime.h>

#include "logits.cuh"

namespace tmk {

namespace {

constexpr int kThreads = 256;
constexpr int kTableBits = 12;           // most entries of an edit CTA's table: 48 KB, four CTAs an SM
constexpr int kLeastBits = 10;           // fewest: room for some hundred biases
constexpr int kShare = 3000;             // history tokens of one edit CTA: at most 0.73 of the table when all differ
constexpr int kProbes = 128;             // past this the table counts as full
constexpr int kSegment = 16384;          // tokens filled at a time
constexpr int kCtasPerSm = 4;
constexpr uint32_t kNoToken = 0xFFFFFFFFu;
// beside the count of an entry's occurrences in the output:
constexpr uint32_t kPrompt = 0x80000000u;  // it is in the prompt
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
    uint32_t *token, *entry;
    float *bias;
    int bits, size;
    __device__ Table(unsigned char *smem, int bits_) : bits(bits_), size(1 << bits_) {
        token = reinterpret_cast<uint32_t *>(smem);
        entry = token + size;
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

// The slot of token t, entered if it is not there; -1: the table is full. A slot
// never changes once it holds a token, so one that is seen to hold t is t's:
// frequent tokens then cost a read, not an atomic that all lanes queue for.
__device__ __forceinline__ int32_t slot_of(const Table &table, uint32_t t) {
    uint32_t at = (mix(t) * 0xC2B2AE35u) >> (32 - table.bits);
    for (int i = 0; i < kProbes; i++) {
        uint32_t old = *static_cast<volatile uint32_t *>(table.token + at);
        if (old == kNoToken) old = atomicCAS(table.token + at, kNoToken, t);
        if (old == kNoToken || old == t) return int32_t(at);
        at = (at + 1) & uint32_t(table.size - 1);
    }
    return -1;
}

// Enters the row's history and biases. `base` < 0: into the hash table (false
// when it is full); else into the window of tokens base .. base + table.size - 1.
__device__ bool enter(const PenalizeArgs &a, const Table &table, int32_t b, uint32_t shard, int64_t base) {
    bool fits = true;
    auto find = [&](uint32_t t) -> int32_t {
        if (t >= uint32_t(a.V) || !in_shard(a, t, shard)) return -2;
        if (base >= 0) return int64_t(t) >= base && int64_t(t) < base + table.size ? int32_t(int64_t(t) - base) : -2;
        const int32_t at = slot_of(table, t);
        fits &= at >= 0;
        return at;
    };
    if (a.history) {
        const int32_t len = max(0, min(__ldg(a.length + b), a.H));
        const int32_t prompt = a.prompt ? __ldg(a.prompt + b) : 0;
        const int32_t *h = a.history + b * a.history_stride;
        auto say = [&](int32_t i, uint32_t t) {
            const int32_t at = find(t);
            if (at < 0) return;
            if (i >= prompt) atomicAdd(table.entry + at, 1u);
            else if (!(*static_cast<volatile uint32_t *>(table.entry + at) & kPrompt)) atomicOr(table.entry + at, kPrompt);
        };
        // to a 16-byte boundary, by fours, and the rest
        const int32_t head = min(len, int32_t((16 - (reinterpret_cast<uintptr_t>(h) & 15)) & 15) / 4);
        const int32_t fours = (len - head) / 4, tail = head + fours * 4;
        if (int32_t(threadIdx.x) < head) say(int32_t(threadIdx.x), uint32_t(__ldg(h + threadIdx.x)));
        const int4 *q = reinterpret_cast<const int4 *>(h + head);
        for (int32_t i = threadIdx.x; i < fours && fits; i += 2 * kThreads) {
            const bool two = i + kThreads < fours;
            const int4 x = __ldg(q + i), y = two ? __ldg(q + i + kThreads) : make_int4(-1, -1, -1, -1);
            const int32_t at = head + 4 * i, next = at + 4 * kThreads;
            say(at, uint32_t(x.x)), say(at + 1, uint32_t(x.y)), say(at + 2, uint32_t(x.z)), say(at + 3, uint32_t(x.w));
            if (two) say(next, uint32_t(y.x)), say(next + 1, uint32_t(y.y)), say(next + 2, uint32_t(y.z)), say(next + 3, uint32_t(y.w));
        }
        if (tail + int32_t(threadIdx.x) < len) say(tail + int32_t(threadIdx.x), uint32_t(__ldg(h + tail + threadIdx.x)));
    }
    if (a.bias_offsets) {
        const int32_t lo = __ldg(a.bias_offsets + b), hi = __ldg(a.bias_offsets + b + 1);
        for (int32_t i = lo + int32_t(threadIdx.x); i < hi && fits; i += kThreads) {
            const int32_t at = find(uint32_t(__ldg(a.bias_tokens + i)));
            if (at < 0) continue;
            if (atomicOr(table.entry + at, kBiased) & kBiased) atomicOr(table.entry + at, kAgain);
            else table.bias[at] = __ldg(a.bias_values + i);
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

__device__ __forceinline__ float penalized(float x, uint32_t entry, const Rates &k, float bias) {
    const uint32_t c = entry & kCount;
    if (c || (entry & kPrompt)) x = x > 0.0f ? __fdiv_rn(x, k.r) : __fmul_rn(x, k.r);
    if (c) x = __fsub_rn(__fsub_rn(x, __fmul_rn(k.f, float(c))), k.p);
    if (entry & kBiased) x = __fadd_rn(x, bias);
    return x;
}

// Writes the logits of the table's entries (base >= 0: a window's) and clears it.
template <typename T>
__device__ void write_entries(const PenalizeArgs &a, const Table &table, int32_t b, T *logits, int64_t base) {
    Rates k;
    k.r = a.repetition ? __ldg(a.repetition + b) : 1.0f;
    k.p = a.presence ? __ldg(a.presence + b) : 0.0f;
    k.f = a.frequency ? __ldg(a.frequency + b) : 0.0f;
    const GrammarRow row = grammar_row(a.g, b);
    constexpr int kBatch = 4;  // reads in flight a thread; divides the smallest table / kThreads
    for (int s0 = threadIdx.x; s0 < table.size; s0 += kBatch * kThreads) {
        uint32_t entry[kBatch];
        int32_t t[kBatch];
        float x[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; i++) {
            entry[i] = table.entry[s0 + i * kThreads];
            t[i] = base >= 0 ? int32_t(base) + s0 + i * kThreads : int32_t(table.token[s0 + i * kThreads]);
            if (entry[i] && !row.allows(t[i])) entry[i] = 0u;
        }
#pragma unroll
        for (int i = 0; i < kBatch; i++) x[i] = entry[i] ? to_f32(logits[t[i]]) : 0.0f;
#pragma unroll
        for (int i = 0; i < kBatch; i++) {
            if (!entry[i]) continue;
            const float bias = entry[i] & kAgain ? bias_sum(a, b, t[i]) : table.bias[s0 + i * kThreads];
            logits[t[i]] = from_f32<T>(penalized(x[i], entry[i], k, bias));
        }
    }
}

__device__ __forceinline__ void clear(const Table &table) {
    for (int i = threadIdx.x; i < table.size / 4; i += kThreads) {
        reinterpret_cast<uint4 *>(table.token)[i] = make_uint4(kNoToken, kNoToken, kNoToken, kNoToken);
        reinterpret_cast<uint4 *>(table.entry)[i] = make_uint4(0u, 0u, 0u, 0u);
    }
}

template <typename T>
__device__ void edit_row(const PenalizeArgs &a, const Table &table, int32_t b, uint32_t shard) {
    T *logits = static_cast<T *>(a.logits) + b * a.stride;
    const bool fits = enter(a, table, b, shard, -1);
    if (__syncthreads_and(fits)) {
        write_entries(a, table, b, logits, -1);
        return;
    }
    for (int64_t base = 0; base < a.V; base += table.size) {
        clear(table);
        __syncthreads();
        enter(a, table, b, shard, base);
        __syncthreads();
        write_entries(a, table, b, logits, base);
        __syncthreads();
    }
}

// -inf into the tokens v0 .. v1 - 1 of row b that its state does not allow.
template <typename T>
__device__ void fill_segment(const PenalizeArgs &a, int32_t b, int32_t v0, int32_t v1) {
    constexpr int kVec = 16 / sizeof(T);
    const GrammarRow row = grammar_row(a.g, b);
    if (row.kind == kAllowAll) return;
    T *logits = static_cast<T *>(a.logits) + b * a.stride;
    const T none = from_f32<T>(-INFINITY);
    // chunks of 16 bytes by address; the first may begin before v0, the last end past v1
    const int32_t ahead = int32_t((reinterpret_cast<uintptr_t>(logits + v0) & 15) / sizeof(T));
    const int32_t last = (a.V - 1) >> 5;
    const uint32_t pair = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    const uint4 fill = make_uint4(pair, pair, pair, pair);
#pragma unroll 4
    for (int32_t c = threadIdx.x; c * kVec < v1 - v0 + ahead; c += kThreads) {
        const int32_t t = v0 - ahead + c * kVec;  // the chunk's first token
        const int32_t w = t >> 5;
        const uint32_t lo = w >= 0 ? row.word(w) : 0u, hi = (t & 31) > 32 - kVec && w < last ? row.word(w + 1) : 0u;
        const uint32_t bits = __funnelshift_r(lo, hi, t & 31) & ((1u << kVec) - 1u);
        if (bits == 0u && t >= v0 && t + kVec <= v1) {
            *reinterpret_cast<uint4 *>(logits + t) = fill;
        } else {
#pragma unroll
            for (int i = 0; i < kVec; i++)
                if (!((bits >> i) & 1u) && t + i >= v0 && t + i < v1) logits[t + i] = none;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) k_penalize(PenalizeArgs a) {
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
        return;
    }
    const uint32_t segments = (uint32_t(a.V) + kSegment - 1) / kSegment;
    for (uint64_t i = blockIdx.x - edits; i < uint64_t(a.B) * segments; i += gridDim.x - edits) {
        const int32_t v0 = int32_t(i % segments) * kSegment;
        fill_segment<T>(a, int32_t(i / segments), v0, v0 + min(kSegment, a.V - v0));
    }
}

template <typename T>
cudaError_t launch_penalize(const PenalizeArgs &a, int64_t grid, cudaStream_t st) {
    return launch_pdl_smem(k_penalize<T>, grid, kThreads, size_t(12) << a.bits, st, a);
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
    if (!*bad && d_history) {
        if (!d_length) bad = "d_history without d_length";
        else if (max_length < 0 || max_length > (1 << 28)) bad = "max_length must be in [0, 2^28]";
        else if (history_stride < max_length) bad = "history_stride must be >= max_length";
    }
    if (!*bad && d_bias_offsets && (!d_bias_tokens || !d_bias_values))
        bad = "d_bias_offsets without d_bias_tokens and d_bias_values";
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
    a.shards = !any ? 0 : max_length > kShare ? (max_length + kShare - 1) / kShare : 1;
    a.bits = kLeastBits;
    while (a.bits < kTableBits && (3 << a.bits) / 4 < max_length) a.bits++;
    const int64_t edits = int64_t(B) * a.shards;
    const int64_t segments = d_mask ? (int64_t(V) + kSegment - 1) / kSegment * B : 0;
    // fill CTAs take the places that the edits leave of one round of CTAs, and half of one at least
    const int64_t round = int64_t(sm_count()) * kCtasPerSm;
    const int64_t fills = std::min(segments, std::max(round / 2, round - edits));
    if (edits + fills == 0) return TRIE_OK;  // nothing applies
    if (edits + fills > 0x7FFFFFFF) return set_error(TRIE_EINVAL, "B times max_length is too large");
    const cudaError_t e = dtype == TRIE_DTYPE_F32 ? launch_penalize<float>(a, edits + fills, stream)
                                                  : launch_penalize<__nv_bfloat16>(a, edits + fills, stream);
    if (e != cudaSuccess) return fail_launch(e, "penalize launch");
    return TRIE_OK;
}
