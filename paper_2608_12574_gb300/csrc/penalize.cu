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
//  k_penalize  one CTA per row and window of kWindow tokens: the row's history
//              is counted into a shared-memory table of the window (integer
//              atomics, so the order does not matter), its biases are added
//              up in list order, and the window's logits are written where
//              something applies.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <cuda_runtime.h>

#include "logits.cuh"

namespace tmk {

namespace {

constexpr int kThreads = 256;
constexpr int kWindow = 8192;
constexpr uint32_t kSeen = 0x80000000u;  // beside the count of a table entry

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
    Grammar g;
};

__device__ __forceinline__ float penalized(float x, uint32_t entry, float r, float p, float f) {
    if (!entry) return x;
    x = x > 0.0f ? __fdiv_rn(x, r) : __fmul_rn(x, r);
    const uint32_t c = entry & ~kSeen;
    if (c) x = __fsub_rn(__fsub_rn(x, __fmul_rn(f, float(c))), p);
    return x;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_penalize(PenalizeArgs a) {
    __shared__ uint32_t count[kWindow];
    __shared__ float bias[kWindow];
    const int32_t b = blockIdx.y;
    const int32_t v0 = blockIdx.x * kWindow, v1 = min(a.V - v0, kWindow) + v0;
    const uint32_t n = v1 - v0;
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
        count[i] = 0u;
        bias[i] = 0.0f;
    }
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();
    if (a.history) {
        const int32_t len = max(0, min(__ldg(a.length + b), a.H));
        const int32_t prompt = a.prompt ? __ldg(a.prompt + b) : 0;
        const int32_t *h = a.history + b * a.history_stride;
        for (int32_t i = threadIdx.x; i < len; i += kThreads) {
            const uint32_t t = uint32_t(__ldg(h + i)) - uint32_t(v0);
            if (t < n) {
                if (i >= prompt) atomicAdd(count + t, 1u);
                atomicOr(count + t, kSeen);
            }
        }
    }
    if (a.bias_offsets) {
        const int32_t lo = __ldg(a.bias_offsets + b), hi = __ldg(a.bias_offsets + b + 1);
        for (int32_t i = lo + int32_t(threadIdx.x); i < hi; i += kThreads) {
            const int32_t t = __ldg(a.bias_tokens + i);
            if (uint32_t(t) - uint32_t(v0) >= n) continue;
            bool first = true;  // the first of a token's entries adds up all of them, in list order
            for (int32_t j = lo; j < i && first; j++) first = __ldg(a.bias_tokens + j) != t;
            if (!first) continue;
            float sum = __ldg(a.bias_values + i);
            for (int32_t j = i + 1; j < hi; j++)
                if (__ldg(a.bias_tokens + j) == t) sum = __fadd_rn(sum, __ldg(a.bias_values + j));
            bias[t - v0] = sum;
        }
    }
    __syncthreads();
    const float r = a.repetition ? __ldg(a.repetition + b) : 1.0f;
    const float p = a.presence ? __ldg(a.presence + b) : 0.0f;
    const float f = a.frequency ? __ldg(a.frequency + b) : 0.0f;
    const GrammarRow row = grammar_row(a.g, b);
    T *logits = static_cast<T *>(a.logits) + b * a.stride + v0;
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
        if (!row.allows(v0 + int32_t(i))) {
            logits[i] = from_f32<T>(-INFINITY);
            continue;
        }
        const uint32_t c = count[i];
        const float add = bias[i];
        if (c || add != 0.0f) {
            float x = penalized(to_f32(logits[i]), c, r, p, f);
            if (add != 0.0f) x = __fadd_rn(x, add);
            logits[i] = from_f32<T>(x);
        }
    }
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
        else if (max_length < 0 || max_length > (1 << 30)) bad = "max_length must be in [0, 2^30]";
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
    const dim3 grid((unsigned(V) + kWindow - 1) / kWindow, unsigned(B));
    const cudaError_t e = dtype == TRIE_DTYPE_F32 ? launch_pdl_grid(k_penalize<float>, grid, kThreads, 0, stream, a)
                                                  : launch_pdl_grid(k_penalize<__nv_bfloat16>, grid, kThreads, 0, stream, a);
    if (e != cudaSuccess) return fail_launch(e, "penalize launch");
    return TRIE_OK;
}
