// What the calls on logits (penalize.cu, sample.cu, head.cu) share: the grammar
// of a batch and the element types.
#pragma once

#include <stdint.h>
#include <stdio.h>

#include <atomic>

#include <cuda_bf16.h>

#include "tm_internal.h"
#include "triemask.h"

namespace tmk {

// The grammar of a batch: a mask of `rows` rows of W words and a state for each
// row of the batch. A state in [0, rows) allows what its row of the mask holds,
// TRIE_STATE_FREE (or no mask) every token, any other only the last token.
struct Grammar {
    const uint32_t *mask;
    const int32_t *states;
    int32_t rows;
    int32_t V;
    int64_t W;
};

enum : int { kAllowAll = 0, kAllowRow = 1, kAllowEos = 2 };

struct GrammarRow {
    const uint32_t *words;
    int32_t V;
    int kind;
    // Bits of tokens 32 w .. 32 w + 31, w < W. Bits at or past V may be set.
    __device__ __forceinline__ uint32_t word(int32_t w) const {
        if (kind == kAllowAll) return ~0u;
        if (kind == kAllowRow) return __ldg(words + w);
        return w == (V - 1) >> 5 ? 1u << ((V - 1) & 31) : 0u;
    }
    __device__ __forceinline__ bool allows(int32_t v) const { return (word(v >> 5) >> (v & 31)) & 1u; }
};

// What a row in state s allows.
__device__ __forceinline__ GrammarRow grammar_state(const Grammar &g, int32_t s) {
    GrammarRow r;
    r.V = g.V;
    r.words = nullptr;
    r.kind = s == TRIE_STATE_FREE ? kAllowAll : kAllowEos;
    if (s >= 0 && s < g.rows) {
        r.words = g.mask + int64_t(s) * g.W;
        r.kind = kAllowRow;
    }
    return r;
}
__device__ __forceinline__ GrammarRow grammar_row(const Grammar &g, int32_t b) {
    return grammar_state(g, g.mask ? __ldg(g.states + b) : TRIE_STATE_FREE);
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

constexpr int32_t kMaxV = 0x7FFFFFFF - 1023;  // so that a tile past the end still has 32-bit ids

// Host side: the checks that every call on logits makes. "" when all hold.
inline const char *check_logits(const void *d_logits, int dtype, int64_t stride, int32_t B, int32_t V) {
    if (dtype != TRIE_DTYPE_F32 && dtype != TRIE_DTYPE_BF16) return "unknown dtype";
    if (B < 0) return "B must be >= 0";
    if (V < 2 || V > kMaxV) return "V must be in [2, 2^31 - 1024]";
    if (stride < V) return "the row stride must be >= V";
    if (B > 0 && !d_logits) return "d_logits is NULL";
    if (reinterpret_cast<uintptr_t>(d_logits) & uintptr_t(dtype == TRIE_DTYPE_F32 ? 3 : 1))
        return "d_logits is not aligned to its element size";
    return "";
}
// Whether an address (or several, or-ed) is off a boundary of `size` bytes; NULL is on any.
template <typename... P>
inline bool off_boundary(size_t size, const P *...p) {
    return ((reinterpret_cast<uintptr_t>(p) | ...) & (size - 1)) != 0;
}
inline const char *check_grammar(const uint32_t *d_mask, int32_t mask_rows, const int32_t *d_states) {
    if (!d_mask) return d_states ? "d_states without d_mask" : "";
    if (!d_states) return "d_mask without d_states";
    if (mask_rows < 0) return "mask_rows must be >= 0";
    if (off_boundary(4, d_mask, d_states)) return "d_mask / d_states are not aligned to 4 bytes";
    return "";
}
inline Grammar make_grammar(const uint32_t *d_mask, int32_t mask_rows, const int32_t *d_states, int32_t V) {
    Grammar g;
    g.mask = d_mask;
    g.states = d_states;
    g.rows = mask_rows;
    g.V = V;
    g.W = (int64_t(V) + 31) / 32;
    return g;
}
// SMs of the current device (152 on a GB300).
inline int sm_count() {
    static std::atomic<int> known[16];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 16) return 152;
    if ((n = known[dev].load(std::memory_order_relaxed))) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 152;
    known[dev].store(n, std::memory_order_relaxed);
    return n;
}
// Lets a kernel have up to kBytes of dynamic shared memory on the current device. Asked
// once for each: the call takes 2 us of the host's time. (Always for the same bytes, so that it does
// not matter which of two threads comes last.)
template <auto kKernel, int kBytes>
inline cudaError_t allow_smem() {
    static std::atomic<bool> allowed[16];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    const bool known = e == cudaSuccess && dev >= 0 && dev < 16;
    if (e == cudaSuccess && !(known && allowed[dev].load(std::memory_order_relaxed))) {
        e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        if (e == cudaSuccess && known) allowed[dev].store(true, std::memory_order_relaxed);
    }
    return e;
}
// Records a failed CUDA call as the thread's last error.
inline int fail_launch(cudaError_t e, const char *what) {
    cudaGetLastError();
    static thread_local char msg[256];
    snprintf(msg, sizeof msg, "%s: %s", what, cudaGetErrorString(e));
    return set_error(TRIE_ECUDA, msg);
}

}  // namespace tmk
