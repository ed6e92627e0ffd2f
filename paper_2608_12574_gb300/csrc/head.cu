// The logits head in 8-bit floating point (e4m3) with block scales, under a
// grammar: trie_head_quantize, trie_head_quantize_weight, trie_head_logits.
//
//   x[m, k] ~ q[m, k] s[k / 128, m],  W[v, k] ~ w[v, k] S[v / 128, k / 128]
//   logit[m, v] = sum_kb s[kb, m] S[v / 128, kb] sum_{k in block kb} q[m, k] w[v, k]
// and -inf where row m's state does not allow token v. Products of a block are
// summed, and blocks are scaled and added, in 32 bits; one rounding to bf16 at
// the end. A scale is the block's largest magnitude times 1/448, in 32 bits (1
// where that is 0): the largest value maps to the largest e4m3 number.
//
//  k_head_quantize         a warp per row and block of 128 columns.
//  k_head_quantize_weight  a CTA per block of 128 x 128.
//  k_head_logits           64 tokens x 64 rows a CTA.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include "logits.cuh"

namespace tmk {

namespace {

constexpr int kBlock = 128;  // columns (and weight rows) that share a scale
constexpr float kPerMax = 1.0f / 448.0f;  // 448: the largest e4m3 number
constexpr int kQuantThreads = 256;
constexpr int kTile = 64;

__device__ __forceinline__ uint8_t to_e4m3(float x) {
    return uint8_t(__nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3));
}
__device__ __forceinline__ float from_e4m3(uint8_t x) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(x, __NV_E4M3)));
}

// NaN does not show in the maximum, but a NaN element becomes a NaN in e4m3 and
// an infinite one makes the scale infinite and itself NaN: either way the row's
// logits are NaN.
__device__ __forceinline__ float scale_of(float amax) {
    const float s = __fmul_rn(amax, kPerMax);
    return s > 0.0f ? s : 1.0f;
}

template <typename T>
__global__ void __launch_bounds__(kQuantThreads) k_head_quantize(const T *x, int64_t stride, int32_t M, int32_t D,
                                                                 uint8_t *q, float *scales, int64_t pitch) {
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int32_t blocks = (D + kBlock - 1) / kBlock;
    const int64_t at = int64_t(blockIdx.x) * (kQuantThreads / 32) + (threadIdx.x >> 5);
    if (at >= int64_t(M) * blocks) return;
    const int32_t m = int32_t(at / blocks), kb = int32_t(at % blocks);
    float v[kBlock / 32], amax = 0.0f;
#pragma unroll
    for (int i = 0; i < kBlock / 32; i++) {
        const int32_t k = kb * kBlock + i * 32 + lane;
        v[i] = k < D ? to_f32(x[m * stride + k]) : 0.0f;
        amax = fmaxf(amax, fabsf(v[i]));
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, d));
    const float s = scale_of(amax);
#pragma unroll
    for (int i = 0; i < kBlock / 32; i++) {
        const int32_t k = kb * kBlock + i * 32 + lane;
        if (k < D) q[int64_t(m) * D + k] = to_e4m3(__fdiv_rn(v[i], s));
    }
    if (lane == 0) scales[kb * pitch + m] = s;
}

template <typename T>
__global__ void __launch_bounds__(kQuantThreads) k_head_quantize_weight(const T *w, int64_t stride, int32_t V, int32_t D,
                                                                        uint8_t *q, float *scales) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float part[kQuantThreads / 32];
    const int32_t blocks = (D + kBlock - 1) / kBlock;
    const int32_t vb = int32_t(blockIdx.x / blocks), kb = int32_t(blockIdx.x % blocks);
    const int32_t k = kb * kBlock + int32_t(threadIdx.x % kBlock);
    float amax = 0.0f;
    for (int r = threadIdx.x / kBlock; r < kBlock; r += kQuantThreads / kBlock) {
        const int64_t v = int64_t(vb) * kBlock + r;
        if (v < V && k < D) amax = fmaxf(amax, fabsf(to_f32(w[v * stride + k])));
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, d));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = amax;
    __syncthreads();
    for (int i = 0; i < kQuantThreads / 32; i++) amax = fmaxf(amax, part[i]);
    const float s = scale_of(amax);
    for (int r = threadIdx.x / kBlock; r < kBlock; r += kQuantThreads / kBlock) {
        const int64_t v = int64_t(vb) * kBlock + r;
        if (v < V && k < D) q[v * D + k] = to_e4m3(__fdiv_rn(to_f32(w[v * stride + k]), s));
    }
    if (threadIdx.x == 0) scales[int64_t(vb) * blocks + kb] = s;
}

struct HeadArgs {
    const uint8_t *q;      // [M, D]
    const float *s;        // [blocks][pitch]
    int64_t pitch;
    const uint8_t *w;      // [V, D]
    const float *ws;       // [ceil(V / 128)][blocks]
    int32_t M, V, D, blocks;
    void *logits;
    int64_t stride;
    Grammar g;
};

template <typename T>
__global__ void __launch_bounds__(256) k_head_logits(HeadArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ float ws[kTile][33], xs[kTile][33];
    const int32_t v0 = blockIdx.x * kTile, m0 = blockIdx.y * kTile;
    const int tv = threadIdx.x & 15, tm = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int32_t kb = 0; kb < a.blocks; kb++) {
        float part[4][4] = {};
        for (int32_t k0 = kb * kBlock; k0 < min(a.D, (kb + 1) * kBlock); k0 += 32) {
            __syncthreads();
            for (int i = threadIdx.x; i < kTile * 32; i += 256) {
                const int r = i >> 5;
                const int32_t k = k0 + (i & 31);
                ws[r][i & 31] = v0 + r < a.V && k < a.D ? from_e4m3(a.w[int64_t(v0 + r) * a.D + k]) : 0.0f;
                xs[r][i & 31] = m0 + r < a.M && k < a.D ? from_e4m3(a.q[int64_t(m0 + r) * a.D + k]) : 0.0f;
            }
            __syncthreads();
#pragma unroll 8
            for (int k = 0; k < 32; k++)
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) part[i][j] += xs[tm + 16 * i][k] * ws[tv + 16 * j][k];
        }
        const float sw = __ldg(a.ws + int64_t(v0 / kBlock) * a.blocks + kb);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int32_t m = m0 + tm + 16 * i;
            const float f = m < a.M ? __ldg(a.s + kb * a.pitch + m) * sw : 0.0f;
#pragma unroll
            for (int j = 0; j < 4; j++) acc[i][j] += part[i][j] * f;
        }
    }
    for (int i = 0; i < 4; i++) {
        const int32_t m = m0 + tm + 16 * i;
        if (m >= a.M) continue;
        const GrammarRow row = grammar_row(a.g, m);
        for (int j = 0; j < 4; j++) {
            const int32_t v = v0 + tv + 16 * j;
            if (v < a.V)
                static_cast<T *>(a.logits)[m * a.stride + v] = from_f32<T>(row.allows(v) ? acc[i][j] : -INFINITY);
        }
    }
}

const char *check_quantize(const void *x, int dtype, int64_t stride, int32_t rows, int32_t D, const void *q,
                           const float *scales) {
    if (dtype != TRIE_DTYPE_F32 && dtype != TRIE_DTYPE_BF16) return "unknown dtype";
    if (rows < 0) return "the number of rows must be >= 0";
    if (D < 1) return "D must be >= 1";
    if (stride < D) return "the row stride must be >= D";
    if (rows > 0 && (!x || !q || !scales)) return "NULL pointer";
    if (reinterpret_cast<uintptr_t>(x) & uintptr_t(dtype == TRIE_DTYPE_F32 ? 3 : 1)) return "the input is not aligned to its element size";
    if (reinterpret_cast<uintptr_t>(scales) & 3) return "the scales are not aligned to 4 bytes";
    return "";
}

}  // namespace

}  // namespace tmk

extern "C" int trie_head_quantize(const void *d_x, int dtype, int64_t stride, int32_t M, int32_t D, uint8_t *d_q,
                                  float *d_scales, int64_t pitch, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_quantize(d_x, dtype, stride, M, D, d_q, d_scales);
    if (!*bad && pitch < M) bad = "pitch must be >= M";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (M == 0) return TRIE_OK;
    const int64_t warps = int64_t(M) * ((D + kBlock - 1) / kBlock);
    const int64_t grid = (warps + kQuantThreads / 32 - 1) / (kQuantThreads / 32);
    const cudaError_t e = dtype == TRIE_DTYPE_F32
        ? launch_pdl(k_head_quantize<float>, grid, kQuantThreads, stream, static_cast<const float *>(d_x), stride, M, D,
                     d_q, d_scales, pitch)
        : launch_pdl(k_head_quantize<__nv_bfloat16>, grid, kQuantThreads, stream,
                     static_cast<const __nv_bfloat16 *>(d_x), stride, M, D, d_q, d_scales, pitch);
    if (e != cudaSuccess) return fail_launch(e, "head quantize launch");
    return TRIE_OK;
}

extern "C" int trie_head_quantize_weight(const void *d_w, int dtype, int64_t stride, int32_t V, int32_t D, uint8_t *d_q,
                                         float *d_scales, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_quantize(d_w, dtype, stride, V, D, d_q, d_scales);
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (V == 0) return TRIE_OK;
    const int64_t grid = ((int64_t(V) + kBlock - 1) / kBlock) * ((D + kBlock - 1) / kBlock);
    const cudaError_t e = dtype == TRIE_DTYPE_F32
        ? launch_pdl(k_head_quantize_weight<float>, grid, kQuantThreads, stream, static_cast<const float *>(d_w), stride,
                     V, D, d_q, d_scales)
        : launch_pdl(k_head_quantize_weight<__nv_bfloat16>, grid, kQuantThreads, stream,
                     static_cast<const __nv_bfloat16 *>(d_w), stride, V, D, d_q, d_scales);
    if (e != cudaSuccess) return fail_launch(e, "head weight quantize launch");
    return TRIE_OK;
}

extern "C" int trie_head_logits(const uint8_t *d_q, const float *d_scales, int64_t pitch, const uint8_t *d_w,
                                const float *d_w_scales, int32_t M, int32_t V, int32_t D, void *d_logits, int dtype,
                                int64_t stride, const uint32_t *d_mask, int32_t mask_rows, const int32_t *d_states,
                                cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_logits(d_logits, dtype, stride, M, V);
    if (!*bad) bad = check_grammar(d_mask, mask_rows, d_states);
    if (!*bad && (D < 16 || D % 16)) bad = "D must be a positive multiple of 16";
    if (!*bad && (pitch < M || pitch % 4)) bad = "pitch must be a multiple of 4 and >= M";
    if (!*bad && M > 0 && (!d_q || !d_scales || !d_w || !d_w_scales)) bad = "NULL pointer";
    if (!*bad && ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_w) |
                   reinterpret_cast<uintptr_t>(d_scales)) & 15))
        bad = "d_q, d_w and d_scales must be aligned to 16 bytes";
    if (!*bad && (reinterpret_cast<uintptr_t>(d_w_scales) & 3)) bad = "d_w_scales is not aligned to 4 bytes";
    if (!*bad && M > (1 << 20)) bad = "M must be <= 2^20";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (M == 0) return TRIE_OK;
    HeadArgs a;
    a.q = d_q;
    a.s = d_scales;
    a.pitch = pitch;
    a.w = d_w;
    a.ws = d_w_scales;
    a.M = M;
    a.V = V;
    a.D = D;
    a.blocks = (D + kBlock - 1) / kBlock;
    a.logits = d_logits;
    a.stride = stride;
    a.g = make_grammar(d_mask, mask_rows, d_states, V);
    const dim3 grid((unsigned(V) + kTile - 1) / kTile, (unsigned(M) + kTile - 1) / kTile);
    const cudaError_t e = dtype == TRIE_DTYPE_F32 ? launch_pdl_grid(k_head_logits<float>, grid, 256, 0, stream, a)
                                                  : launch_pdl_grid(k_head_logits<__nv_bfloat16>, grid, 256, 0, stream, a);
    if (e != cudaSuccess) return fail_launch(e, "head launch");
    return TRIE_OK;
}
