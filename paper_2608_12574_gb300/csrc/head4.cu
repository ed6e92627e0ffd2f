// The logits head in microscaled 4-bit floating point, under a grammar:
// trie_head4_logits.
//
//   logit[m, v] = S[m] T[v] sum_b s[m, b] t[v, b] sum_{k in block b} q[m, k] w[v, k]
// and -inf where row m's state does not allow token v: q and w in e2m1, s and t
// in e4m3 for 16 columns of a row, S and T in 32 bits for a row (quantize.cuh).
// Sums are kept in 32 bits and rounded once to the logits' type.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <cuda_runtime.h>

#include "blackwell.cuh"
#include "quantize.cuh"

namespace tmk {

namespace {

constexpr int kThreads4 = 256;

struct Head4Args {
    const uint8_t *q, *s, *w, *ws;
    const float *q_rows, *w_rows;
    int32_t M, V, D;
    void *logits;
    int64_t stride;
    Grammar g;
};

__device__ __forceinline__ float2 from_e2m1x2(uint8_t x) {
    return __half22float2(__half2(__nv_cvt_fp4x2_to_halfraw2(__nv_fp4x2_storage_t(x), __NV_E2M1)));
}

// A thread a logit.
template <typename T>
__global__ void __launch_bounds__(kThreads4) k_head4(const Head4Args a) {
    pdl_launch_dependents();
    pdl_wait();
    const int32_t v = int32_t(blockIdx.x) * kThreads4 + int32_t(threadIdx.x), m = blockIdx.y;
    if (v >= a.V) return;
    const int64_t bytes = row_bytes4(a.D), tiles = scale_tiles4(a.D);
    float sum = -INFINITY;
    if (grammar_row(a.g, m).allows(v)) {
        sum = 0.0f;
        for (int32_t k = 0; k < a.D; k += kGroup4) {
            const uint8_t *q = a.q + m * bytes + k / 2, *w = a.w + v * bytes + k / 2;
            float part = 0.0f;
            for (int i = 0; i < kGroup4 / 2; i++) {
                const float2 x = from_e2m1x2(__ldg(q + i)), y = from_e2m1x2(__ldg(w + i));
                part = fmaf(x.x, y.x, part);
                part = fmaf(x.y, y.y, part);
            }
            const int j = k % 64 / kGroup4;
            sum = fmaf(part, from_e4m3(__ldg(a.s + scale_word4(m, k / 64, tiles) + j)) *
                                 from_e4m3(__ldg(a.ws + scale_word4(v, k / 64, tiles) + j)), sum);
        }
        sum *= __ldg(a.q_rows + m) * __ldg(a.w_rows + v);
    }
    static_cast<T *>(a.logits)[m * a.stride + v] = from_f32<T>(sum);
}

}  // namespace

}  // namespace tmk

extern "C" int trie_head4_logits(const uint8_t *d_q, const uint8_t *d_scales, const float *d_row_scales, const uint8_t *d_w,
                                 const uint8_t *d_w_scales, const float *d_w_row_scales, int32_t M, int32_t V, int32_t D,
                                 void *d_logits, int dtype, int64_t stride, const uint32_t *d_mask, int32_t mask_rows,
                                 const int32_t *d_states, void *d_workspace, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_logits(d_logits, dtype, stride, M, V);
    if (!*bad) bad = check_grammar(d_mask, mask_rows, d_states);
    if (!*bad && (D < 1 || D > (1 << 24))) bad = "D must be in [1, 2^24]";
    if (!*bad && M > 0 && (!d_q || !d_scales || !d_row_scales || !d_w || !d_w_scales || !d_w_row_scales)) bad = "NULL pointer";
    if (!*bad && off_boundary(16, d_q, d_scales, d_w, d_w_scales)) bad = "d_q, d_w and their scales must be aligned to 16 bytes";
    if (!*bad && off_boundary(4, d_row_scales, d_w_row_scales)) bad = "the row scales are not aligned to 4 bytes";
    if (!*bad && M > 65535) bad = "M must be <= 65535";
    if (!*bad && M > 0 && d_mask && !d_workspace) bad = "d_mask without d_workspace";
    if (!*bad && off_boundary(16, static_cast<const char *>(d_workspace))) bad = "d_workspace is not aligned to 16 bytes";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (M == 0) return TRIE_OK;
    Head4Args a = {d_q, d_scales, d_w, d_w_scales, d_row_scales, d_w_row_scales, M, V, D, d_logits, stride,
                   make_grammar(d_mask, mask_rows, d_states, V)};
    const dim3 grid(unsigned((int64_t(V) + kThreads4 - 1) / kThreads4), unsigned(M));
    const cudaError_t e = dtype == TRIE_DTYPE_F32 ? launch_pdl_grid(k_head4<float>, grid, kThreads4, 0, stream, a)
                                                  : launch_pdl_grid(k_head4<__nv_bfloat16>, grid, kThreads4, 0, stream, a);
    if (e != cudaSuccess) return fail_launch(e, "4-bit head launch");
    return TRIE_OK;
}
