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

#include <cuda_runtime.h>

#include "logits.cuh"

namespace tmk {

namespace {

constexpr int kPolicyThreads = 512;

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
    __device__ __forceinline__ void add(float x, float c) {
        if (x > top) {
            sum = sum * exp2_of((top - x) * c) + 1.0f;
            top = x;
        } else if (x != -INFINITY) {
            sum += exp2_of((x - top) * c);
        }
    }
};

template <typename T>
__global__ void __launch_bounds__(kPolicyThreads) k_policy(const PolicyArgs a) {
    __shared__ Mass parts[kPolicyThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t b = blockIdx.x, V = a.V;
    const T *x = static_cast<const T *>(a.logits) + b * a.stride;
    const GrammarRow row = grammar_row(a.g, b);
    const float given = a.temperature ? __ldg(a.temperature + b) : 1.0f;
    const float temperature = given > 0.0f ? fminf(fmaxf(given, 1.17549435e-38f), 3.40282347e38f) : 1.0f;
    const float c = 1.44269504f / temperature;
    Mass all = {-INFINITY, 0.0f};
    for (int32_t v = threadIdx.x; v < V; v += kPolicyThreads)
        if (row.allows(v)) all.add(to_f32(x[v]), c);
    for (int d = 16; d; d >>= 1)
        all.join(__shfl_xor_sync(~0u, all.top, d), __shfl_xor_sync(~0u, all.sum, d), c);
    if (lane == 0) parts[warp] = all;
    const int32_t t = __ldg(a.tokens + b);
    const float xt = t >= 0 && t < V && row.allows(t) ? to_f32(x[t]) : -INFINITY;
    __syncthreads();
    all = parts[0];
    for (int i = 1; i < kPolicyThreads / 32; i++) all.join(parts[i].top, parts[i].sum, c);
    float lp = (xt - all.top) / temperature - logf(all.sum);
    if (all.top == INFINITY) lp = __int_as_float(0x7FC00000);
    if (xt == -INFINITY) lp = -INFINITY;
    const float weight = a.weights ? __ldg(a.weights + b) : 1.0f;
    float loss = 0.0f, slope = 0.0f;
    if (lp != -INFINITY && weight != 0.0f) {
        const float A = __ldg(a.advantages + b), rho = expf(lp - __ldg(a.old + b));
        const float free = rho * A, held = fminf(fmaxf(rho, a.low), a.high) * A;
        loss = -(free > held ? held : free);  // a NaN stays one
        slope = free > held ? 0.0f : -free;
        if (a.ref) {
            const float d = __ldg(a.ref + b) - lp, e = expm1f(d);
            loss += a.kl * (e - d);
            slope -= a.kl * e;
        }
        loss *= weight;
        slope *= weight;
    }
    if (threadIdx.x == 0) {
        a.losses[b] = loss;
        a.logprobs[b] = lp;
    }
    if (!a.grad) return;
    T *grad = static_cast<T *>(a.grad) + b * a.grad_stride;
    const float per = 1.0f / temperature, f = -slope / all.sum;
    for (int32_t v = threadIdx.x; v < V; v += kPolicyThreads) {
        float g = 0.0f;
        if (slope != 0.0f && row.allows(v)) {
            if (v == t) g = slope * -expm1f(lp) * per;
            else g = f * exp2_of((to_f32(x[v]) - all.top) * c) * per;
        }
        grad[v] = from_f32<T>(g);
    }
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
                    d_losses, d_logprobs, d_grad, grad_stride};
    const cudaError_t e = dtype == TRIE_DTYPE_F32 ? launch_pdl(k_policy<float>, B, kPolicyThreads, stream, a)
                                                  : launch_pdl(k_policy<__nv_bfloat16>, B, kPolicyThreads, stream, a);
    if (e != cudaSuccess) return fail_launch(e, "policy loss launch");
    return TRIE_OK;
}
