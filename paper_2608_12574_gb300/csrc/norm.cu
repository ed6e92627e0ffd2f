// Rows for the logits heads: trie_head_norm_quantize, trie_head4_norm_quantize,
// trie_head4_quantize.
//
//   h = round(x + residual), written back;  r = round(1 / sqrt(mean(h^2) + eps))
//   y = round(round(h r) gain)
// and y in e4m3 with scales of 128 columns as trie_head_quantize makes it, or in
// e2m1 with scales of 16 columns and of the row (quantize.cuh). h is in the
// residual's type, r and y in 32 bits.
//
// The sum of squares is kept as a pair of floats (the rounding of each square
// and of each addition is added up beside the sum) and r comes from one Newton
// step on such pairs: their error, some 2^-46, moves r's last bit in one row of
// a million, so that the 8- and 4-bit values, which lie next to rounding borders
// by chance, do not depend on the order of the sum.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <cuda_runtime.h>

#include "quantize.cuh"

namespace tmk {

namespace {

constexpr int kNormThreads = 256;
constexpr int kEach = 8;  // columns of a thread at a time

struct NormArgs {
    const void *x;         // [M] rows
    int64_t stride;
    int32_t M, D;
    void *residual;        // [M] rows or NULL
    int64_t residual_stride;
    const void *gain;      // [D]
    bool residual_f32, gain_f32;
    bool wide_x, wide_residual, wide_gain, wide_q;  // 16-byte (q: 8-byte) accesses of eight columns
    double eps;
    uint8_t *q;
    float *scales;         // 8 bits: [ceil(D/128)][pitch]
    int64_t pitch;
    uint8_t *scales4;      // 4 bits: of 16 columns
    float *row_scales;
};

// Eight columns from column c of a row of D; zeros behind the end.
template <typename T>
__device__ __forceinline__ void load8(const T *row, int32_t c, int32_t D, bool wide, float (&v)[kEach]) {
    if (wide && c + kEach <= D) {
        union {
            uint4 raw[kEach * sizeof(T) / 16];
            T x[kEach];
        } u;
#pragma unroll
        for (int i = 0; i < int(kEach * sizeof(T) / 16); i++) u.raw[i] = reinterpret_cast<const uint4 *>(row + c)[i];
#pragma unroll
        for (int i = 0; i < kEach; i++) v[i] = to_f32(u.x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; i++) v[i] = c + i < D ? to_f32(row[c + i]) : 0.0f;
    }
}
// Rounds v to the row's type, in it and in v.
template <typename T>
__device__ __forceinline__ void store8(T *row, int32_t c, int32_t D, bool wide, float (&v)[kEach]) {
    union {
        uint4 raw[kEach * sizeof(T) / 16];
        T x[kEach];
    } u;
#pragma unroll
    for (int i = 0; i < kEach; i++) {
        u.x[i] = from_f32<T>(v[i]);
        v[i] = to_f32(u.x[i]);
    }
    if (wide && c + kEach <= D) {
#pragma unroll
        for (int i = 0; i < int(kEach * sizeof(T) / 16); i++) reinterpret_cast<uint4 *>(row + c)[i] = u.raw[i];
    } else {
#pragma unroll
        for (int i = 0; i < kEach; i++)
            if (c + i < D) row[c + i] = u.x[i];
    }
}

// A sum and what its roundings have left out.
struct Pair {
    float sum, rest;
    __device__ __forceinline__ void add(float x) {
        const float s = sum + x, b = s - sum;
        rest += (sum - (s - b)) + (x - b);
        sum = s;
    }
    __device__ __forceinline__ void add_square(float x) {
        const float p = __fmul_rn(x, x);
        rest += __fmaf_rn(x, x, -p);
        add(p);
    }
};

// 1 / sqrt(mean + eps) of n values, rounded once. In doubles where the squares
// leave the range that pairs of floats are exact in (the same way in all threads).
__device__ __forceinline__ bool root_of(const Pair &p, float n, double eps, float *r) {
    const float mean = __fdiv_rn(p.sum, n);
    Pair m = {mean, __fdiv_rn(__fmaf_rn(-mean, n, p.sum) + p.rest, n)};
    const float e = float(eps);
    m.add(e);
    m.rest += float(eps - double(e));
    if (!(m.sum > 8.0779357e-28f && m.sum < 1.3292280e36f)) return false;  // 2^-90, 2^120
    const float r0 = rsqrtf(m.sum), s = __fmul_rn(r0, r0), s_rest = __fmaf_rn(r0, r0, -s);
    const float left = __fmaf_rn(-m.sum, s, 1.0f) - (m.sum * s_rest + m.rest * s);  // 1 - m r0^2
    *r = __fmaf_rn(0.5f * r0, left, r0);
    return true;
}

template <typename TX, bool kNorm, int kBits>
__global__ void __launch_bounds__(kNormThreads) k_norm_quantize(const NormArgs a) {
    __shared__ Pair pairs[kNormThreads / 32];
    __shared__ double doubles[kNormThreads / 32];
    __shared__ uint32_t maxima[kNormThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t m = blockIdx.x, D = a.D;
    const TX *x = static_cast<const TX *>(a.x) + m * a.stride;
    float *residual_f32 = static_cast<float *>(a.residual) + m * a.residual_stride;
    __nv_bfloat16 *residual_bf16 = static_cast<__nv_bfloat16 *>(a.residual) + m * a.residual_stride;
    const int32_t end = kBits == 8 ? (D + 127) / 128 * 128 : (D + 63) / 64 * 64;
    float r = 0.0f;

    // h of eight columns, the first time and again
    auto first = [&](int32_t c, float (&h)[kEach]) {
        load8(x, c, D, a.wide_x, h);
        if (!kNorm || !a.residual) return;
        float v[kEach];
        if (a.residual_f32) load8(residual_f32, c, D, a.wide_residual, v);
        else load8(residual_bf16, c, D, a.wide_residual, v);
#pragma unroll
        for (int i = 0; i < kEach; i++) h[i] = __fadd_rn(h[i], v[i]);
        if (a.residual_f32) store8(residual_f32, c, D, a.wide_residual, h);
        else store8(residual_bf16, c, D, a.wide_residual, h);
    };
    auto again = [&](int32_t c, float (&h)[kEach]) {
        if (!kNorm || !a.residual) load8(x, c, D, a.wide_x, h);
        else if (a.residual_f32) load8(residual_f32, c, D, a.wide_residual, h);
        else load8(residual_bf16, c, D, a.wide_residual, h);
    };
    auto norm = [&](int32_t c, float (&h)[kEach]) {
        if (!kNorm) return;
        float g[kEach];
        if (a.gain_f32) load8(static_cast<const float *>(a.gain), c, D, a.wide_gain, g);
        else load8(static_cast<const __nv_bfloat16 *>(a.gain), c, D, a.wide_gain, g);
#pragma unroll
        for (int i = 0; i < kEach; i++) h[i] = c + i < D ? __fmul_rn(__fmul_rn(h[i], r), g[i]) : 0.0f;
    };

    if (kNorm) {
        Pair p = {0.0f, 0.0f};
        for (int32_t c = int32_t(threadIdx.x) * kEach; c < D; c += kNormThreads * kEach) {
            float h[kEach];
            first(c, h);
#pragma unroll
            for (int i = 0; i < kEach; i++) p.add_square(h[i]);
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const float s = __shfl_xor_sync(~0u, p.sum, d), rest = __shfl_xor_sync(~0u, p.rest, d);
            p.add(s);
            p.rest += rest;
        }
        if (lane == 0) pairs[warp] = p;
        __syncthreads();
        Pair all = pairs[0];
        for (int i = 1; i < kNormThreads / 32; i++) {
            all.add(pairs[i].sum);
            all.rest += pairs[i].rest;
        }
        if (!root_of(all, float(D), a.eps, &r)) {
            double s = 0.0;
            for (int32_t c = int32_t(threadIdx.x) * kEach; c < D; c += kNormThreads * kEach) {
                float h[kEach];
                again(c, h);
                for (int i = 0; i < kEach; i++) s += double(h[i]) * h[i];
            }
            for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
            if (lane == 0) doubles[warp] = s;
            __syncthreads();
            s = doubles[0];
            for (int i = 1; i < kNormThreads / 32; i++) s += doubles[i];
            r = float(1.0 / sqrt(s / D + a.eps));
        }
    }

    if (kBits == 8) {
        for (int32_t c = int32_t(threadIdx.x) * kEach; c - lane * kEach < end; c += kNormThreads * kEach) {
            float y[kEach], amax = 0.0f;
            again(c, y);
            norm(c, y);
#pragma unroll
            for (int i = 0; i < kEach; i++) amax = fmaxf(amax, fabsf(y[i]));
#pragma unroll
            for (int d = 8; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, d));
            const float s = scale_of(amax);
            uint32_t out[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < kEach; i++) out[i / 4] |= uint32_t(to_e4m3(__fdiv_rn(y[i], s))) << (i % 4 * 8);
            uint8_t *q = a.q + int64_t(m) * D + c;
            if (a.wide_q && c + kEach <= D) {
                *reinterpret_cast<uint2 *>(q) = make_uint2(out[0], out[1]);
            } else {
#pragma unroll
                for (int i = 0; i < kEach; i++)
                    if (c + i < D) q[i] = uint8_t(out[i / 4] >> (i % 4 * 8));
            }
            if ((lane & 15) == 0 && c < end) a.scales[int64_t(c / kBlock) * a.pitch + m] = s;
        }
    } else {
        uint32_t most = 0;  // of the magnitudes' bits: NaN above infinity above numbers
        for (int32_t c = int32_t(threadIdx.x) * kEach; c < D; c += kNormThreads * kEach) {
            float y[kEach];
            again(c, y);
            norm(c, y);
#pragma unroll
            for (int i = 0; i < kEach; i++) most = max(most, __float_as_uint(y[i]) & 0x7FFFFFFFu);
        }
        most = __reduce_max_sync(~0u, most);
        if (lane == 0) maxima[warp] = most;
        __syncthreads();
        for (int i = 0; i < kNormThreads / 32; i++) most = max(most, maxima[i]);
        const float row_scale = row_scale4(most);
        if (threadIdx.x == 0) a.row_scales[m] = row_scale;
        const int64_t tiles = scale_tiles4(D);
        for (int32_t c = int32_t(threadIdx.x) * kEach; c - lane * kEach < end; c += kNormThreads * kEach) {
            float y[kEach], amax = 0.0f;
            again(c, y);
            norm(c, y);
#pragma unroll
            for (int i = 0; i < kEach; i++) amax = fmaxf(amax, fabsf(y[i]));
            amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
            const uint8_t s = block_scale4(amax, row_scale);
            const float per = per_step4(s, row_scale);
            uint32_t out = 0;
#pragma unroll
            for (int i = 0; i < kEach; i += 2)
                out |= uint32_t(to_e2m1x2(__fmul_rn(y[i], per), __fmul_rn(y[i + 1], per))) << (4 * i);
            if (c < row_bytes4(D) * 2) *reinterpret_cast<uint32_t *>(a.q + m * row_bytes4(D) + c / 2) = out;
            uint32_t word = uint32_t(s) << (8 * ((lane >> 1) & 3));
            word |= __shfl_xor_sync(~0u, word, 2);
            word |= __shfl_xor_sync(~0u, word, 4);
            if ((lane & 7) == 0 && c < end) *reinterpret_cast<uint32_t *>(a.scales4 + scale_word4(m, c / 64, tiles)) = word;
        }
    }
}

template <bool kNorm, int kBits>
int launch_norm(const NormArgs &a, int dtype, cudaStream_t st) {
    const cudaError_t e = dtype == TRIE_DTYPE_F32
        ? launch_pdl(k_norm_quantize<float, kNorm, kBits>, a.M, kNormThreads, st, a)
        : launch_pdl(k_norm_quantize<__nv_bfloat16, kNorm, kBits>, a.M, kNormThreads, st, a);
    return e == cudaSuccess ? TRIE_OK : fail_launch(e, "norm quantize launch");
}

bool is_dtype(int dtype) { return dtype == TRIE_DTYPE_F32 || dtype == TRIE_DTYPE_BF16; }
size_t size_of(int dtype) { return dtype == TRIE_DTYPE_F32 ? 4 : 2; }
// Whether rows of a type can be read 16 bytes at a time.
bool wide_rows(const void *p, int dtype, int64_t stride, int32_t rows) {
    return !off_boundary(16, static_cast<const char *>(p)) && (rows < 2 || stride * int64_t(size_of(dtype)) % 16 == 0);
}

const char *check_rows(const void *x, int dtype, int64_t stride, int32_t rows, int32_t D, const void *q, const void *scales) {
    if (!is_dtype(dtype)) return "unknown dtype";
    if (rows < 0) return "the number of rows must be >= 0";
    if (D < 1 || D > (1 << 24)) return "D must be in [1, 2^24]";
    if (stride < D) return "the row stride must be >= D";
    if (rows > 0 && (!x || !q || !scales)) return "NULL pointer";
    if (off_boundary(size_of(dtype), static_cast<const char *>(x))) return "the input is not aligned to its element size";
    return "";
}
const char *check_norm(const void *residual, int residual_dtype, int64_t residual_stride, const void *gain, int gain_dtype,
                       double eps, int32_t rows, int32_t D) {
    if (!is_dtype(gain_dtype) || (residual && !is_dtype(residual_dtype))) return "unknown dtype of the residual or the gain";
    if (residual && residual_stride < D) return "the residual's row stride must be >= D";
    if (rows > 0 && !gain) return "NULL pointer";
    if (off_boundary(size_of(gain_dtype), static_cast<const char *>(gain)) ||
        (residual && off_boundary(size_of(residual_dtype), static_cast<const char *>(residual))))
        return "the residual or the gain is not aligned to its element size";
    if (!(eps >= 1e-30 && eps <= 1e30)) return "eps must be in [1e-30, 1e30]";
    return "";
}
const char *check_out4(const uint8_t *q, const uint8_t *scales, const float *row_scales, int32_t rows) {
    if (off_boundary(16, q, scales)) return "d_q and d_scales must be aligned to 16 bytes";
    if (off_boundary(4, row_scales)) return "d_row_scales is not aligned to 4 bytes";
    if (rows > 0 && !row_scales) return "NULL pointer";
    return "";
}
NormArgs make_norm(const void *x, int dtype, int64_t stride, int32_t M, int32_t D, void *residual, int residual_dtype,
                   int64_t residual_stride, const void *gain, int gain_dtype, double eps) {
    NormArgs a = {};
    a.x = x;
    a.stride = stride;
    a.M = M;
    a.D = D;
    a.residual = residual;
    a.residual_stride = residual_stride;
    a.gain = gain;
    a.residual_f32 = residual_dtype == TRIE_DTYPE_F32;
    a.gain_f32 = gain_dtype == TRIE_DTYPE_F32;
    a.wide_x = wide_rows(x, dtype, stride, M);
    a.wide_residual = residual && wide_rows(residual, residual_dtype, residual_stride, M);
    a.wide_gain = gain && wide_rows(gain, gain_dtype, 0, 1);
    a.eps = eps;
    return a;
}

}  // namespace

}  // namespace tmk

extern "C" int trie_head_norm_quantize(const void *d_x, int dtype, int64_t stride, void *d_residual, int residual_dtype,
                                       int64_t residual_stride, const void *d_gain, int gain_dtype, double eps, int32_t M,
                                       int32_t D, uint8_t *d_q, float *d_scales, int64_t pitch, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_rows(d_x, dtype, stride, M, D, d_q, d_scales);
    if (!*bad) bad = check_norm(d_residual, residual_dtype, residual_stride, d_gain, gain_dtype, eps, M, D);
    if (!*bad && off_boundary(4, d_scales)) bad = "the scales are not aligned to 4 bytes";
    if (!*bad && pitch < M) bad = "pitch must be >= M";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (M == 0) return TRIE_OK;
    NormArgs a = make_norm(d_x, dtype, stride, M, D, d_residual, residual_dtype, residual_stride, d_gain, gain_dtype, eps);
    a.q = d_q;
    a.wide_q = !off_boundary(8, d_q) && D % 8 == 0;
    a.scales = d_scales;
    a.pitch = pitch;
    return launch_norm<true, 8>(a, dtype, stream);
}

extern "C" int64_t trie_head4_row_bytes(int32_t D) { return D < 1 || D > (1 << 24) ? -1 : tmk::row_bytes4(D); }

extern "C" int64_t trie_head4_scale_bytes(int32_t rows, int32_t D) {
    if (rows < 0 || D < 1 || D > (1 << 24)) return -1;
    return (int64_t(rows) + 127) / 128 * tmk::scale_tiles4(D) * 512;
}

extern "C" int trie_head4_quantize(const void *d_x, int dtype, int64_t stride, int32_t rows, int32_t D, uint8_t *d_q,
                                   uint8_t *d_scales, float *d_row_scales, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_rows(d_x, dtype, stride, rows, D, d_q, d_scales);
    if (!*bad) bad = check_out4(d_q, d_scales, d_row_scales, rows);
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (rows == 0) return TRIE_OK;
    NormArgs a = make_norm(d_x, dtype, stride, rows, D, nullptr, 0, 0, nullptr, 0, 1.0);
    a.q = d_q;
    a.scales4 = d_scales;
    a.row_scales = d_row_scales;
    return launch_norm<false, 4>(a, dtype, stream);
}

extern "C" int trie_head4_norm_quantize(const void *d_x, int dtype, int64_t stride, void *d_residual, int residual_dtype,
                                        int64_t residual_stride, const void *d_gain, int gain_dtype, double eps, int32_t M,
                                        int32_t D, uint8_t *d_q, uint8_t *d_scales, float *d_row_scales, cudaStream_t stream) {
    using namespace tmk;
    const char *bad = check_rows(d_x, dtype, stride, M, D, d_q, d_scales);
    if (!*bad) bad = check_norm(d_residual, residual_dtype, residual_stride, d_gain, gain_dtype, eps, M, D);
    if (!*bad) bad = check_out4(d_q, d_scales, d_row_scales, M);
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (M == 0) return TRIE_OK;
    NormArgs a = make_norm(d_x, dtype, stride, M, D, d_residual, residual_dtype, residual_stride, d_gain, gain_dtype, eps);
    a.q = d_q;
    a.scales4 = d_scales;
    a.row_scales = d_row_scales;
    return launch_norm<true, 4>(a, dtype, stream);
}
