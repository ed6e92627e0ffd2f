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
//
//  k_norm_rows  aligned rows, few or in bf16: read once, held in registers.
//  k_norm_long  any others: read again in each pass.
//
// What bounds it (residual and x in bf16, 8 bits; times of calls that follow one another).
//   16,384 rows, D 5,120: 112 us, 5.3 TB/s. 32 instructions a value (11 of them in the
//     quantization, 9 in the sum of squares and its root), beside HBM: without any one part it is 101
//     to 107. With a loop that reads rows again 147, with each warp adding up all warps' sums 125,
//     with the next row's copies ahead but in registers, so that fewer CTAs fit, 174.
//     D 4,096: 84 us, 5.6 TB/s. x and the residual in f32, D 8,192: 12,010 rows read again 205 us, 6.3 TB/s.
//   256 rows, D 4,096, the residual in f32: 4.5 us; 1 row 2.6 us: launch and a chain of waits.
//   1,000 rows, D 4,112, all f32: 12.5 us, 4.3 TB/s: 1,000 CTAs at once, each a chain of three passes.
//   4,924 rows, D 7,363, all f32: 120 us; a value at a time, as rows of this D lie, 198.
//   Into 4 bits: 16,384 rows, D 5,120 121 us, 4.5 TB/s, 102 without residual (8 bits: 95); all f32 199 and 143 (8 bits: 109).
//   trie_head4_quantize of weights, V 152,064, D 4,096: 396 us, 4.0 TB/s; f32, read twice, 563.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <type_traits>

#include <cuda_runtime.h>

#include "blackwell.cuh"
#include "quantize.cuh"
#include "two.cuh"

namespace tmk {

namespace {

constexpr int kNormThreads = 256;  // where many rows are read again, at most
constexpr int kMaxThreads = 1024;  // of a row of one step a thread
constexpr int kHoldThreads = 512;  // of more
// A CTA stays where it has more rows than this: 16,384 rows, D 5,120 112 us, and 132 by a CTA a row; 4,000 rows 31 and 35.
constexpr int kStayRows = 1;
constexpr size_t kMostSpace = 220 * 1024;  // of an SM's shared memory
constexpr int kEach = 8;           // columns of a thread at a time

struct NormArgs {
    const void *x;         // [M] rows
    int64_t stride;
    int32_t M, D;
    void *residual;        // [M] rows or NULL
    int64_t residual_stride;
    const void *gain;      // [D]
    bool x_f32, residual_f32, gain_f32;
    bool wide, wide_q;     // rows can be read (q: written) eight columns at a time
    double eps;
    int32_t buffers;       // of k_norm_rows: 2 where a CTA takes several rows
    float eps_32, eps_rest, per_column, per_column_rest;  // eps and 1 / D as pairs
    uint8_t *q;
    float *scales;         // 8 bits: [ceil(D/128)][pitch]
    int64_t pitch;
    uint8_t *scales4;      // 4 bits: of 16 columns
    float *row_scales;
};

// Eight columns of a row as they were read: with kWide in w[0..3] (bf16) or w[0..7]
// (f32) as they lie in memory, else an element in each. Nothing is done with
// them until all of a thread's reads are on their way.
struct Raw {
    uint32_t w[kEach];
};
template <bool kWide>
__device__ __forceinline__ Raw load8(const void *row, bool f32, int32_t c, int32_t D) {
    Raw r;
    if (kWide) {  // D is a multiple of eight
        const uint4 *at = reinterpret_cast<const uint4 *>(static_cast<const char *>(row) + int64_t(c) * (f32 ? 4 : 2));
        uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
        if (c < D) lo = at[0];
        if (c < D && f32) hi = at[1];
        r.w[0] = lo.x, r.w[1] = lo.y, r.w[2] = lo.z, r.w[3] = lo.w, r.w[4] = hi.x, r.w[5] = hi.y, r.w[6] = hi.z, r.w[7] = hi.w;
    } else if (c >= kEach && c + 2 * kEach <= D) {  // the 16-byte pieces that they lie in are the row's, too
        const char *from = static_cast<const char *>(row) + int64_t(c) * (f32 ? 4 : 2);
        const uint32_t off = reinterpret_cast<uintptr_t>(from) & 15u;
        const uint4 *at = reinterpret_cast<const uint4 *>(from - off);
        const uint4 p0 = at[0], p1 = at[1], p2 = f32 ? at[2] : p1;
        uint32_t u[12] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w, p2.x, p2.y, p2.z, p2.w};
#pragma unroll
        for (int d = 1; d <= 2; d *= 2)
#pragma unroll
            for (int i = 0; i + d < 12; i++) u[i] = off & (4u * d) ? u[i + d] : u[i];
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            const uint32_t pair = off & 2u ? __funnelshift_r(u[i / 2], u[i / 2 + 1], 16) : u[i / 2];
            r.w[i] = f32 ? u[i] : i & 1 ? pair >> 16 : pair & 0xFFFFu;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            r.w[i] = 0u;
            if (f32 && c + i < D) r.w[i] = static_cast<const uint32_t *>(row)[c + i];
            if (!f32 && c + i < D) r.w[i] = static_cast<const uint16_t *>(row)[c + i];
        }
    }
    return r;
}
template <bool kWide>
__device__ __forceinline__ void values8(const Raw &r, bool f32, Two (&v)[kEach / 2]) {
#pragma unroll
    for (int i = 0; i < kEach / 2; i++) {
        uint32_t x = r.w[2 * i], y = r.w[2 * i + 1];
        if (!f32) {
            x = (kWide ? r.w[i] : x) << 16;
            y = kWide ? r.w[i] & 0xFFFF0000u : y << 16;
        }
        v[i] = two(__uint_as_float(x), __uint_as_float(y));
    }
}
// Rounds v to the row's type, in it and in v.
template <bool kWide>
__device__ __forceinline__ void store8(void *row, bool f32, int32_t c, int32_t D, Two (&v)[kEach / 2]) {
    Raw r;
#pragma unroll
    for (int i = 0; i < kEach / 2; i++) {
        const float2 f = apart(v[i]);
        r.w[2 * i] = __float_as_uint(f.x), r.w[2 * i + 1] = __float_as_uint(f.y);
        if (!f32) {
            const __nv_bfloat162 both = __floats2bfloat162_rn(f.x, f.y);
            const uint32_t w = *reinterpret_cast<const uint32_t *>(&both);
            v[i] = two(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
            if (kWide) r.w[i] = w;
            else r.w[2 * i] = w & 0xFFFFu, r.w[2 * i + 1] = w >> 16;
        }
    }
    if (kWide) {
        uint4 *at = reinterpret_cast<uint4 *>(static_cast<char *>(row) + int64_t(c) * (f32 ? 4 : 2));
        if (c < D) at[0] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
        if (c < D && f32) at[1] = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
    } else if (c + kEach <= D) {  // in pairs, from the second on where the first lies off a pair's boundary
        char *to = static_cast<char *>(row) + int64_t(c) * (f32 ? 4 : 2);
        const bool odd = reinterpret_cast<uintptr_t>(to) & (f32 ? 4u : 2u);
        if (f32) {
            if (odd) reinterpret_cast<uint32_t *>(to)[0] = r.w[0], reinterpret_cast<uint32_t *>(to)[7] = r.w[7];
#pragma unroll
            for (int i = 0; i < kEach; i += 2)
                if (!odd) *reinterpret_cast<uint2 *>(to + 4 * i) = make_uint2(r.w[i], r.w[i + 1]);
                else if (i < 6) *reinterpret_cast<uint2 *>(to + 4 * i + 4) = make_uint2(r.w[i + 1], r.w[i + 2]);
        } else {
            if (odd) reinterpret_cast<uint16_t *>(to)[0] = uint16_t(r.w[0]), reinterpret_cast<uint16_t *>(to)[7] = uint16_t(r.w[7]);
#pragma unroll
            for (int i = 0; i < kEach; i += 2)
                if (!odd) *reinterpret_cast<uint32_t *>(to + 2 * i) = r.w[i] | r.w[i + 1] << 16;
                else if (i < 6) *reinterpret_cast<uint32_t *>(to + 2 * i + 2) = r.w[i + 1] | r.w[i + 2] << 16;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; i++)
            if (c + i < D) {
                if (f32) static_cast<uint32_t *>(row)[c + i] = r.w[i];
                else static_cast<uint16_t *>(row)[c + i] = uint16_t(r.w[i]);
            }
    }
}

// A sum and what its roundings have left out (of additions: Knuth's two-sum).
struct Pair {
    float sum, rest;
    __device__ __forceinline__ void add(float x) {
        const float s = sum + x, b = s - sum;
        rest += (sum - (s - b)) + (x - b);
        sum = s;
    }
};

// 1 / sqrt(mean + eps) of the sum of D squares, rounded once: the mean by 1 / D, which
// is a pair too, and one Newton step. False where the squares leave the range that pairs of
// floats are exact in (the same way in all threads).
__device__ __forceinline__ bool root_of(const Pair &p, const NormArgs &a, float *r) {
    const float mean = __fmul_rn(p.sum, a.per_column);
    Pair m = {mean, __fmaf_rn(p.sum, a.per_column, -mean) + (p.sum * a.per_column_rest + p.rest * a.per_column)};
    m.add(a.eps_32);
    m.rest += a.eps_rest;
    if (!(m.sum > 0x1p-90f && m.sum < 0x1p120f)) return false;
    const float r0 = rsqrtf(m.sum), s = __fmul_rn(r0, r0), s_rest = __fmaf_rn(r0, r0, -s);
    const float left = __fmaf_rn(-m.sum, s, 1.0f) - (m.sum * s_rest + m.rest * s);  // 1 - m r0^2
    *r = __fmaf_rn(0.5f * r0, left, r0);
    return true;
}

// The sum of squares of a thread's numbers, two at a time: Pair::add of two
// squares, and what their own rounding left out, which of bf16 numbers (kShort) is
// nothing. Differences are multiply-adds with -1: one instruction for two numbers, a
// subtraction is three.
template <bool kShort>
struct Squares {
    Two sum = 0, rest = 0;
    __device__ __forceinline__ void add(const Two (&h)[kEach / 2]) {
        const Two minus = two(-1.0f, -1.0f);
#pragma unroll
        for (int i = 0; i < kEach / 2; i++) {
            if (kShort) {
                const Two p = mul2(h[i], h[i]), s = add2(sum, p), b = fma2(s, minus, sum);  // b: minus what sum grew by
                rest = add2(rest, add2(fma2(add2(s, b), minus, sum), add2(p, b)));
                sum = s;
            } else {
                const Two p = mul2(mul2(h[i], minus), h[i]);  // minus the square
                const Two s = fma2(p, minus, sum), b = fma2(s, minus, sum), left = fma2(h[i], h[i], p);
                rest = add2(rest, add2(add2(fma2(add2(s, b), minus, sum), fma2(p, minus, b)), left));
                sum = s;
            }
        }
    }
    __device__ __forceinline__ Pair pair() const {
        const float2 s = apart(sum), left = apart(rest);
        Pair p = {s.x, left.x + left.y};
        p.add(s.y);
        return p;
    }
};
__device__ __forceinline__ double squares_of(const Two (&h)[kEach / 2]) {
    double s = 0.0;
    for (int i = 0; i < kEach / 2; i++) {
        const float2 f = apart(h[i]);
        s += double(f.x) * f.x + double(f.y) * f.y;
    }
    return s;
}
// The largest magnitude's bits: NaN above infinity above numbers.
__device__ __forceinline__ uint32_t largest_of(const Two (&y)[kEach / 2]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kEach / 2; i++) most = max(most, max(uint32_t(y[i]) & 0x7FFFFFFFu, uint32_t(y[i] >> 32) & 0x7FFFFFFFu));
    return most;
}

__device__ __forceinline__ Pair warp_sum(Pair p, int lanes) {
    for (int d = lanes / 2; d; d >>= 1) {
        const float s = __shfl_xor_sync(~0u, p.sum, d), rest = __shfl_xor_sync(~0u, p.rest, d);
        p.add(s);
        p.rest += rest;
    }
    return p;
}
// root_of all threads' sums, in all of them: below 0 where it is false. By one warp, as
// in all of them it would be half of the kernel's instructions.
struct RootSpace {
    Pair pairs[32];
    float root;
};
__device__ __forceinline__ float block_root(const Pair &mine, const NormArgs &a, RootSpace &space) {
    const int lane = threadIdx.x & 31;
    Pair p = mine;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const float s = __shfl_xor_sync(~0u, p.sum, d), rest = __shfl_xor_sync(~0u, p.rest, d);
        p.add(s);
        p.rest += rest;
    }
    if (lane == 0) space.pairs[threadIdx.x >> 5] = p;
    __syncthreads();
    if (threadIdx.x < 32) {
        const int warps = int(blockDim.x) >> 5;
        p = {0.0f, 0.0f};
        if (lane < warps) p = space.pairs[lane];
        float r = -1.0f;
        const bool ok = root_of(warp_sum(p, warps <= 8 ? 8 : 32), a, &r);  // lane 0's is of all
        if (lane == 0) space.root = ok ? r : -1.0f;
    }
    __syncthreads();
    return space.root;
}
__device__ __forceinline__ double block_sum(double s, double *doubles) {
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    if ((threadIdx.x & 31) == 0) doubles[threadIdx.x >> 5] = s;
    __syncthreads();
    s = doubles[0];
    for (int i = 1; i < int(blockDim.x) >> 5; i++) s += doubles[i];
    return s;
}
__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t *maxima) {
    const int lane = threadIdx.x & 31;
    m = __reduce_max_sync(~0u, m);
    if (lane == 0) maxima[threadIdx.x >> 5] = m;
    __syncthreads();
    return __reduce_max_sync(~0u, lane < int(blockDim.x) >> 5 ? maxima[lane] : 0u);
}

// x / s for two numbers, each rounded once: with r = 1 / s rounded once, q = x r is
// off by a unit of its last place at most, x - q s is a number of 32 bits, and q + (x - q s) r
// rounds as x / s does (Markstein's theorem), as long as nothing leaves the range. The sign of
// a 0 is put back.
__device__ __forceinline__ Two divide2(Two x, Two minus_s, Two r) {
    const Two q = mul2(x, r);
    return fma2(fma2(q, minus_s, x), r, q) | (x & 0x8000000080000000ull);
}

// Eight columns from c on of y as e4m3, with the scale of their block of 128: all
// of 16 threads' columns.
__device__ __forceinline__ void put8(const NormArgs &a, int64_t m, int32_t c, const Two (&y)[kEach / 2]) {
    float v[kEach], amax = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach / 2; i++) {
        const float2 f = apart(y[i]);
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
        amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
    }
#pragma unroll
    for (int d = 8; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, d));
    const float s = scale_of(amax);
    if (s > 0x1p-60f && s < 0x1p60f) {
        const float r = __frcp_rn(s);
#pragma unroll
        for (int i = 0; i < kEach / 2; i++) {
            const float2 f = apart(divide2(y[i], two(-s, -s), two(r, r)));
            v[2 * i] = f.x, v[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; i++) v[i] = __fdiv_rn(v[i], s);
    }
    uint32_t out[2];
#pragma unroll
    for (int i = 0; i < 2; i++)
        out[i] = uint32_t(__nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3)) |
                 uint32_t(__nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3)) << 16;
    uint8_t *q = a.q + m * a.D + c;
    if (a.wide_q && c + kEach <= a.D) {
        *reinterpret_cast<uint2 *>(q) = make_uint2(out[0], out[1]);
    } else if (c + kEach <= a.D) {  // as large as they can be, the same in all threads of a row
        const uint32_t off = reinterpret_cast<uintptr_t>(q) & 3u;
        if (off == 0) {
            reinterpret_cast<uint32_t *>(q)[0] = out[0];
            reinterpret_cast<uint32_t *>(q)[1] = out[1];
        } else if (off == 2) {
            *reinterpret_cast<uint16_t *>(q) = uint16_t(out[0]);
            *reinterpret_cast<uint32_t *>(q + 2) = __funnelshift_r(out[0], out[1], 16);
            *reinterpret_cast<uint16_t *>(q + 6) = uint16_t(out[1] >> 16);
        } else if (off == 1) {
            q[0] = uint8_t(out[0]);
            *reinterpret_cast<uint16_t *>(q + 1) = uint16_t(out[0] >> 8);
            *reinterpret_cast<uint32_t *>(q + 3) = __funnelshift_r(out[0], out[1], 24);
            q[7] = uint8_t(out[1] >> 24);
        } else {
            q[0] = uint8_t(out[0]);
            *reinterpret_cast<uint32_t *>(q + 1) = __funnelshift_r(out[0], out[1], 8);
            *reinterpret_cast<uint16_t *>(q + 5) = uint16_t(out[1] >> 8);
            q[7] = uint8_t(out[1] >> 24);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; i++)
            if (c + i < a.D) q[i] = uint8_t(out[i / 4] >> (i % 4 * 8));
    }
    if ((threadIdx.x & 15) == 0 && c < a.D) a.scales[int64_t(c / kBlock) * a.pitch + m] = s;
}
// The same as e2m1; a block of 16 is two threads', a word of scales eight threads'.
__device__ __forceinline__ void put4(const NormArgs &a, int64_t m, int32_t c, const Two (&y)[kEach / 2], float row_scale, float per_row) {
    const int lane = threadIdx.x & 31;
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach / 2; i++) {
        const float2 f = apart(y[i]);
        amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
    }
    amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
    const bool in_range = row_scale > 0x1p-60f && row_scale < 0x1p60f;
    const float t = in_range ? apart(divide2(two(amax, 0.0f), two(-row_scale, 0.0f), two(per_row, 0.0f))).x : __fdiv_rn(amax, row_scale);
    const uint8_t s = to_e4m3(__fmul_rn(t, 1.0f / 6.0f));
    const float per = per_step4(s, row_scale);
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < kEach / 2; i++) {
        const float2 f = apart(mul2(y[i], two(per, per)));
        out |= uint32_t(to_e2m1x2(f.x, f.y)) << (8 * i);
    }
    if (c < row_bytes4(a.D) * 2) *reinterpret_cast<uint32_t *>(a.q + m * row_bytes4(a.D) + c / 2) = out;
    uint32_t word = uint32_t(s) << (8 * ((lane >> 1) & 3));
    word |= __shfl_xor_sync(~0u, word, 2);
    word |= __shfl_xor_sync(~0u, word, 4);
    const int64_t tiles = scale_tiles4(a.D);
    if ((lane & 7) == 0 && c < tiles * 64) *reinterpret_cast<uint32_t *>(a.scales4 + scale_word4(m, c / 64, tiles)) = word;
}

// Rows of any length and alignment, a CTA a row: read again in each pass (the
// residual as it was written).
template <bool kWide, bool kFew, bool kNorm, int kBits>
__global__ void __launch_bounds__(kFew ? kMaxThreads : kNormThreads) k_norm_long(const __grid_constant__ NormArgs a) {
    __shared__ RootSpace space;
    __shared__ double doubles[32];
    __shared__ uint32_t maxima[32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int32_t m = blockIdx.x, D = a.D, mine = int32_t(threadIdx.x) * kEach;
    const int32_t stride = int32_t(blockDim.x) * kEach;
    const void *x = static_cast<const char *>(a.x) + m * a.stride * (a.x_f32 ? 4 : 2);
    void *residual = static_cast<char *>(a.residual) + m * a.residual_stride * (a.residual_f32 ? 4 : 2);
    const bool has_residual = kNorm && a.residual;
    float r = 0.0f;

    auto again = [&](int32_t c, Two (&h)[kEach / 2]) {
        const bool f32 = has_residual ? a.residual_f32 : a.x_f32;
        values8<kWide>(load8<kWide>(has_residual ? residual : x, f32, c, D), f32, h);
    };
    auto normed = [&](int32_t c, Two (&h)[kEach / 2]) {
        again(c, h);
        if (!kNorm) return;
        Two g[kEach / 2];
        values8<kWide>(load8<kWide>(a.gain, a.gain_f32, c, D), a.gain_f32, g);
#pragma unroll
        for (int i = 0; i < kEach / 2; i++) {
            h[i] = mul2(mul2(h[i], two(r, r)), g[i]);
            const float2 f = apart(h[i]);  // 0 behind the end, whatever r is
            h[i] = two(c + 2 * i < D ? f.x : 0.0f, c + 2 * i + 1 < D ? f.y : 0.0f);
        }
    };
    if (kNorm) {
        Squares<false> all;
        for (int32_t c = mine; c < D; c += stride) {
            Two h[kEach / 2];
            values8<kWide>(load8<kWide>(x, a.x_f32, c, D), a.x_f32, h);
            if (has_residual) {
                Two v[kEach / 2];
                values8<kWide>(load8<kWide>(residual, a.residual_f32, c, D), a.residual_f32, v);
#pragma unroll
                for (int i = 0; i < kEach / 2; i++) h[i] = add2(h[i], v[i]);
                store8<kWide>(residual, a.residual_f32, c, D, h);
            }
            all.add(h);
        }
        r = block_root(all.pair(), a, space);
        if (r < 0.0f) {
            double wide = 0.0;
            for (int32_t c = mine; c < D; c += stride) {
                Two h[kEach / 2];
                again(c, h);
                wide += squares_of(h);
            }
            r = float(1.0 / sqrt(block_sum(wide, doubles) / D + a.eps));
        }
    }
    float row_scale = 0.0f, per_row = 0.0f;  // and its reciprocal
    if (kBits == 4) {
        uint32_t most = 0;
        for (int32_t c = mine; c < D; c += stride) {
            Two y[kEach / 2];
            normed(c, y);
            most = max(most, largest_of(y));
        }
        row_scale = row_scale4(block_max(most, maxima));
        per_row = __frcp_rn(row_scale);
        if (threadIdx.x == 0) a.row_scales[m] = row_scale;
    }
    for (int32_t c = mine; c - lane * kEach < (D + 127) / 128 * 128; c += stride) {
        Two y[kEach / 2];
        normed(c, y);
        if (kBits == 8) put8(a, m, c, y);
        else put4(a, m, c, y, row_scale, per_row);
    }
}

// 16 bytes to shared memory, zeros where `there` is false; asynchronous.
__device__ __forceinline__ void copy16(uint32_t to, const void *from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

template <bool kWide, bool kNorm, int kBits>
cudaError_t launch_long(const NormArgs &a, cudaStream_t st) {
    const int32_t eights = (a.D + kEach - 1) / kEach;
    // Few rows: as many threads as there are eights (300 rows, D 7,363, f32 13 us, and 22 in more rounds).
    if (a.M <= 2 * sm_count())
        return launch_pdl(k_norm_long<kWide, true, kNorm, kBits>, a.M, std::min(kMaxThreads, (eights + 31) / 32 * 32), st, a);
    // Many: the number that is idle least in the last round, of two rounds or more where there are so many (16,384
    // rows, D 5,120, f32 without residual 160 threads 108 us, 256 117).
    int threads = (std::min(eights, 128) + 31) / 32 * 32, least = (eights + threads - 1) / threads * threads;
    for (int n = 160; n <= kNormThreads && n < eights; n += 32) {
        const int32_t all = (eights + n - 1) / n * n;
        if (all <= least) threads = n, least = all;
    }
    return launch_pdl(k_norm_long<kWide, false, kNorm, kBits>, a.M, threads, st, a);
}

struct None {};
template <typename T>
constexpr int kPieces = std::is_same<T, None>::value ? 0 : int(sizeof(T)) / 2;  // 16-byte pieces of eight columns

// Aligned rows of whole eights of columns that kSteps steps of a CTA's threads
// hold: CTAs stay and go over the rows, and copy the next row's columns to shared
// memory while they look at this one's. A thread copies and reads its own columns
// only. TR: the residual's type, or None.
template <typename TX, typename TR, bool kNorm, int kBits, int kSteps>
__global__ void __launch_bounds__(kSteps == 1 ? kMaxThreads : kHoldThreads, kSteps)
    k_norm_rows(const __grid_constant__ NormArgs a) {
    constexpr bool kResidual = !std::is_same<TR, None>::value;
    using R = typename std::conditional<kResidual, TR, float>::type;
    constexpr int kX = kPieces<TX>, kEachStep = kX + kPieces<TR>;
    extern __shared__ __align__(16) uint4 space[];  // [a.buffers][kSteps][kEachStep][threads], then the gain as [kSteps][4][threads] pairs
    __shared__ RootSpace roots[2];
    __shared__ double doubles[32];
    __shared__ uint32_t maxima[2][32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, threads = blockDim.x;
    const int32_t D = a.D, stride = threads * kEach, mine = int32_t(threadIdx.x) * kEach;
    uint4 *const own = space + threadIdx.x;
    Two *const gains = reinterpret_cast<Two *>(space + a.buffers * kSteps * kEachStep * threads) + threadIdx.x;
    const TX *x = static_cast<const TX *>(a.x) + blockIdx.x * a.stride + mine;
    R *residual = static_cast<R *>(a.residual) + blockIdx.x * a.residual_stride + mine;
    const int64_t x_step = int64_t(gridDim.x) * a.stride, residual_step = int64_t(gridDim.x) * a.residual_stride;
    auto ask = [&](int turn, const TX *from, const R *from_residual) {
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            const bool there = mine + i * stride < D;
#pragma unroll
            for (int k = 0; k < kEachStep; k++) {
                const void *at = k < kX ? static_cast<const void *>(reinterpret_cast<const uint4 *>(from + (there ? i * stride : 0)) + k)
                                        : static_cast<const void *>(reinterpret_cast<const uint4 *>(from_residual + (there ? i * stride : 0)) + k - kX);
                copy16(smem_addr(own + ((turn * kSteps + i) * kEachStep + k) * threads), at, there);
            }
        }
    };
    auto values = [&](int turn, int i, int k0, bool f32, Two (&v)[kEach / 2]) {
        const uint4 lo = own[((turn * kSteps + i) * kEachStep + k0) * threads];
        const uint4 hi = f32 ? own[((turn * kSteps + i) * kEachStep + k0 + 1) * threads] : lo;
        values8<true>(Raw{{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}}, f32, v);
    };
    ask(0, x, residual);
    copies_commit();
    if (kNorm) {
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            Two g[kEach / 2];
            values8<true>(load8<true>(a.gain, a.gain_f32, mine + i * stride, D), a.gain_f32, g);
#pragma unroll
            for (int k = 0; k < kEach / 2; k++) gains[(i * (kEach / 2) + k) * threads] = g[k];
        }
    }
    int turn = 0;
    for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x, turn ^= 1) {
        x += x_step;
        if (kResidual) residual += residual_step;
        if (m + gridDim.x < a.M) ask(turn ^ 1, x, residual);
        copies_commit();
        copies_wait<1>();
        Two held[kSteps][kEach / 2];
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            values(turn, i, 0, kX == 2, held[i]);
            if (kResidual) {
                Two v[kEach / 2];
                values(turn, i, kX, sizeof(R) == 4, v);
#pragma unroll
                for (int k = 0; k < kEach / 2; k++) held[i][k] = add2(held[i][k], v[k]);
                store8<true>(residual - residual_step - mine, sizeof(R) == 4, mine + i * stride, D, held[i]);
            }
        }
        if (kNorm) {
            Squares<(kResidual ? sizeof(R) : sizeof(TX)) == 2> all;
#pragma unroll
            for (int i = 0; i < kSteps; i++) all.add(held[i]);
            float r = block_root(all.pair(), a, roots[turn]);
            if (r < 0.0f) {
                double wide = 0.0;
                for (int i = 0; i < kSteps; i++) wide += squares_of(held[i]);
                __syncthreads();  // the row before may still be reading
                r = float(1.0 / sqrt(block_sum(wide, doubles) / D + a.eps));
            }
            const Two rr = two(r, r);  // behind the end both factors are 0 (and where r is a NaN the row is)
#pragma unroll
            for (int i = 0; i < kSteps; i++)
#pragma unroll
                for (int k = 0; k < kEach / 2; k++) held[i][k] = mul2(mul2(held[i][k], rr), gains[(i * (kEach / 2) + k) * threads]);
        }
        float row_scale = 0.0f, per_row = 0.0f;  // and its reciprocal
        if (kBits == 4) {
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < kSteps; i++) most = max(most, largest_of(held[i]));
            row_scale = row_scale4(block_max(most, maxima[turn]));
            per_row = __frcp_rn(row_scale);
            if (threadIdx.x == 0) a.row_scales[m] = row_scale;
        }
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            const int32_t c = mine + i * stride;
            if (c - lane * kEach >= (D + 127) / 128 * 128) break;  // the warp has nothing there
            if (kBits == 8) put8(a, m, c, held[i]);
            else put4(a, m, c, held[i], row_scale, per_row);
        }
    }
}

template <typename TX, typename TR, bool kNorm, int kBits, int kSteps>
cudaError_t launch_held(NormArgs a, int threads, cudaStream_t st) {
    auto space = [&](int buffers) {
        return size_t(threads) * kSteps * (buffers * (kPieces<TX> + kPieces<TR>) * sizeof(uint4) + (kNorm ? kEach * sizeof(float) : 0));
    };
    // CTAs that stay, as many as fit an SM by threads (64 registers each) and shared
    // memory; where they would take few rows each, a CTA a row.
    const int fit = std::max(1, std::min(1024 / threads, int(kMostSpace / (space(2) + 2048))));
    const int64_t stay = int64_t(sm_count()) * fit;
    a.buffers = a.M > kStayRows * stay ? 2 : 1;
    const size_t smem = space(a.buffers);
    static_assert(size_t(kMaxThreads) * (2 * 4 * sizeof(uint4) + kEach * sizeof(float)) <= kMostSpace, "any row that is held");
    if (smem > 40 * 1024) {  // what is declared in the kernel counts towards the 48 KB that need no leave
        const cudaError_t e = allow_smem<k_norm_rows<TX, TR, kNorm, kBits, kSteps>, int(kMostSpace)>();
        if (e != cudaSuccess) return e;
    }
    return launch_pdl_smem(k_norm_rows<TX, TR, kNorm, kBits, kSteps>, a.buffers == 2 ? stay : int64_t(a.M), threads, smem, st, a);
}

template <typename TX, typename TR, bool kNorm, int kBits>
cudaError_t launch_rows(const NormArgs &a, cudaStream_t st) {
    const int32_t eights = int32_t((int64_t(a.D) + 63) / 64 * 64 / kEach);
    auto threads = [&](int steps) { return ((eights + steps - 1) / steps + 31) / 32 * 32; };
    if (a.M <= 2 * sm_count()) {
        // Few rows: a step a thread, as many threads as that takes, for the shortest chain (256 rows, D 4,096 4.6
        // us, and 6.1 in two steps).
        if (eights <= kMaxThreads) return launch_held<TX, TR, kNorm, kBits, 1>(a, threads(1), st);
    } else if constexpr (kPieces<TX> < 2 && kPieces<TR> < 2) {
        // Many: two steps, so that what a warp does for a row is shared by more of its columns.
        if (eights <= 64) return launch_held<TX, TR, kNorm, kBits, 1>(a, threads(1), st);
        if (eights <= 2 * kHoldThreads) return launch_held<TX, TR, kNorm, kBits, 2>(a, threads(2), st);
    }
    // Longer rows; and many with 32-bit values, which take so much shared memory that too few CTAs fit (12,010 rows,
    // D 8,192, x and the residual in f32 205 us, and 310 in two steps; in bf16 158 and 131).
    return launch_long<true, kNorm, kBits>(a, st);
}

template <typename TX, bool kNorm, int kBits>
cudaError_t launch_typed(const NormArgs &a, cudaStream_t st) {
    if constexpr (kNorm) {
        if (a.residual) return a.residual_f32 ? launch_rows<TX, float, kNorm, kBits>(a, st) : launch_rows<TX, __nv_bfloat16, kNorm, kBits>(a, st);
    }
    return launch_rows<TX, None, kNorm, kBits>(a, st);
}

template <bool kNorm, int kBits>
int launch_norm(const NormArgs &a, cudaStream_t st) {
    const cudaError_t e = !a.wide ? launch_long<false, kNorm, kBits>(a, st)
                          : a.x_f32 ? launch_typed<float, kNorm, kBits>(a, st) : launch_typed<__nv_bfloat16, kNorm, kBits>(a, st);
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
    a.x_f32 = dtype == TRIE_DTYPE_F32;
    a.wide = D % 8 == 0 && wide_rows(x, dtype, stride, M) && (!residual || wide_rows(residual, residual_dtype, residual_stride, M)) &&
             (!gain || wide_rows(gain, gain_dtype, 0, 1));
    a.eps = eps;
    a.eps_32 = float(eps);
    a.eps_rest = float(eps - double(a.eps_32));
    a.per_column = 1.0f / float(D);
    a.per_column_rest = float(1.0 / D - double(a.per_column));
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
    return launch_norm<true, 8>(a, stream);
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
    return launch_norm<false, 4>(a, stream);
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
    return launch_norm<true, 4>(a, stream);
}
