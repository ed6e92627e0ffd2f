// What the quantizing kernels (head.cu, norm.cu) share: e4m3 with scales of 128
// columns, and e2m1 with e4m3 scales of 16 columns and a 32-bit scale of a row.
#pragma once

#include <stdint.h>

#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "logits.cuh"

namespace tmk {

constexpr int kBlock = 128;  // columns (and rows of 8-bit weights) that share a scale
constexpr float kPerMax = 1.0f / 448.0f;  // 448: the largest e4m3 number

__device__ __forceinline__ uint8_t to_e4m3(float x) {
    return uint8_t(__nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3));
}

// NaN does not show in the maximum, but a NaN element becomes a NaN in e4m3 and
// an infinite one makes the scale infinite and itself NaN: either way the row's
// logits are NaN.
__device__ __forceinline__ float scale_of(float amax) {
    const float s = __fmul_rn(amax, kPerMax);
    return s > 0.0f ? s : 1.0f;
}

// ---- 4 bits: x ~ q s S, q e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives),
// s e4m3 for 16 columns of a row, S 32 bits for the row. The row's largest
// magnitude is 6 x 448 of S, so that the largest block's scale is e4m3's largest
// number and blocks down to 1/28,000 of it keep three bits. e2m1 has no NaN: a
// row with a NaN or an infinity has S = NaN, so its logits are NaN.
constexpr int kGroup4 = 16;                     // columns that share an e4m3 scale
constexpr float kPerMax4 = 1.0f / 2688.0f;      // 6 x 448
constexpr float kTinyRow4 = 7.8886090522101181e-31f;  // 2^-100: the steps s S and their reciprocals stay normal numbers

__device__ __forceinline__ float row_scale4(uint32_t amax_bits) {
    if (amax_bits >= 0x7F800000u) return __int_as_float(0x7FC00000);
    return fmaxf(__fmul_rn(__uint_as_float(amax_bits), kPerMax4), kTinyRow4);
}
__device__ __forceinline__ float from_e4m3(uint8_t x) {
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(__nv_fp8_storage_t(x), __NV_E4M3)));
}
// What values of a block are multiplied by before they are rounded to e2m1.
__device__ __forceinline__ float per_step4(uint8_t scale, float row_scale) {
    const float step = __fmul_rn(from_e4m3(scale), row_scale);
    return step > 0.0f ? __fdiv_rn(1.0f, step) : 0.0f;
}
// Two codes, the first in the low half.
__device__ __forceinline__ uint8_t to_e2m1x2(float x, float y) {
    return uint8_t(__nv_cvt_float2_to_fp4x2(make_float2(x, y), __NV_E2M1, cudaRoundNearest));
}

// Sizes of the 4-bit form: bytes of a row (32 columns are 16 bytes: rows start on
// 16-byte boundaries), and of the scales, which lie as the tensor core takes them: 128 rows x 64 columns
// in 512 bytes, row r and columns 16 j on at (r % 32) 16 + r / 32 4 + j.
__host__ __device__ constexpr int64_t row_bytes4(int32_t D) { return (int64_t(D) + 31) / 32 * 16; }
__host__ __device__ constexpr int64_t scale_tiles4(int32_t D) { return (int64_t(D) + 63) / 64; }
__host__ __device__ constexpr int64_t scale_word4(int64_t row, int32_t tile, int64_t tiles) {
    return ((row >> 7) * tiles + tile) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4;
}

}  // namespace tmk
