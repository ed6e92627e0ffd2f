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
//  k_head_logits           the product on the tensor cores.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include "blackwell.cuh"
#include "logits.cuh"

namespace tmk {

namespace {

constexpr int kBlock = 128;  // columns (and weight rows) that share a scale
constexpr float kPerMax = 1.0f / 448.0f;  // 448: the largest e4m3 number
constexpr int kQuantThreads = 256;

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

// ---- the product
//
// A tile is up to 128 rows of the batch, the MMA's rows, by NT tokens, its
// columns; a thread of the epilogue then holds one row, and the scale of a
// block is one number for it and 64 tokens (a weight scale covers 128). One
// thread streams blocks of 128 columns of K of both operands into a ring of
// stages by TMA, one issues a block's four MMAs into one of two accumulators in
// tensor memory, and the epilogue warps read each block's sums out and add
// them, scaled, to sums in registers, a warp 32 rows by 64 tokens. Rows that a
// batch does not have are not loaded (the MMA multiplies what lies there into
// rows nobody reads), and warps that would have only such rows do nothing.
constexpr int kRows = 128;
constexpr int kColumns = 64;       // tokens of an epilogue warp
constexpr int kMaxStages = 8;

struct HeadArgs {
    CUtensorMap map_w, map_q;
    const float *s;        // [blocks][pitch]
    int64_t pitch;
    const float *ws;       // [ceil(V / 128)][blocks]
    int32_t M, V, blocks;
    int32_t m_tiles;       // tiles of kRows rows
    int32_t box_rows;      // rows of a tile that are loaded
    int32_t stages;        // of the ring
    void *logits;
    int64_t stride;
    Grammar g;
};

template <int NT>
struct HeadShape {
    static constexpr int kEpilogue = 4 * (NT / kColumns);  // warps
    static constexpr int kThreads = 64 + 32 * kEpilogue;
    static constexpr int kCtas = NT == 128 ? 2 : 1;        // of an SM
    static constexpr int kTmem = 2 * NT;
    static constexpr int kBudget = (kCtas == 2 ? 111 : 222) * 1024;  // bytes of shared memory
    static constexpr int kWeightBytes = NT * kBlock;
};

// Writes -inf to rows [m0, m1) of tokens [v0, v1) (at most 256), by all threads.
template <typename T>
__device__ void fill_tile(const HeadArgs &a, int32_t m0, int32_t m1, int32_t v0, int32_t v1) {
    const int lane = threadIdx.x & 31;
    const T none = from_f32<T>(-INFINITY);
    for (int32_t m = m0 + int32_t(threadIdx.x >> 5); m < m1; m += int32_t(blockDim.x >> 5)) {
        T *out = static_cast<T *>(a.logits) + m * a.stride + v0;
        if ((v1 - v0) % 128 == 0 && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(T) - 1)) == 0) {
            for (int32_t i = lane; i < (v1 - v0) / 4; i += 32) {
                if (sizeof(T) == 2) reinterpret_cast<uint2 *>(out)[i] = make_uint2(0xFF80FF80u, 0xFF80FF80u);
                else reinterpret_cast<uint4 *>(out)[i] = make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u);
            }
        } else {
            for (int32_t i = lane; i < v1 - v0; i += 32) out[i] = none;
        }
    }
}

// A warp's 32 rows x 64 tokens of sums to memory: turned in shared memory
// (`turn`: 32 rows of 64 values and 4 bytes, so that neither side has bank
// conflicts), so that a row's tokens are written side by side.
template <typename T>
__device__ __forceinline__ void store_block(const HeadArgs &a, unsigned char *turn, const uint64_t (&sum)[kColumns / 2],
                                            int32_t m, int32_t m1, int32_t v, int lane) {
    constexpr int kPitch = kColumns * int(sizeof(T)) / 4 + 1;  // words
    uint32_t *mine = reinterpret_cast<uint32_t *>(turn) + lane * kPitch;
#pragma unroll
    for (int i = 0; i < kColumns / 2; i++) {
        float lo, hi;
        unpack2(sum[i], lo, hi);
        if (sizeof(T) == 2) {
            const __nv_bfloat162 both = __floats2bfloat162_rn(lo, hi);
            mine[i] = *reinterpret_cast<const uint32_t *>(&both);
        } else {
            mine[2 * i] = __float_as_uint(lo);
            mine[2 * i + 1] = __float_as_uint(hi);
        }
    }
    __syncwarp();
    const int32_t rows = min(32, m1 - m), left = a.V - v;  // of this warp, of its tokens
    T *out = static_cast<T *>(a.logits) + m * a.stride + v;
    if (sizeof(T) == 2 && left >= kColumns && (reinterpret_cast<uintptr_t>(out) & 3) == 0 && (a.stride & 1) == 0) {
        for (int32_t r = 0; r < rows; r++)
            reinterpret_cast<uint32_t *>(out + r * a.stride)[lane] = reinterpret_cast<uint32_t *>(turn)[r * kPitch + lane];
    } else {
        for (int32_t r = 0; r < rows; r++) {
            const T *from = reinterpret_cast<const T *>(reinterpret_cast<uint32_t *>(turn) + r * kPitch);
            if (lane < left) out[r * a.stride + lane] = from[lane];
            if (lane + 32 < left) out[r * a.stride + lane + 32] = from[lane + 32];
        }
    }
}

template <typename T, int NT>
__global__ void __launch_bounds__(HeadShape<NT>::kThreads, HeadShape<NT>::kCtas) k_head_logits(const __grid_constant__ HeadArgs a) {
    using S = HeadShape<NT>;
    extern __shared__ unsigned char dynamic_smem[];
    __shared__ uint64_t bars[2 * kMaxStages + 4];
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int32_t vt = int32_t(blockIdx.x / unsigned(a.m_tiles)), v0 = vt * NT;
    const int32_t m0 = int32_t(blockIdx.x % unsigned(a.m_tiles)) * kRows, m1 = min(a.M, m0 + kRows);
    const int quarters = (m1 - m0 + 31) / 32;  // warps' rows that there are
    const uint32_t full = smem_addr(bars), empty = full + 8 * kMaxStages;
    const uint32_t ready = empty + 8 * kMaxStages, drained = ready + 16;
    unsigned char *ring = dynamic_smem + ((1024u - (smem_addr(dynamic_smem) & 1023u)) & 1023u);
    const uint32_t stages = smem_addr(ring), stage_bytes = uint32_t(S::kWeightBytes + a.box_rows * kBlock);
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int i = 0; i < a.stages; i++) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; i++) {
            bar_init(ready + 8 * i, 1);
            bar_init(drained + 8 * i, uint32_t(quarters * (NT / kColumns)));
        }
        bar_init_fence();
        tma_prefetch_map(&a.map_w);
        tma_prefetch_map(&a.map_q);
    }
    pdl_launch_dependents();
    pdl_wait();
    if (a.g.mask) {
        // a tile that no row of the batch allows a token of needs no weights
        bool any = false;
        const int32_t w0 = v0 >> 5, words = min(NT / 32, int32_t(a.g.W) - w0);
        for (int32_t m = m0 + int32_t(threadIdx.x); m < m1 && !any; m += int32_t(blockDim.x)) {
            const GrammarRow row = grammar_row(a.g, m);
            for (int32_t i = 0; i < words; i++) any |= row.word(w0 + i) != 0u;
        }
        if (!__syncthreads_or(any)) {
            fill_tile<T>(a, m0, m1, v0, min(a.V, v0 + NT));
            return;
        }
    }
    if (warp == 1) tmem_alloc(smem_addr(&tmem_base), S::kTmem);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = *static_cast<volatile uint32_t *>(&tmem_base);

    if (warp == 0) {
        if (lane == 0) {
            int32_t kb = 0;
            int stage = 0;
            uint32_t phase = 1;  // of the stage's last use: the first time round there is none
            for (; kb < a.blocks; kb++) {
                const uint32_t at = stages + uint32_t(stage) * stage_bytes, bar = full + 8 * stage;
                if (!bar_wait(empty + 8 * stage, phase, &gave_up)) break;
                bar_expect(bar, stage_bytes);
                tma_load_2d(at, &a.map_w, kb * kBlock, v0, bar);
                tma_load_2d(at + S::kWeightBytes, &a.map_q, kb * kBlock, m0, bar);
                if (++stage == a.stages) stage = 0, phase ^= 1;
            }
            if (gave_up) {  // copies may still write to shared memory: wait for them
                int none = 0;
                for (int32_t i = max(0, kb - a.stages); i < kb; i++)
                    bar_wait(full + 8 * (i % a.stages), (i / a.stages) & 1, &none);
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = mma_idesc_e4m3(kRows, NT);
            int stage = 0;
            uint32_t phase = 0;
            for (int32_t kb = 0; kb < a.blocks; kb++) {
                const int acc = kb & 1;
                if (!bar_wait(drained + 8 * acc, ((kb >> 1) & 1) ^ 1, &gave_up)) break;
                if (!bar_wait(full + 8 * stage, phase, &gave_up)) break;
                tcgen05_fence_after();
                const uint32_t at = stages + uint32_t(stage) * stage_bytes;
                const uint64_t dw = mma_desc(at), dq = mma_desc(at + S::kWeightBytes);
#pragma unroll
                for (int k = 0; k < kBlock / 32; k++) mma_e4m3(tmem + acc * NT, dq + 2 * k, dw + 2 * k, idesc, k > 0);
                mma_commit(empty + 8 * stage);
                mma_commit(ready + 8 * acc);
                if (++stage == a.stages) stage = 0, phase ^= 1;
            }
        }
    } else if ((warp & 3) < quarters) {
        const int quarter = warp & 3, column = (warp - 2) / 4 * kColumns;
        const uint32_t from = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(column);
        const int32_t row = min(m0 + quarter * 32 + lane, a.M - 1), v = v0 + column;
        uint64_t sum[kColumns / 2];
#pragma unroll
        for (int i = 0; i < kColumns / 2; i++) sum[i] = 0ull;
        bool ok = true;
        // scales are read two blocks ahead
        const float *sp = a.s + row, *wp = a.ws + int64_t(min(v, a.V - 1) / kBlock) * a.blocks;
        float s0 = __ldg(sp) * __ldg(wp), s1 = 0.0f;
        if (a.blocks > 1) s1 = __ldg(sp + a.pitch) * __ldg(wp + 1);
        for (int32_t kb = 0; kb < a.blocks; kb++) {
            const int acc = kb & 1;
            const uint64_t scale = pack2(s0, s0);
            s0 = s1;
            if (kb + 2 < a.blocks) s1 = __ldg(sp + (kb + 2) * a.pitch) * __ldg(wp + kb + 2);
            ok = __all_sync(~0u, bar_wait(ready + 8 * acc, (kb >> 1) & 1, &gave_up));
            if (!ok) break;
            tcgen05_fence_after();
#pragma unroll
            for (int c = 0; c < kColumns; c += 16) {
                uint32_t r[16];
                tmem_load16(from + acc * NT + c, r);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; i += 2) sum[(c + i) / 2] = fma2(pack2u(r[i], r[i + 1]), scale, sum[(c + i) / 2]);
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(drained + 8 * acc);
        }
        // a tile that gave up waiting has no result: NaN
        if (!ok) {
#pragma unroll
            for (int i = 0; i < kColumns / 2; i++) sum[i] = 0x7FFFFFFF7FFFFFFFull;
        }
        if (a.g.mask) {
            const GrammarRow allow = grammar_row(a.g, row);
#pragma unroll
            for (int c = 0; c < kColumns; c += 32) {
                const uint32_t word = (v + c) >> 5 < a.g.W ? allow.word((v + c) >> 5) : 0u;
                if (word == ~0u) continue;
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    float lo, hi;
                    unpack2(sum[(c + i) / 2], lo, hi);
                    if (!((word >> i) & 1u)) lo = -INFINITY;
                    if (!((word >> (i + 1)) & 1u)) hi = -INFINITY;
                    sum[(c + i) / 2] = pack2(lo, hi);
                }
            }
        }
        // every MMA is done (the last `ready`), so the ring is free to turn the block in
        if (ok && v < a.V)
            store_block<T>(a, ring + (warp - 2) * 32 * (kColumns * int(sizeof(T)) + 4), sum, m0 + quarter * 32, m1, v, lane);
    }
    __syncwarp();
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    if (warp == 1) tmem_free(tmem, S::kTmem);
}

// [rows][D] bytes in boxes of box_rows x 128, 128-byte swizzle, zeros outside.
bool make_map(CUtensorMap *map, const void *base, int64_t rows, int32_t D, int32_t box_rows) {
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult got;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &got) != cudaSuccess ||
            got != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<Encode>(f);
    }();
    if (!encode) return false;
    const cuuint64_t dims[2] = {cuuint64_t(D), cuuint64_t(rows)}, strides[1] = {cuuint64_t(D)};
    const cuuint32_t box[2] = {cuuint32_t(kBlock), cuuint32_t(box_rows)}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int NT>
cudaError_t launch_head(HeadArgs a, int64_t grid, cudaStream_t st) {
    using S = HeadShape<NT>;
    const int stage = S::kWeightBytes + a.box_rows * kBlock;
    // the last stage's MMA reads kRows rows, whatever was loaded; and room to align the ring
    const int beyond = (kRows - a.box_rows) * kBlock + 1024;
    a.stages = std::min(kMaxStages, (S::kBudget - beyond) / stage);
    const int turn = S::kEpilogue * 32 * (kColumns * int(sizeof(T)) + 4) + 1024;
    const int smem = std::max(a.stages * stage + beyond, turn);
    const cudaError_t e = cudaFuncSetAttribute(k_head_logits<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBudget);
    if (e != cudaSuccess) return e;
    return launch_pdl_smem(k_head_logits<T, NT>, grid, S::kThreads, smem, st, a);
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
    HeadArgs a = {};
    a.s = d_scales;
    a.pitch = pitch;
    a.ws = d_w_scales;
    a.M = M;
    a.V = V;
    a.blocks = (D + kBlock - 1) / kBlock;
    a.m_tiles = (M + kRows - 1) / kRows;
    a.box_rows = std::min(kRows, (M + 7) / 8 * 8);
    a.logits = d_logits;
    a.stride = stride;
    a.g = make_grammar(d_mask, mask_rows, d_states, V);
    const int nt = M <= 64 ? 128 : 256;
    if (!make_map(&a.map_w, d_w, V, D, nt) || !make_map(&a.map_q, d_q, M, D, a.box_rows))
        return set_error(TRIE_ECUDA, "cuTensorMapEncodeTiled failed");
    const int64_t grid = (int64_t(V) + nt - 1) / nt * a.m_tiles;
    if (grid > 0x7FFFFFFF) return set_error(TRIE_EINVAL, "M x V is too large");
    const bool f32 = dtype == TRIE_DTYPE_F32;
    const cudaError_t e = nt == 128 ? (f32 ? launch_head<float, 128>(a, grid, stream) : launch_head<__nv_bfloat16, 128>(a, grid, stream))
                                    : (f32 ? launch_head<float, 256>(a, grid, stream) : launch_head<__nv_bfloat16, 256>(a, grid, stream));
    if (e != cudaSuccess) return fail_launch(e, "head launch");
    return TRIE_OK;
}
