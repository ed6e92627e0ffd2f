// What the logits heads (head.cu, head4.cu) share: the rows of a batch that allow
// few tokens, the parts of a tile's epilogue, and the maps of their operands.
#pragma once

#include <math.h>
#include <stdint.h>

#include <cuda_runtime.h>

#include "blackwell.cuh"
#include "quantize.cuh"

namespace tmk {

namespace {

constexpr int kRows = 128;         // of a CTA's tile
constexpr int kMaxStages = 8;
constexpr int kColumns = 64;       // tokens of an epilogue warp
constexpr int kHeadSmem = 226 * 1024;
constexpr int kFewMaxD = 32768;    // longest hidden state whose row fits k_head_rows' shared memory
constexpr int kNeedTiles = 2048;   // tiles of a CTA whose need is looked up ahead
constexpr int kLookRows = 16384;   // largest batch of which every CTA looks whether a row is left to it (64 KB)

struct HeadOut {
    int32_t M, V, D;
    void *logits;
    int64_t stride;
    Grammar g;
    // with a grammar, of each row (k_head_rows):
    int32_t *dense;        // [M] 0: k_head_rows wrote its logits, 1: the tiles' kernel does
    uint32_t *used;        // [M][used_words] bit i: it allows one of tokens 128 i .. 128 i + 127
    int32_t used_words;
};

// ---- rows that allow few tokens
//
// A trie's nodes allow a handful of tokens, so a constrained row's logits are a
// few dot products of its hidden state with rows of the weights that are
// scattered over the vocabulary: reading whole tiles of weights for them would
// cost hundreds of times more. A CTA per row counts the row's allowed tokens;
// where they are at most kFew (and the batch has no free row nearby, whose
// tiles are multiplied anyway) it computes their logits, a warp a token, while
// other warps write -inf over the row, and writes them last: the tiles' kernel
// leaves such a row out. 256 constrained rows, V 152,064, D 4,096: 35 us, and 173
// by tiles. A longer list than kFew would be as much to read, scattered, as tiles are.
constexpr int kFew = 256;
constexpr int kNear = 256;         // rows among which one free row makes all dense
constexpr int kRowThreads = 512;
constexpr int kBatch = 8;          // reads in flight a thread
static_assert(kFew <= kRowThreads, "a thread writes a logit");

// A head's own part, for its arguments `Args`:
//   few_load(a, m, smem)   row m's values and scales into shared memory, by the CTA
//   few_ask(a, v, lane)    token v's weights into L2, by a warp
//   few_part(a, v, smem, lane)   a lane's part of the row's product with them
//   few_logit(a, m, v, sum)      the logit from the sum of the parts
template <typename T, typename Args>
__global__ void __launch_bounds__(kRowThreads, 2) k_head_rows(Args a) {
    extern __shared__ __align__(16) unsigned char dynamic_smem[];  // the row's values, then its scales
    __shared__ int32_t few[kFew];
    __shared__ float value[kFew];
    __shared__ int32_t n_few, pieces;
    pdl_launch_dependents();
    if (threadIdx.x == 0) n_few = pieces = 0;
    __syncthreads();
    pdl_wait();
    const int32_t m = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const GrammarRow row = grammar_row(a.g, m);
    const int32_t first = m / kNear * kNear, near = first + int32_t(threadIdx.x);
    const bool free_near = threadIdx.x < kNear && near < a.M && grammar_row(a.g, near).kind == kAllowAll;
    uint8_t *used = reinterpret_cast<uint8_t *>(a.used + int64_t(m) * a.used_words);
    const int32_t W = int32_t(a.g.W), all = a.used_words * 128;  // words of the mask, of which four make a bit of `used`
    for (int32_t w0 = int32_t(threadIdx.x); w0 - lane < all; w0 += kBatch * kRowThreads) {
        uint32_t word[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; i++) {
            const int32_t w = w0 + i * kRowThreads;
            word[i] = w < W ? row.word(w) : 0u;
            if (w == W - 1 && a.V & 31) word[i] &= (1u << (a.V & 31)) - 1u;  // bits past V are nobody's
        }
#pragma unroll
        for (int i = 0; i < kBatch; i++) {
            const int32_t w = w0 + i * kRowThreads;
            const uint32_t any = __ballot_sync(~0u, word[i] != 0u);
            uint32_t bits = 0;
#pragma unroll
            for (int b = 0; b < 8; b++) bits |= uint32_t(((any >> (4 * b)) & 15u) != 0u) << b;
            if (lane == 0 && w < all) used[w / 32] = uint8_t(bits);
            if (word[i]) {
                int32_t at = atomicAdd(&n_few, __popc(word[i]));
                for (uint32_t x = word[i]; x && at < kFew; x &= x - 1) few[at++] = w * 32 + __ffs(x) - 1;
            }
        }
    }
    const bool dense = __syncthreads_or(free_near);
    const int32_t n = n_few;
    if (row.kind == kAllowAll || dense || n > kFew || a.D > kFewMaxD) {
        if (threadIdx.x == 0) a.dense[m] = 1;
        return;
    }
    if (threadIdx.x == 0) a.dense[m] = 0;
    for (int32_t i = warp; i < n; i += kRowThreads / 32) few_ask(a, few[i], lane);
    few_load(a, m, dynamic_smem);
    __syncthreads();
    for (int32_t i = warp; i < n; i += kRowThreads / 32) {
        float sum = few_part(a, few[i], dynamic_smem, lane);
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
        if (lane == 0) value[i] = few_logit(a, m, few[i], sum);
    }
    // -inf: to a 16-byte boundary, 16 bytes at a time, and the rest; warps without
    // a token (most of them) come first and take most pieces
    T *out = static_cast<T *>(a.logits) + m * a.stride;
    constexpr int kVec = 16 / int(sizeof(T)), kPiece = 8 * 32;
    const int32_t ahead = int32_t((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / int32_t(sizeof(T)), head = min(ahead, a.V);
    const int32_t body = (a.V - head) / kVec, tail = head + body * kVec;
    const uint32_t pair = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    if (int32_t(threadIdx.x) < head) out[threadIdx.x] = from_f32<T>(-INFINITY);
    if (tail + int32_t(threadIdx.x) < a.V) out[tail + threadIdx.x] = from_f32<T>(-INFINITY);
    for (;;) {
        int32_t piece = lane == 0 ? atomicAdd(&pieces, 1) : 0;
        piece = __shfl_sync(~0u, piece, 0);
        if (piece > body / kPiece) break;
#pragma unroll
        for (int i = 0; i < kPiece / 32; i++) {
            const int32_t at = piece * kPiece + i * 32 + lane;
            if (at < body) reinterpret_cast<uint4 *>(out + head)[at] = make_uint4(pair, pair, pair, pair);
        }
    }
    __syncthreads();
    if (int32_t(threadIdx.x) < n) out[few[threadIdx.x]] = from_f32<T>(value[threadIdx.x]);
}

// Whether row m allows a token of tokens v0 .. v0 + 127 (v0 a multiple of 128).
__device__ __forceinline__ bool row_uses(const HeadOut &a, int32_t m, int32_t v0) {
    return (__ldg(a.used + int64_t(m) * a.used_words + (v0 >> 12)) >> ((v0 >> 7) & 31)) & 1u;
}

// The dense rows of [m0, m1) in a tile that none of them allows a token of: -inf.
// By the epilogue warps; NT tokens, fewer at the end.
// (A call, so that its unrolled stores take no registers from the sums of the other tiles.)
template <typename T, int NT, int kWarps>
__device__ __noinline__ void fill_tile(const HeadOut &a, int32_t m0, int32_t m1, int32_t v0, int warp, int lane) {
    constexpr int kVec = 16 / int(sizeof(T)), kEach = kRows / kWarps;
    const int32_t v1 = min(a.V, v0 + NT);
    const uint32_t pair = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    const int32_t mine = m0 + warp + lane * kWarps;  // a lane a row
    const uint32_t dense = __ballot_sync(~0u, lane < kEach && mine < m1 && __ldg(a.dense + mine));
#pragma unroll 4
    for (int j = 0; j < kEach; j++) {
        if (!((dense >> j) & 1u)) continue;
        T *out = static_cast<T *>(a.logits) + (m0 + warp + j * kWarps) * a.stride + v0;
        if (v1 - v0 == NT && (reinterpret_cast<uintptr_t>(out) & 15) == 0) {
#pragma unroll
            for (int i = 0; i < NT / kVec; i += 32)
                if (i + lane < NT / kVec) reinterpret_cast<uint4 *>(out)[i + lane] = make_uint4(pair, pair, pair, pair);
        } else {
            for (int32_t i = lane; i < v1 - v0; i += 32) out[i] = from_f32<T>(-INFINITY);
        }
    }
}

// cuTensorMapEncodeTiled, NULL where the driver has none.
using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                            const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                            CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline Encode tensor_map_encode() {
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
    return encode;
}
// [rows][bytes] in boxes of box_rows x 128, 128-byte swizzle, zeros outside.
inline bool make_map(CUtensorMap *map, const void *base, int64_t rows, int64_t bytes, int32_t box_rows) {
    const Encode encode = tensor_map_encode();
    if (!encode) return false;
    const cuuint64_t dims[2] = {cuuint64_t(bytes), cuuint64_t(rows)}, strides[1] = {cuuint64_t(bytes)};
    const cuuint32_t box[2] = {128u, cuuint32_t(box_rows)}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Where the parts of the workspace lie.
struct HeadSpace {
    int32_t used_words;
    int64_t dense, used, bytes;
    HeadSpace(int32_t M, int32_t V) {
        used_words = int32_t((int64_t(V) + 4095) / 4096);
        dense = 0;
        used = (int64_t(M) * 4 + 15) / 16 * 16;
        bytes = used + int64_t(M) * used_words * 4;
    }
};

}  // namespace

}  // namespace tmk
