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
//  k_head_rows             with a grammar: the logits of rows that allow few tokens.
//  k_head_logits           the product on the tensor cores.
//
// What bounds it (bf16 hidden states and logits, quantization included; times of
// calls that follow one another).
//   1 row, V 32,000, D 2,048: 17 us, 3.9 TB/s of weights; three launch latencies
//     and the ring's first fill are about half of it.
//   64 rows, V 128,000, D 4,096: 93 us, 5.8 TB/s; V 128,011: 102, rows that start
//     at any two bytes are written through shared memory.
//   256 rows, V 152,064, D 4,096: 148 to 165 us by the box, 4.3 to 4.7 TB/s and 1.94
//     to 2.15 PFLOP/s. Nothing is full (HBM 57 %, tensor pipe 48 %, issue slots 60 %): the
//     epilogue waits for each block's sums from tensor memory before it scales them.
//   1,000 rows, V 128,000, D 4,112, f32: 549 to 567 us, 1.9 PFLOP/s: the same.
//   256 constrained rows (15 tokens each), V 152,064, D 4,096: 35 us, most of it -inf
//     written to 78 MB behind a chain of waits (mask, list, weights).
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
    // Whole blocks on 16-byte boundaries are read once, 16 bytes at a time, and held:
    // 152,064 x 4,096 in bf16 360 us (1.87 GB at 5.2 TB/s), by elements 1,110.
    constexpr int kVec = 16 / int(sizeof(T)), kAcross = kBlock / kVec, kSteps = kBlock * kAcross / kQuantThreads;
    const bool wide = (vb + 1) * int64_t(kBlock) <= V && (kb + 1) * kBlock <= D && D % 8 == 0 &&
                      ((reinterpret_cast<uintptr_t>(w) | uintptr_t(stride * int64_t(sizeof(T)))) & 15) == 0 &&
                      (reinterpret_cast<uintptr_t>(q) & 7) == 0;
    const int64_t row = int64_t(vb) * kBlock + threadIdx.x / kAcross;
    const int32_t column = kb * kBlock + int32_t(threadIdx.x % kAcross) * kVec;
    union Piece {
        uint4 raw;
        T x[kVec];
        __device__ Piece() {}
    } held[kSteps];
    float amax = 0.0f;
    if (wide) {
#pragma unroll
        for (int i = 0; i < kSteps; i++)
            held[i].raw = __ldg(reinterpret_cast<const uint4 *>(w + (row + i * (kQuantThreads / kAcross)) * stride + column));
#pragma unroll
        for (int i = 0; i < kSteps; i++)
#pragma unroll
            for (int e = 0; e < kVec; e++) amax = fmaxf(amax, fabsf(to_f32(held[i].x[e])));
    } else {
        for (int r = threadIdx.x / kBlock; r < kBlock; r += kQuantThreads / kBlock) {
            const int64_t v = int64_t(vb) * kBlock + r;
            if (v < V && k < D) amax = fmaxf(amax, fabsf(to_f32(w[v * stride + k])));
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, d));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = amax;
    __syncthreads();
    for (int i = 0; i < kQuantThreads / 32; i++) amax = fmaxf(amax, part[i]);
    const float s = scale_of(amax);
    if (wide) {
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            uint32_t out[2] = {0u, 0u};
#pragma unroll
            for (int e = 0; e < kVec; e++) out[e / 4] |= uint32_t(to_e4m3(__fdiv_rn(to_f32(held[i].x[e]), s))) << (e % 4 * 8);
            uint8_t *to = q + (row + i * (kQuantThreads / kAcross)) * D + column;
            if (kVec == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(out[0], out[1]);
            else *reinterpret_cast<uint32_t *>(to) = out[0];
        }
    } else {
        for (int r = threadIdx.x / kBlock; r < kBlock; r += kQuantThreads / kBlock) {
            const int64_t v = int64_t(vb) * kBlock + r;
            if (v < V && k < D) q[v * D + k] = to_e4m3(__fdiv_rn(to_f32(w[v * stride + k]), s));
        }
    }
    if (threadIdx.x == 0) scales[int64_t(vb) * blocks + kb] = s;
}

// ---- the product
//
// A tile is 128 rows of the batch, the MMA's rows, by 128 tokens, its columns,
// on one CTA; or, for more than 128 rows, 256 by 256 on a pair of CTAs, whose
// MMA reads each CTA's half of either operand, so that a CTA loads 32 KB for
// twice the products (what limits larger batches is the 64 bytes a cycle that
// an SM takes in): 192 rows, V 128,000, D 4,096 126 us on pairs and 169 on single
// CTAs, 256 rows, V 152,064 148 and 195; but 128 rows, V 128,000 123 and 99,
// where half of a pair's rows would be nobody's. Either way a thread of the epilogue holds one row, and the
// scale of a block is one number for it and the 64 or 128 tokens that it has.
// CTAs stay and go over the tiles: one thread streams blocks of 128 columns of
// K of both operands into a ring of stages by TMA, one issues a block's four
// MMAs into one of several accumulators in tensor memory, and the epilogue
// warps read each block's sums out and add them, scaled, to sums in registers,
// so that the next tile's weights arrive while this one's logits are written.
// Rows that a batch does not have are not loaded (the MMA multiplies what lies
// there into rows nobody reads).
constexpr int kRows = 128;         // of a CTA's tile
constexpr int kMaxStages = 8;
constexpr int kColumns = 64;       // tokens of an epilogue warp
constexpr int kHeadSmem = 226 * 1024;
constexpr int kFewMaxD = 32768;    // longest hidden state whose row fits k_head_rows' shared memory
constexpr int kNeedTiles = 2048;   // tiles of a CTA whose need is looked up ahead
constexpr int kLookRows = 16384;   // largest batch of which every CTA looks whether a row is left to it (64 KB)
constexpr int kScaleSlots = 8;     // of two blocks' scales: more blocks than can be between the copies and the epilogue
constexpr int kTurn = 32 * 17;     // words of a warp's block of 16 tokens, turned

struct HeadArgs {
    CUtensorMap map_w, map_q;
    const uint8_t *q, *w;  // [M][D], [V][D]
    const float *s;        // [blocks][pitch]
    int64_t pitch;
    const float *ws;       // [ceil(V / 128)][blocks]
    int32_t M, V, D, blocks;
    int32_t m_tiles;       // of 128 rows (a pair: 256)
    int32_t tiles;
    int32_t box_rows;      // rows of a CTA's tile that are loaded
    int32_t stages;        // of the ring
    void *logits;
    int64_t stride;
    Grammar g;
    // with a grammar, of each row (k_head_rows):
    int32_t *dense;        // [M] 0: k_head_rows wrote its logits, 1: k_head_logits does
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
static_assert(kFew <= kRowThreads, "a thread writes a logit");

// Sum of 16 products of e4m3 numbers (exact in 32 bits but for the additions).
__device__ __forceinline__ float dot16(const uint4 &x, const uint4 &w) {
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ws[4] = {w.x, w.y, w.z, w.w};
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(xs[i] >> (16 * h)), __NV_E4M3);
            const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2(__nv_fp8x2_storage_t(ws[i] >> (16 * h)), __NV_E4M3);
            const float2 fa = __half22float2(__half2(a)), fb = __half22float2(__half2(b));
            sum = fmaf(fa.x, fb.x, sum);
            sum = fmaf(fa.y, fb.y, sum);
        }
    }
    return sum;
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads, 2) k_head_rows(HeadArgs a) {
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
    constexpr int kBatch = 8;  // reads in flight a thread
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
    for (int32_t i = warp; i < n; i += kRowThreads / 32)
        for (int32_t c = lane * 128; c < a.D; c += 32 * 128) prefetch_l2(a.w + int64_t(few[i]) * a.D + c);
    float *scales = reinterpret_cast<float *>(dynamic_smem + a.D);
    for (int32_t i = threadIdx.x; i < a.D / 16; i += kRowThreads)
        reinterpret_cast<uint4 *>(dynamic_smem)[i] = __ldg(reinterpret_cast<const uint4 *>(a.q + int64_t(m) * a.D) + i);
    for (int32_t i = threadIdx.x; i < a.blocks; i += kRowThreads) scales[i] = __ldg(a.s + i * a.pitch + m);
    __syncthreads();
    for (int32_t i = warp; i < n; i += kRowThreads / 32) {
        const int32_t v = few[i];
        const uint4 *w = reinterpret_cast<const uint4 *>(a.w + int64_t(v) * a.D);
        const float *ws = a.ws + int64_t(v / kBlock) * a.blocks;
        float sum = 0.0f;
        for (int32_t c0 = lane; c0 < a.D / 16; c0 += 32 * kBatch) {
            uint4 x[kBatch];
            float f[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; j++) {
                const int32_t c = c0 + 32 * j;
                x[j] = c < a.D / 16 ? __ldg(w + c) : make_uint4(0u, 0u, 0u, 0u);
                f[j] = c < a.D / 16 ? __ldg(ws + c / (kBlock / 16)) : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < kBatch; j++) {
                const int32_t c = c0 + 32 * j;
                if (c < a.D / 16)
                    sum = fmaf(dot16(reinterpret_cast<const uint4 *>(dynamic_smem)[c], x[j]), f[j] * scales[c / (kBlock / 16)], sum);
            }
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
        if (lane == 0) value[i] = sum;
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
__device__ __forceinline__ bool row_uses(const HeadArgs &a, int32_t m, int32_t v0) {
    return (__ldg(a.used + int64_t(m) * a.used_words + (v0 >> 12)) >> ((v0 >> 7) & 31)) & 1u;
}

// The dense rows of [m0, m1) in a tile that none of them allows a token of: -inf.
// By the epilogue warps; NT tokens, fewer at the end.
// (A call, so that its unrolled stores take no registers from the sums of the other tiles.)
template <typename T, int NT, int kWarps>
__device__ __noinline__ void fill_tile(const HeadArgs &a, int32_t m0, int32_t m1, int32_t v0, int warp, int lane) {
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

// 16 tokens from v on of a warp's 32 rows from m on (of which `rows` are there, and
// with kSome those whose bit of `some` is set), a row a thread. Where every row is
// on a 32-byte boundary a thread writes its own 32 bytes at a time; else the block
// is turned in shared memory, so that lanes write consecutive tokens (256 aligned
// rows: 148 and 159 us, 64: 93 and 101). One test more for each store, in kSome
// only, costs 64 unaligned rows 6 us of 101.
template <typename T, bool kSome>
__device__ __forceinline__ void store16(const HeadArgs &a, float *turn, const float *x, int32_t m, int32_t rows, uint32_t some,
                                        int32_t v, int lane, bool wide) {
    T *out = static_cast<T *>(a.logits) + m * a.stride + v;
    if (wide && v + 16 <= a.V) {
        if (lane >= rows || (kSome && !((some >> lane) & 1u))) return;
        T *mine = out + lane * a.stride;
        uint32_t r[8];
        if (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const __nv_bfloat162 both = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                r[i] = *reinterpret_cast<const uint32_t *>(&both);
            }
            store32(mine, r);
        } else {
#pragma unroll
            for (int h = 0; h < 2; h++) {
#pragma unroll
                for (int i = 0; i < 8; i++) r[i] = __float_as_uint(x[8 * h + i]);
                store32(mine + 8 * h, r);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; i++) turn[lane * 17 + i] = x[i];
    __syncwarp();
    const int c = lane & 15;
    if (v + c < a.V)
        for (int r = lane >> 4; r < rows; r += 2)
            if (!kSome || ((some >> r) & 1u)) out[r * a.stride + c] = from_f32<T>(turn[r * 17 + c]);
    __syncwarp();
}

// Epilogue warps: four quarters of the rows, two or four columns of tokens.
template <bool kPair>
constexpr int kEpilogueWarps = kPair ? 16 : 8;
// The warps before them: one for the copies, one for the MMAs, and for a pair two
// more that make up a warpgroup, which leaves registers to the epilogue: launched
// with 96 a thread (640 threads), 128 threads keep 32 and 512 get 112.
template <bool kPair>
constexpr int kFirstWarp = kPair ? 4 : 2;
template <bool kPair>
constexpr int kHeadThreads = 32 * (kFirstWarp<kPair> + kEpilogueWarps<kPair>);

template <typename T, bool kPair>
__global__ void __launch_bounds__(kHeadThreads<kPair>, 1) k_head_logits(const __grid_constant__ HeadArgs a) {
    constexpr int NT = kPair ? 256 : 128;          // tokens of a tile
    constexpr int kAccumulators = 512 / NT;
    constexpr int kEpilogue = kEpilogueWarps<kPair>, kFirst = kFirstWarp<kPair>;
    constexpr int kCtas = kPair ? 2 : 1;
    constexpr int kWeightBytes = 128 * kBlock;     // a CTA's part of the weights of a block
    extern __shared__ unsigned char dynamic_smem[];
    __shared__ uint64_t bars[2 * kMaxStages + 2 * kAccumulators + 2 * kScaleSlots];
    __shared__ __align__(16) float scales[kScaleSlots][2][kRows];
    __shared__ float turn[kEpilogue][kTurn];
    __shared__ uint32_t need[kNeedTiles / 32];
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up;
    const int warp = __shfl_sync(~0u, int(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = kPair ? int(cluster_rank()) : 0;
    const int32_t unit = int32_t(blockIdx.x) / kCtas, units = int32_t(gridDim.x) / kCtas;
    const uint32_t full = smem_addr(bars), empty = full + 8 * kMaxStages;
    const uint32_t ready = empty + 8 * kMaxStages, drained = ready + 8 * kAccumulators;
    const uint32_t s_full = drained + 8 * kAccumulators, s_empty = s_full + 8 * kScaleSlots;
    const uint32_t stages = (smem_addr(dynamic_smem) + 1023u) & ~1023u, stage_bytes = uint32_t(kWeightBytes + a.box_rows * kBlock);
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int i = 0; i < a.stages; i++) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < kAccumulators; i++) {
            bar_init(ready + 8 * i, 1);
            bar_init(drained + 8 * i, kEpilogue * kCtas);
        }
        for (int i = 0; i < kScaleSlots; i++) {
            bar_init(s_full + 8 * i, 1);
            bar_init(s_empty + 8 * i, kEpilogue);
        }
        bar_init_fence();
        tma_prefetch_map(&a.map_w);
        tma_prefetch_map(&a.map_q);
    }
    for (int i = threadIdx.x; i < kNeedTiles / 32; i += kHeadThreads<kPair>) need[i] = 0u;
    pdl_launch_dependents();
    pdl_wait();
    if (a.g.mask && a.M <= kLookRows) {  // k_head_rows may have left nothing to do (the same answer in all CTAs)
        bool any = false;
        for (int32_t m = threadIdx.x; m < a.M; m += kHeadThreads<kPair>) any |= __ldg(a.dense + m) != 0;
        if (!__syncthreads_or(any)) return;
    }
    if (warp == 1) tmem_alloc<kPair>(smem_addr(&tmem_base), 512);
    __syncthreads();
    if (a.g.mask) {
        // which of this CTA's tiles a dense row allows a token of
        for (int32_t i = 0, t = unit; t < a.tiles && i < kNeedTiles; i++, t += units) {
            const int32_t m = t % a.m_tiles * (kRows * kCtas) + int32_t(threadIdx.x), v0 = t / a.m_tiles * NT;
            bool any = false;
            if (threadIdx.x < kRows * kCtas && m < a.M && __ldg(a.dense + m))
                any = row_uses(a, m, v0) || (NT > 128 && v0 + 128 < a.V && row_uses(a, m, v0 + 128));
            if (__any_sync(~0u, any) && lane == 0) atomicOr(&need[i >> 5], 1u << (i & 31));
        }
    }
    tcgen05_fence_before();
    if (kPair) cluster_sync();
    else __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = *static_cast<volatile uint32_t *>(&tmem_base);
    auto needed = [&](int32_t i) { return !a.g.mask || i >= kNeedTiles || ((need[i >> 5] >> (i & 31)) & 1u); };

    if (warp >= kFirst) {
        if (kPair) more_registers<112>();
        const int quarter = warp & 3, column = (warp - kFirst) / 4 * kColumns;
        const uint32_t from = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(column);
        const uint32_t drain = kPair ? cluster_addr(drained, 0) : drained;
        const bool wide = ((reinterpret_cast<uintptr_t>(a.logits) | uintptr_t(a.stride * int64_t(sizeof(T)))) & 31) == 0;
        uint32_t it = 0, slot = 0, slot_phase = 0;
        for (int32_t i = 0, t = unit; t < a.tiles; i++, t += units) {
            const int32_t m0 = t % a.m_tiles * (kRows * kCtas) + rank * kRows, m1 = min(a.M, m0 + kRows);
            const int32_t v0 = t / a.m_tiles * NT, v = v0 + column;
            if (!needed(i)) {
                fill_tile<T, NT, kEpilogue>(a, m0, m1, v0, warp - kFirst, lane);
                continue;
            }
            const int32_t mine = m0 + quarter * 32, row = min(mine + lane, a.M - 1);
            const bool there = mine < m1;  // a warp without rows only keeps the barriers going
            float sum[kColumns];
#pragma unroll
            for (int c = 0; c < kColumns; c++) sum[c] = 0.0f;
            // A block's scales of the rows come through a ring of their own, two blocks at
            // a time; the weights' are read 32 blocks at a time, one a lane. (A read from
            // global memory for each block would have to be many blocks ahead, and an
            // instruction that needs a value on its way, even a move, holds the warp up.)
            const float *wp = a.ws + int64_t(min(v, a.V - 1) / kBlock) * a.blocks;
            float w = __ldg(wp + min(lane, a.blocks - 1));
            auto add_block = [&](int32_t kb, const float *scale_of_rows) {
                const uint32_t acc = it % kAccumulators;
                bar_wait(ready + 8 * acc, (it / kAccumulators) & 1, &gave_up);
                tcgen05_fence_after();
                const float scale = scale_of_rows[quarter * 32 + lane] * __shfl_sync(~0u, w, kb & 31);
                if (there) {
#pragma unroll
                    for (int c = 0; c < kColumns; c += 16) {
                        uint32_t r[16];
                        tmem_load16(from + acc * NT + c, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; e++) sum[c + e] = fmaf(__uint_as_float(r[e]), scale, sum[c + e]);
                    }
                }
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (kPair) bar_arrive_remote(drain + 8 * acc);
                    else bar_arrive(drain + 8 * acc);
                }
                it++;
            };
            for (int32_t kb = 0; kb < a.blocks; kb += 2) {
                bar_wait(s_full + 8 * slot, slot_phase, &gave_up);
                add_block(kb, scales[slot][0]);
                if (kb + 1 < a.blocks) add_block(kb + 1, scales[slot][1]);
                if (lane == 0) bar_arrive(s_empty + 8 * slot);
                if (++slot == kScaleSlots) slot = 0, slot_phase ^= 1;
                if ((kb & 31) == 30 && kb + 2 < a.blocks) w = __ldg(wp + min(kb + 2 + lane, a.blocks - 1));
            }
            const bool ok = *static_cast<volatile int *>(&gave_up) == 0;
            if (!there) continue;
            const GrammarRow allow = grammar_row(a.g, row);
            const int32_t rows = min(32, m1 - mine);
            uint32_t some = ~0u;
            if (a.g.mask) some = __ballot_sync(~0u, __ldg(a.dense + row) != 0);
#pragma unroll
            for (int c = 0; c < kColumns; c += 16) {
                uint32_t bits = ~0u;
                if (a.g.mask) bits = (v + c) >> 5 < a.g.W ? allow.word((v + c) >> 5) >> (c & 16) : 0u;
                if (!ok || (bits & 0xFFFFu) != 0xFFFFu) {
#pragma unroll
                    for (int e = 0; e < 16; e++) {
                        if (!ok) sum[c + e] = __int_as_float(0x7FFFFFFF);  // gave up waiting: no result
                        if (!((bits >> e) & 1u)) sum[c + e] = -INFINITY;
                    }
                }
                if (v + c >= a.V) continue;
                if (some == ~0u) store16<T, false>(a, turn[warp - kFirst], sum + c, mine, rows, some, v + c, lane, wide);
                else store16<T, true>(a, turn[warp - kFirst], sum + c, mine, rows, some, v + c, lane, wide);
            }
        }
    } else {
        if (kPair) fewer_registers<32>();
        if (warp == 0) {
            int stage = 0;
            uint32_t phase = 1, used = 0;  // phase: of a stage's last use; the first time round there is none
            uint32_t it = 0;
            bool ok = true;
            const uint32_t leader = kPair ? cluster_addr(full, 0) : full;
            for (int32_t i = 0, t = unit; t < a.tiles && ok; i++, t += units) {
                if (!needed(i)) continue;
                const int32_t m = t % a.m_tiles * (kRows * kCtas) + rank * kRows, v = t / a.m_tiles * NT + rank * 128;
                // a CTA of a pair without rows takes some others' scales
                const int64_t sm = min(int64_t(m), a.pitch - 4);
                const uint32_t scale_bytes = uint32_t(min(int64_t(kRows), a.pitch - sm)) * 4;
                for (int32_t kb = 0; kb < a.blocks; kb++) {
                    const uint32_t at = stages + uint32_t(stage) * stage_bytes, bar = leader + 8 * stage;
                    const uint32_t slot = it % kScaleSlots, two = kb + 1 < a.blocks ? 2 : 1;
                    ok = bar_wait(empty + 8 * stage, phase, &gave_up);
                    if (!(kb & 1)) ok = ok && bar_wait(s_empty + 8 * slot, ((it / kScaleSlots) & 1) ^ 1, &gave_up);
                    ok = __all_sync(~0u, ok);
                    if (!ok) break;
                    if (elect_one()) {
                        if (!(kb & 1)) {
                            bar_expect(s_full + 8 * slot, scale_bytes * two);
                            for (uint32_t j = 0; j < two; j++)
                                bulk_load(smem_addr(scales[slot][j]), a.s + (kb + j) * a.pitch + sm, scale_bytes, s_full + 8 * slot);
                        }
                        if (kPair) {
                            // both CTAs' copies count on the first one's barrier
                            if (rank == 0) bar_expect(full + 8 * stage, 2 * stage_bytes);
                            tma_load_2d_pair(at, &a.map_w, kb * kBlock, v, bar);
                            tma_load_2d_pair(at + kWeightBytes, &a.map_q, kb * kBlock, m, bar);
                        } else {
                            bar_expect(bar, stage_bytes);
                            tma_load_2d(at, &a.map_w, kb * kBlock, v, bar);
                            tma_load_2d(at + kWeightBytes, &a.map_q, kb * kBlock, m, bar);
                        }
                    }
                    __syncwarp();
                    if (!(kb & 1)) it++;
                    used = min(used + 1, uint32_t(a.stages));
                    if (++stage == a.stages) stage = 0, phase ^= 1;
                }
            }
            if (ok) {  // the last MMAs' arrivals on this CTA's barriers come before it ends
                for (int i = 0; i < a.stages; i++) {
                    bar_wait(empty + 8 * stage, phase, &gave_up);
                    if (++stage == a.stages) stage = 0, phase ^= 1;
                }
            } else {  // copies may still write to shared memory: wait for them
                int none = 0;
                for (uint32_t i = it > kScaleSlots ? it - kScaleSlots : 0; i < it; i++)
                    bar_wait(s_full + 8 * (i % kScaleSlots), (i / kScaleSlots) & 1, &none);
                for (uint32_t i = 0; i < used && rank == 0; i++) {
                    if (--stage < 0) stage = a.stages - 1, phase ^= 1;
                    bar_wait(full + 8 * stage, phase ^ 1, &none);
                }
            }
        } else if (warp == 1) {
            if (rank == 0) {
                constexpr uint32_t idesc = mma_idesc_e4m3(kRows * kCtas, NT);
                int stage = 0;
                uint32_t phase = 0, it = 0;
                bool ok = true;
                for (int32_t i = 0, t = unit; t < a.tiles && ok; i++, t += units) {
                    if (!needed(i)) continue;
                    for (int32_t kb = 0; kb < a.blocks; kb++, it++) {
                        const uint32_t acc = it % kAccumulators;
                        ok = bar_wait(drained + 8 * acc, ((it / kAccumulators) & 1) ^ 1, &gave_up) &&
                             bar_wait(full + 8 * stage, phase, &gave_up);
                        ok = __all_sync(~0u, ok);
                        if (!ok) break;
                        tcgen05_fence_after();
                        const uint32_t at = stages + uint32_t(stage) * stage_bytes;
                        const uint64_t dw = mma_desc(at), dq = mma_desc(at + kWeightBytes);
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kBlock / 32; k++)
                                mma_e4m3<kPair>(tmem + acc * NT, dq + 2 * k, dw + 2 * k, idesc, k > 0);
                            mma_commit<kPair>(empty + 8 * stage);
                            mma_commit<kPair>(ready + 8 * acc);
                        }
                        __syncwarp();
                        if (++stage == a.stages) stage = 0, phase ^= 1;
                    }
                }
            }
        }
    }
    __syncwarp();
    tcgen05_fence_before();
    if (kPair) cluster_sync();
    else __syncthreads();
    tcgen05_fence_after();
    if (warp == 1) tmem_free<kPair>(tmem, 512);
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

template <typename T, bool kPair>
cudaError_t launch_head(HeadArgs a, cudaStream_t st) {
    const int stage = 128 * kBlock + a.box_rows * kBlock;
    // the last stage's MMA reads kRows rows, whatever was loaded; and room to align the ring
    const int beyond = (kRows - a.box_rows) * kBlock + 1024;
    const int fixed = int(sizeof(float)) * (kEpilogueWarps<kPair> * kTurn + kScaleSlots * 2 * kRows) + 1024;  // declared in the kernel
    a.stages = std::min(kMaxStages, (kHeadSmem - fixed - beyond) / stage);
    const int smem = a.stages * stage + beyond;
    const cudaError_t e = cudaFuncSetAttribute(k_head_logits<T, kPair>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadSmem - fixed);
    if (e != cudaSuccess) return e;
    const int ctas = kPair ? 2 : 1, units = std::min(a.tiles, sm_count() / ctas);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(units * ctas));
    cfg.blockDim = dim3(kHeadThreads<kPair>);
    cfg.dynamicSmemBytes = size_t(smem);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(ctas);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kPair ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_head_logits<T, kPair>, a);
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

namespace tmk {
namespace {
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

extern "C" int64_t trie_head_workspace(int32_t M, int32_t V) {
    if (M < 0 || M > (1 << 20) || V < 2 || V > tmk::kMaxV) return -1;
    return tmk::HeadSpace(M, V).bytes;
}

extern "C" int trie_head_logits(const uint8_t *d_q, const float *d_scales, int64_t pitch, const uint8_t *d_w,
                                const float *d_w_scales, int32_t M, int32_t V, int32_t D, void *d_logits, int dtype,
                                int64_t stride, const uint32_t *d_mask, int32_t mask_rows, const int32_t *d_states,
                                void *d_workspace, cudaStream_t stream) {
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
    if (!*bad && M > 0 && d_mask && !d_workspace) bad = "d_mask without d_workspace";
    if (!*bad && (reinterpret_cast<uintptr_t>(d_workspace) & 15)) bad = "d_workspace is not aligned to 16 bytes";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (M == 0) return TRIE_OK;
    HeadArgs a = {};
    a.q = d_q;
    a.w = d_w;
    a.s = d_scales;
    a.pitch = pitch;
    a.ws = d_w_scales;
    a.M = M;
    a.V = V;
    a.D = D;
    a.blocks = (D + kBlock - 1) / kBlock;
    const bool pair = M > kRows;
    const int side = pair ? 256 : 128;  // of a tile
    a.m_tiles = (M + side - 1) / side;
    a.box_rows = std::min(kRows, (M + 7) / 8 * 8);
    a.logits = d_logits;
    a.stride = stride;
    a.g = make_grammar(d_mask, mask_rows, d_states, V);
    if (!make_map(&a.map_w, d_w, V, D, 128) || !make_map(&a.map_q, d_q, M, D, a.box_rows))
        return set_error(TRIE_ECUDA, "cuTensorMapEncodeTiled failed");
    const int64_t tiles = (int64_t(V) + side - 1) / side * a.m_tiles;
    if (tiles > 0x3FFFFFFF) return set_error(TRIE_EINVAL, "M x V is too large");
    a.tiles = int32_t(tiles);
    const bool f32 = dtype == TRIE_DTYPE_F32;
    cudaError_t e;
    if (d_mask) {
        const HeadSpace at(M, V);
        unsigned char *base = static_cast<unsigned char *>(d_workspace);
        a.dense = reinterpret_cast<int32_t *>(base + at.dense);
        a.used = reinterpret_cast<uint32_t *>(base + at.used);
        a.used_words = at.used_words;
        const int smem = D <= kFewMaxD ? D + a.blocks * 4 : 0;
        e = f32 ? launch_pdl_smem(k_head_rows<float>, M, kRowThreads, smem, stream, a)
                : launch_pdl_smem(k_head_rows<__nv_bfloat16>, M, kRowThreads, smem, stream, a);
        if (e != cudaSuccess) return fail_launch(e, "head rows launch");
    }
    e = pair ? (f32 ? launch_head<float, true>(a, stream) : launch_head<__nv_bfloat16, true>(a, stream))
             : (f32 ? launch_head<float, false>(a, stream) : launch_head<__nv_bfloat16, false>(a, stream));
    if (e != cudaSuccess) return fail_launch(e, "head launch");
    return TRIE_OK;
}
