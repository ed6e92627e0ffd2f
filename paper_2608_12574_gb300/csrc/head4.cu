// The logits head in microscaled 4-bit floating point, under a grammar:
// trie_head4_logits.
//
//   logit[m, v] = S[m] T[v] sum_b s[m, b] t[v, b] sum_{k in block b} q[m, k] w[v, k]
// and -inf where row m's state does not allow token v: q and w in e2m1, s and t
// in e4m3 for 16 columns of a row, S and T in 32 bits for a row (quantize.cuh).
// Sums are kept in 32 bits and rounded once to the logits' type.
//
//  k_head_rows   with a grammar: the logits of rows that allow few tokens.
//  k_head4       the product on the tensor cores.
//
// What bounds it (bf16 unless said; quantization included; times of calls that follow one another).
//   1 row, V 32,000, D 2,048: 10 us, 3.7 TB/s of weights, of it two launches and the ring's first fill.
//   128 rows, V 152,064, D 4,096: 63 us, 5.9 TB/s; 512 rows 116 us, 5.5 PFLOP/s.
//   256 rows, V 152,064, D 4,096: 73 us, 5.9 TB/s, with the norm in front 75: HBM, whose reads are 128
//     bytes of each of 128 rows at a time.
//   256 rows of which half are constrained: 90 us, all in tiles.
//   1,000 rows, V 128,000, D 4,096: 181 to 190 us, 5.5 PFLOP/s and more, f32 212; the MMAs alone take 120 (8-bit head: 463).
//     V 128,011, whose rows of logits start at any two or four bytes: 193, f32 219.
//   D 4,112, whose rows of codes start off 128-byte lines, so that a stage's 128 bytes of a row are parts of two:
//     128 rows, V 128,000, 77 us; 1,000 rows 259, f32 314; V 128,011 261 to 270, f32 309 to 335.
//   256 constrained rows (15 tokens each), V 152,064, D 4,096, with the norm: 45 us, -inf to 78 MB behind a
//     chain of waits, in which a token's scales are 64 sectors of their own.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>

#include <cuda_runtime.h>

#include "head_tile.cuh"

namespace tmk {

namespace {

// ---- the product
//
// Tiles and the ring are as in head.cu: rows of the batch are the MMA's rows, 128
// x 128 on a CTA up to 128 rows of the batch, 256 x 256 on a pair of CTAs beyond.
// The tensor core applies the blocks' scales itself, so an accumulator takes the
// whole of K and is read out once a tile: the epilogue holds its 64 tokens a
// thread in registers and gives the accumulator back before it scales and stores
// them. A stage is 256 columns, four MMAs deep: 128 bytes of a row of either
// operand, and 512 bytes of scales for 128 rows and 64 columns, which the
// MMAs' thread copies from shared to tensor memory in front of them (copies and
// MMAs of a thread are carried out in order).
// Every CTA loads what its tiles read by itself, the scales of all of a pair's tokens too. (Loads
// into several CTAs at once, by multicast, took 185 us instead of 181 at D 4,096 and 205 instead of 259 at D 4,112
// for 1,000 rows; they are for programs on one GPU alone, and ranks on several load this library.)
constexpr int kStageColumns = 256;
constexpr int kSteps = kStageColumns / 64;  // MMAs of a stage
constexpr int kAskFirst = 256 * 1024, kAskPiece = 16 * 1024;  // bytes of its first tile that a CTA asks for ahead; at a time
constexpr int kScaleTile = 512;             // bytes of the scales of 128 rows x 64 columns

template <bool kPair>
constexpr int kTokens = kPair ? 256 : 128;  // of a tile
template <bool kPair>
constexpr int kWeightBytes4 = 128 * 128 + kTokens<kPair> / 128 * kSteps * kScaleTile;  // of a stage of a CTA: its 128 rows, all scales
constexpr int kHiddenScales = kSteps * kScaleTile;
template <bool kPair>
constexpr int kEpilogueWarps4 = kPair ? 16 : 8;
// The warps before them: as in head.cu.
template <bool kPair>
constexpr int kFirstWarp4 = kPair ? 4 : 2;
template <bool kPair>
constexpr int kThreads4 = 32 * (kFirstWarp4<kPair> + kEpilogueWarps4<kPair>);

struct Head4Args : HeadOut {
    CUtensorMap map_w, map_q, map_ws, map_s;
    const uint8_t *q, *w, *s, *ws;
    const float *q_rows, *w_rows;
    int64_t row_bytes, tiles_k;  // of a row's codes; 64-column tiles of its scales
    int32_t blocks;              // stages of K
    int32_t m_tiles, tiles, box_rows, stages;  // as in HeadArgs
};

// Sum of 32 products and their blocks' scales. e2m1 products are multiples of 1/4 up to 36,
// so eight of them add up exactly in 16 bits.
__device__ __forceinline__ float dot32(const uint4 &x, const uint4 &w, const float *xs, uint32_t ws) {
    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, ww[4] = {w.x, w.y, w.z, w.w};
    float sum = 0.0f;
#pragma unroll
    for (int b = 0; b < 2; b++) {
        __half2 part = __float2half2_rn(0.0f);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const __half2 p(__nv_cvt_fp4x2_to_halfraw2(__nv_fp4x2_storage_t(xw[2 * b + i / 4] >> (i % 4 * 8)), __NV_E2M1));
            const __half2 r(__nv_cvt_fp4x2_to_halfraw2(__nv_fp4x2_storage_t(ww[2 * b + i / 4] >> (i % 4 * 8)), __NV_E2M1));
            part = __hfma2(p, r, part);
        }
        sum = fmaf(__low2float(part) + __high2float(part), xs[b] * from_e4m3(uint8_t(ws >> (8 * b))), sum);
    }
    return sum;
}
__device__ __forceinline__ void few_load(const Head4Args &a, int32_t m, unsigned char *smem) {
    float *scales = reinterpret_cast<float *>(smem + a.row_bytes);
    for (int32_t i = threadIdx.x; i < a.row_bytes / 16; i += kRowThreads)
        reinterpret_cast<uint4 *>(smem)[i] = __ldg(reinterpret_cast<const uint4 *>(a.q + m * a.row_bytes) + i);
    for (int32_t i = threadIdx.x; i < a.row_bytes / 8; i += kRowThreads)
        scales[i] = from_e4m3(__ldg(a.s + scale_word4(m, i / 4, a.tiles_k) + i % 4));
}
__device__ __forceinline__ void few_ask(const Head4Args &a, int32_t v, int lane) {
    for (int32_t c = lane * 128; c < a.row_bytes; c += 32 * 128) prefetch_l2(a.w + v * a.row_bytes + c);
    for (int32_t t = lane; t < a.tiles_k; t += 32) prefetch_l2(a.ws + scale_word4(v, t, a.tiles_k));
}
__device__ __forceinline__ float few_part(const Head4Args &a, int32_t v, const unsigned char *smem, int lane) {
    const float *scales = reinterpret_cast<const float *>(smem + a.row_bytes);
    const uint4 *w = reinterpret_cast<const uint4 *>(a.w + v * a.row_bytes);
    const int32_t n = int32_t(a.row_bytes / 16);
    float sum = 0.0f;
    for (int32_t c0 = lane; c0 < n; c0 += 32 * kBatch) {
        uint4 x[kBatch];
        uint32_t f[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; j++) {
            const int32_t c = c0 + 32 * j;
            x[j] = c < n ? __ldg(w + c) : make_uint4(0u, 0u, 0u, 0u);
            f[j] = c < n ? __ldg(reinterpret_cast<const uint16_t *>(a.ws + scale_word4(v, c / 2, a.tiles_k) + (c & 1) * 2)) : 0u;
        }
#pragma unroll
        for (int j = 0; j < kBatch; j++) {
            const int32_t c = c0 + 32 * j;
            if (c < n) sum += dot32(reinterpret_cast<const uint4 *>(smem)[c], x[j], scales + 2 * c, f[j]);
        }
    }
    return sum;
}
__device__ __forceinline__ float few_logit(const Head4Args &a, int32_t m, int32_t v, float sum) {
    return sum * __ldg(a.q_rows + m) * __ldg(a.w_rows + v);
}

// 16 tokens from v on of a warp's 32 rows from m on (of which `rows` are there, and
// the bit of `some` is set), a row a thread, 32 bytes at a time.
template <typename T, bool kWide>
__device__ __forceinline__ void store16(const HeadOut &a, const float *x, int32_t m, int32_t rows, uint32_t some, int32_t v, int lane) {
    if (lane >= rows || !((some >> lane) & 1u)) return;
    T *mine = static_cast<T *>(a.logits) + (m + lane) * a.stride + v;
    if (v + 16 > a.V || !kWide) {
#pragma unroll
        for (int e = 0; e < 16; e++)
            if (v + e < a.V) mine[e] = from_f32<T>(x[e]);
        return;
    }
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
}

// The same for rows that do not all start on 32-byte boundaries, 64 tokens of a row a thread: shifted, so that whole 32
// bytes that lie on such a boundary are written at once; those that reach into the next 64 tokens too, by the thread
// that has the first of them, where it reads the others (`next`). 1,000 rows, V 128,011, D 4,096: f32 219 us, bf16
// 193; 250 and 222 without `next`, so that both sides' threads write a part. (Turned in shared memory, a row an instruction,
// some 44 more than with it, at D 4,112.)
template <typename T>
struct Shifted {
    static constexpr int kPieces = kColumns * int(sizeof(T)) / 32;
    char *at;              // where the next 32 bytes go
    uint32_t ahead;        // bytes before the first of them
    bool there, head, next;
    uint32_t kept[8];
    // head: whether the bytes ahead are this thread's
    __device__ __forceinline__ Shifted(const HeadOut &a, int32_t m, int32_t v, bool there, bool head, bool next) : there(there), head(head), next(next) {
        at = reinterpret_cast<char *>(static_cast<T *>(a.logits) + m * a.stride + v);
        ahead = uint32_t(32 - (reinterpret_cast<uintptr_t>(at) & 31)) & 31u;
        at += ahead;
    }
    // x behind the bytes ahead (15 words of it)
    __device__ __forceinline__ void shift(uint32_t (&x)[16]) const {
        if (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 16; i++) x[i] = ahead & 2u ? __funnelshift_r(x[i], i < 15 ? x[i + 1] : 0u, 16) : x[i];
        }
#pragma unroll
        for (int d = 1; d <= 4; d *= 2)
#pragma unroll
            for (int i = 0; i + d < 16; i++) x[i] = ahead & (4u * d) ? x[i + d] : x[i];
    }
    // The next eight words, number `piece` of kPieces.
    __device__ __forceinline__ void put(const uint32_t *w, int piece) {
        if (piece > 0) {
            uint32_t x[16];
#pragma unroll
            for (int i = 0; i < 16; i++) x[i] = i < 8 ? kept[i] : w[i - 8];
            shift(x);
            if (there) store_words(at, x, 8);
            at += 32;
            if (piece == kPieces - 1 && there && !next) {
                if (ahead == 0u) store_words(at, x + 8, 8);
                else store_few(at, x + 8, 32u - ahead);
            }
        } else if (head && there) {
            // `ahead` bytes, up to a boundary, so the smallest first
            uint32_t x[8];
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = w[i];
            if (sizeof(T) == 2 && (ahead & 2u)) {
                *reinterpret_cast<uint16_t *>(at - ahead) = uint16_t(x[0]);
#pragma unroll
                for (int i = 0; i < 8; i++) x[i] = __funnelshift_r(x[i], i < 7 ? x[i + 1] : 0u, 16);
            }
#pragma unroll
            for (int d = 1; d <= 4; d *= 2)
                if (ahead & (4u * d)) {
                    store_words(at - (ahead & ~(4u * d - 1u)), x, d);
#pragma unroll
                    for (int i = 0; i + d < 8; i++) x[i] = x[i + d];
                }
        }
#pragma unroll
        for (int i = 0; i < 8; i++) kept[i] = w[i];
    }
    // `bytes` < 32 from a boundary on, so the largest first.
    __device__ __forceinline__ static void store_few(char *to, uint32_t *x, uint32_t bytes) {
#pragma unroll
        for (int d = 4; d >= 1; d /= 2)
            if (bytes & (4u * d)) {
                store_words(to, x, d);
                to += 4 * d;
#pragma unroll
                for (int i = 0; i + d < 8; i++) x[i] = x[i + d];
            }
        if (sizeof(T) == 2 && (bytes & 2u)) *reinterpret_cast<uint16_t *>(to) = uint16_t(x[0]);
    }
    __device__ __forceinline__ static void store_words(char *to, const uint32_t *x, int n) {
        if (n == 8) {
            const uint32_t r[8] = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
            store32(to, r);
        } else if (n == 4) {
            *reinterpret_cast<uint4 *>(to) = make_uint4(x[0], x[1], x[2], x[3]);
        } else if (n == 2) {
            *reinterpret_cast<uint2 *>(to) = make_uint2(x[0], x[1]);
        } else {
            *reinterpret_cast<uint32_t *>(to) = x[0];
        }
    }
};

template <typename T, bool kPair, bool kWide>
__global__ void __launch_bounds__(kThreads4<kPair>, 1) k_head4(const __grid_constant__ Head4Args a) {
    constexpr int NT = kTokens<kPair>;
    constexpr int kAccumulators = 256 / NT;  // the other 256 columns of tensor memory are for scales
    constexpr int kEpilogue = kEpilogueWarps4<kPair>, kFirst = kFirstWarp4<kPair>;
    constexpr int kCtas = kPair ? 2 : 1;
    constexpr uint32_t kHiddenColumns = kSteps * 4, kSlotColumns = 64;  // of a stage's scales in tensor memory
    static_assert(kHiddenColumns + kSteps * NT / 32 <= kSlotColumns, "a stage's scales fit a slot");
    extern __shared__ unsigned char dynamic_smem[];
    __shared__ uint64_t bars[2 * kMaxStages + 2 * kAccumulators];
    __shared__ __align__(16) float token_scales[kEpilogue][kColumns + 16];  // and of the 16 tokens behind its own
    __shared__ uint32_t need[kNeedTiles / 32];
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up;
    const int warp = __shfl_sync(~0u, int(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = kPair ? int(cluster_rank()) : 0;
    const int32_t unit = int32_t(blockIdx.x) / kCtas, units = int32_t(gridDim.x) / kCtas;
    const uint32_t full = smem_addr(bars), empty = full + 8 * kMaxStages;
    const uint32_t ready = empty + 8 * kMaxStages, drained = ready + 8 * kAccumulators;
    const uint32_t stages = (smem_addr(dynamic_smem) + 1023u) & ~1023u;
    const uint32_t stage_bytes = uint32_t(kWeightBytes4<kPair> + kHiddenScales + a.box_rows * 128);
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
        bar_init_fence();
        tma_prefetch_map(&a.map_w);
        tma_prefetch_map(&a.map_q);
        tma_prefetch_map(&a.map_ws);
        tma_prefetch_map(&a.map_s);
    }
    for (int i = threadIdx.x; i < kNeedTiles / 32; i += kThreads4<kPair>) need[i] = 0u;
    pdl_launch_dependents();
    if (warp == 0 && !a.g.mask && unit < a.tiles && elect_one()) {
        // while the kernel before runs, the first tile's weights come to L2 (where they are in one piece)
        const int32_t v = unit / a.m_tiles * NT + rank * 128;
        const int64_t all = min(128, a.V - v) * a.row_bytes;
        for (int64_t at = 0; at < min(all, int64_t(kAskFirst)); at += kAskPiece)
            bulk_prefetch(a.w + v * a.row_bytes + at, uint32_t(min(int64_t(kAskPiece), all - at)));
    }
    pdl_wait();
    if (a.g.mask && a.M <= kLookRows) {  // k_head_rows may have left nothing to do (the same answer in all CTAs)
        bool any = false;
        for (int32_t m = threadIdx.x; m < a.M; m += kThreads4<kPair>) any |= __ldg(a.dense + m) != 0;
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
                for (int32_t v = v0; v < min(a.V, v0 + NT); v += 128) any |= row_uses(a, m, v);
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
        float *const tokens = token_scales[warp - kFirst];
        uint32_t it = 0;
        // a tile's scales, read while the tile before is stored
        float row_next = 0.0f, token_next[3] = {0.0f, 0.0f, 0.0f};
        auto read_scales = [&](int32_t t) {
            if (t >= a.tiles) return;
            const int32_t m = t % a.m_tiles * (kRows * kCtas) + rank * kRows + quarter * 32, v = t / a.m_tiles * NT + column;
            row_next = __ldg(a.q_rows + min(m + lane, a.M - 1));
            token_next[0] = __ldg(a.w_rows + min(v + lane, a.V - 1));
            token_next[1] = __ldg(a.w_rows + min(v + lane + 32, a.V - 1));
            if (!kWide) token_next[2] = __ldg(a.w_rows + min(v + lane + 64, a.V - 1));
        };
        read_scales(unit);
        for (int32_t i = 0, t = unit; t < a.tiles; i++, t += units) {
            const int32_t m0 = t % a.m_tiles * (kRows * kCtas) + rank * kRows, m1 = min(a.M, m0 + kRows);
            const int32_t v0 = t / a.m_tiles * NT, v = v0 + column;
            const float row_scale = row_next;
            tokens[lane] = token_next[0];
            tokens[lane + 32] = token_next[1];
            if (!kWide && lane < 16) tokens[lane + 64] = token_next[2];
            read_scales(t + units);
            __syncwarp();
            if (!needed(i)) {
                fill_tile<T, NT, kEpilogue>(a, m0, m1, v0, warp - kFirst, lane);
                __syncwarp();
                continue;
            }
            const int32_t mine = m0 + quarter * 32, row = min(mine + lane, a.M - 1);
            const bool there = mine < m1;  // a warp without rows only keeps the barriers going
            const uint32_t acc = it % kAccumulators;
            bar_wait(ready + 8 * acc, (it / kAccumulators) & 1, &gave_up);
            it++;
            tcgen05_fence_after();
            const bool ok = *static_cast<volatile int *>(&gave_up) == 0;
            const GrammarRow allow = grammar_row(a.g, row);
            // 16 tokens from v + c on
            auto logits = [&](const uint32_t (&sums)[16], int c, float (&x)[16]) {
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const float4 f = *reinterpret_cast<const float4 *>(tokens + c + e);
                    x[e] = __uint_as_float(sums[e]) * row_scale * f.x;
                    x[e + 1] = __uint_as_float(sums[e + 1]) * row_scale * f.y;
                    x[e + 2] = __uint_as_float(sums[e + 2]) * row_scale * f.z;
                    x[e + 3] = __uint_as_float(sums[e + 3]) * row_scale * f.w;
                }
                uint32_t bits = ~0u;
                if (a.g.mask) bits = (v + c) >> 5 < a.g.W ? allow.word((v + c) >> 5) >> (c & 16) : 0u;
                if (!ok || (bits & 0xFFFFu) != 0xFFFFu) {
#pragma unroll
                    for (int e = 0; e < 16; e++) {
                        if (!ok) x[e] = __int_as_float(0x7FFFFFFF);  // gave up waiting: no result
                        if (!((bits >> e) & 1u)) x[e] = -INFINITY;
                    }
                }
            };
            auto word = [](const float (&x)[16], int i) {
                const __nv_bfloat162 both = __floats2bfloat162_rn(x[2 * i % 16], x[2 * i % 16 + 1]);
                return sizeof(T) == 4 ? __float_as_uint(x[i]) : *reinterpret_cast<const uint32_t *>(&both);
            };
            // what this warp needs of the tokens behind its own, where they are all there and it is to write some of them
            const bool next = !kWide && column + kColumns < NT && v + 2 * kColumns <= a.V;
            uint32_t raw[kColumns / 16][16], following[8];
            if (there && next) {
                tmem_load16(from + acc * NT + kColumns, raw[0]);
                tmem_wait_ld();
                float x[16];
                logits(raw[0], kColumns, x);
#pragma unroll
                for (int i = 0; i < 8; i++) following[i] = word(x, i);
            }
            if (there) {
#pragma unroll
                for (int c = 0; c < kColumns / 16; c++) tmem_load16(from + acc * NT + 16 * c, raw[c]);
                tmem_wait_ld();
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (kPair) bar_arrive_remote(drain + 8 * acc);
                else bar_arrive(drain + 8 * acc);
            }
            if (there) {
                const int32_t rows = min(32, m1 - mine);
                uint32_t some = ~0u;
                if (a.g.mask) some = __ballot_sync(~0u, __ldg(a.dense + row) != 0);
                if (kWide || v + kColumns > a.V) {
#pragma unroll
                    for (int c = 0; c < kColumns; c += 16) {
                        float x[16];
                        logits(raw[c / 16], c, x);
                        if (v + c < a.V) store16<T, kWide>(a, x, mine, rows, some, v + c, lane);
                    }
                } else {
                    Shifted<T> shifted(a, mine + lane, v, lane < rows && ((some >> lane) & 1u), column == 0, next);
                    constexpr int kWords = int(sizeof(T)) * 4;  // of 16 tokens
#pragma unroll
                    for (int c = 0; c < kColumns; c += 16) {
                        float x[16];
                        uint32_t w[kWords];
                        logits(raw[c / 16], c, x);
#pragma unroll
                        for (int i = 0; i < kWords; i++) w[i] = word(x, i);
#pragma unroll
                        for (int i = 0; i < kWords; i += 8) shifted.put(w + i, (c / 16 * kWords + i) / 8);
                    }
                    if (next) shifted.put(following, Shifted<T>::kPieces);
                }
            }
            __syncwarp();  // the next tile's scales are written where these were read
        }
    } else {
        if (kPair) fewer_registers<32>();
        if (warp == 0) {
            int stage = 0;
            uint32_t phase = 1, used = 0;  // phase: of a stage's last use; the first time round there is none
            bool ok = true;
            const uint32_t leader = kPair ? cluster_addr(full, 0) : full;
            for (int32_t i = 0, t = unit; t < a.tiles && ok; i++, t += units) {
                if (!needed(i)) continue;
                const int32_t m = t % a.m_tiles * (kRows * kCtas) + rank * kRows, v0 = t / a.m_tiles * NT;
                for (int32_t kb = 0; kb < a.blocks; kb++) {
                    const uint32_t at = stages + uint32_t(stage) * stage_bytes, bar = leader + 8 * stage;
                    const uint32_t scales = at + 128 * 128, hidden_scales = at + kWeightBytes4<kPair>, hidden = hidden_scales + kHiddenScales;
                    ok = bar_wait(empty + 8 * stage, phase, &gave_up);
                    ok = __all_sync(~0u, ok);
                    if (!ok) break;
                    if (elect_one()) {
                        // all that comes to a tile's CTAs counts on its first one's barrier
                        if (rank == 0) bar_expect(full + 8 * stage, kCtas * stage_bytes);
                        if (kPair) {
                            tma_load_2d_pair(at, &a.map_w, kb * 128, v0 + rank * 128, bar);
                            tma_load_3d_pair(scales, &a.map_ws, 0, kb * kSteps, v0 / 128, bar);
                            tma_load_3d_pair(hidden_scales, &a.map_s, 0, kb * kSteps, m / 128, bar);
                            tma_load_2d_pair(hidden, &a.map_q, kb * 128, m, bar);
                        } else {
                            tma_load_2d(at, &a.map_w, kb * 128, v0, bar);
                            tma_load_3d(scales, &a.map_ws, 0, kb * kSteps, v0 / 128, bar);
                            tma_load_3d(hidden_scales, &a.map_s, 0, kb * kSteps, m / 128, bar);
                            tma_load_2d(hidden, &a.map_q, kb * 128, m, bar);
                        }
                    }
                    __syncwarp();
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
                for (uint32_t i = 0; i < used && rank == 0; i++) {
                    if (--stage < 0) stage = a.stages - 1, phase ^= 1;
                    bar_wait(full + 8 * stage, phase ^ 1, &none);
                }
            }
        } else if (warp == 1) {
            if (rank == 0) {
                constexpr uint32_t idesc = mma_idesc_e2m1(kRows * kCtas, NT);
                int stage = 0;
                uint32_t phase = 0, it = 0, slot = 0;
                bool ok = true;
                for (int32_t i = 0, t = unit; t < a.tiles && ok; i++, t += units) {
                    if (!needed(i)) continue;
                    const uint32_t acc = it % kAccumulators;
                    ok = bar_wait(drained + 8 * acc, ((it / kAccumulators) & 1) ^ 1, &gave_up);
                    it++;
                    for (int32_t kb = 0; kb < a.blocks; kb++) {
                        ok = ok && bar_wait(full + 8 * stage, phase, &gave_up);
                        ok = __all_sync(~0u, ok);
                        if (!ok) break;
                        tcgen05_fence_after();
                        const uint32_t at = stages + uint32_t(stage) * stage_bytes;
                        const uint32_t scales = at + 128 * 128, hidden_scales = at + kWeightBytes4<kPair>;
                        const uint64_t dw = mma_desc(at), dq = mma_desc(hidden_scales + kHiddenScales);
                        const uint32_t sq = tmem + 256 + slot * kSlotColumns, sw = sq + kHiddenColumns;
                        const int32_t steps = int32_t(min(int64_t(kSteps), a.tiles_k - int64_t(kb) * kSteps));
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < kSteps; k++) {
                                if (k >= steps) break;
                                tmem_copy_scales<kPair>(sq + 4 * k, hidden_scales + k * kScaleTile);
#pragma unroll
                                for (int j = 0; j < NT / 128; j++)
                                    tmem_copy_scales<kPair>(sw + k * (NT / 32) + 4 * j, scales + (j * kSteps + k) * kScaleTile);
                            }
#pragma unroll
                            for (int k = 0; k < kSteps; k++) {
                                if (k >= steps) break;
                                mma_e2m1<kPair>(tmem + acc * NT, dq + 2 * k, dw + 2 * k, idesc, sq + 4 * k, sw + k * (NT / 32), kb > 0 || k > 0);
                            }
                            mma_commit<kPair>(empty + 8 * stage);
                            if (kb == a.blocks - 1) mma_commit<kPair>(ready + 8 * acc);
                        }
                        __syncwarp();
                        slot ^= 1;
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

// [rows / 128][columns / 64][512 bytes] in boxes of `box_rows` x kSteps x 512 bytes, zeros outside.
bool make_scale_map(CUtensorMap *map, const void *base, int64_t rows, int64_t tiles, int32_t box_rows) {
    const Encode encode = tensor_map_encode();
    if (!encode) return false;
    const cuuint64_t dims[3] = {kScaleTile / 4, cuuint64_t(tiles), cuuint64_t((rows + 127) / 128)};
    const cuuint64_t strides[2] = {kScaleTile, cuuint64_t(tiles) * kScaleTile};
    const cuuint32_t box[3] = {kScaleTile / 4, kSteps, cuuint32_t(box_rows)}, steps[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void *>(base), dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, bool kPair, bool kWide>
cudaError_t launch_head4(Head4Args a, cudaStream_t st) {
    const int stage = kWeightBytes4<kPair> + kHiddenScales + a.box_rows * 128;
    // the last stage's MMA reads kRows rows, whatever was loaded; and room to align the ring
    const int beyond = (kRows - a.box_rows) * 128 + 1024;
    constexpr int fixed = kEpilogueWarps4<kPair> * int(sizeof(float)) * (kColumns + 16) + 1024;  // declared in the kernel
    a.stages = std::min(kMaxStages, (kHeadSmem - fixed - beyond) / stage);
    const int smem = a.stages * stage + beyond;
    const cudaError_t e = allow_smem<k_head4<T, kPair, kWide>, kHeadSmem - fixed>();
    if (e != cudaSuccess) return e;
    constexpr int kCluster = kPair ? 2 : 1;
    const int units = std::min(a.tiles, std::max(1, sm_count() / kCluster));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(units * kCluster));
    cfg.blockDim = dim3(kThreads4<kPair>);
    cfg.dynamicSmemBytes = size_t(smem);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = unsigned(kCluster);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kCluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_head4<T, kPair, kWide>, a);
}

template <typename T, bool kWide>
cudaError_t launch_wide(const Head4Args &a, bool pair, cudaStream_t st) {
    return pair ? launch_head4<T, true, kWide>(a, st) : launch_head4<T, false, kWide>(a, st);
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
    if (!*bad && M > (1 << 20)) bad = "M must be <= 2^20";
    if (!*bad && M > 0 && d_mask && !d_workspace) bad = "d_mask without d_workspace";
    if (!*bad && off_boundary(16, static_cast<const char *>(d_workspace))) bad = "d_workspace is not aligned to 16 bytes";
    if (*bad) return set_error(TRIE_EINVAL, bad);
    if (M == 0) return TRIE_OK;
    Head4Args a = {};
    a.q = d_q;
    a.s = d_scales;
    a.q_rows = d_row_scales;
    a.w = d_w;
    a.ws = d_w_scales;
    a.w_rows = d_w_row_scales;
    a.M = M;
    a.V = V;
    a.D = D;
    a.row_bytes = row_bytes4(D);
    a.tiles_k = scale_tiles4(D);
    a.blocks = (D + kStageColumns - 1) / kStageColumns;
    const bool pair = M > kRows;
    const int side = pair ? 256 : 128;  // of a tile
    a.m_tiles = (M + side - 1) / side;
    a.box_rows = std::min(kRows, (M + 15) / 16 * 16);
    a.logits = d_logits;
    a.stride = stride;
    const bool wide = ((reinterpret_cast<uintptr_t>(d_logits) | uintptr_t(stride * (dtype == TRIE_DTYPE_F32 ? 4 : 2))) & 31) == 0;
    a.g = make_grammar(d_mask, mask_rows, d_states, V);
    if (!make_map(&a.map_w, d_w, V, a.row_bytes, 128) || !make_map(&a.map_q, d_q, M, a.row_bytes, a.box_rows) ||
        !make_scale_map(&a.map_ws, d_w_scales, V, a.tiles_k, side / 128) || !make_scale_map(&a.map_s, d_scales, M, a.tiles_k, 1))
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
        const int smem = D <= kFewMaxD ? int(a.row_bytes + a.row_bytes / 8 * 4) : 0;
        e = f32 ? launch_pdl_smem(k_head_rows<float, Head4Args>, M, kRowThreads, smem, stream, a)
                : launch_pdl_smem(k_head_rows<__nv_bfloat16, Head4Args>, M, kRowThreads, smem, stream, a);
        if (e != cudaSuccess) return fail_launch(e, "4-bit head rows launch");
    }
    if (f32) e = wide ? launch_wide<float, true>(a, pair, stream) : launch_wide<float, false>(a, pair, stream);
    else e = wide ? launch_wide<__nv_bfloat16, true>(a, pair, stream) : launch_wide<__nv_bfloat16, false>(a, pair, stream);
    if (e != cudaSuccess) return fail_launch(e, "4-bit head launch");
    return TRIE_OK;
}
