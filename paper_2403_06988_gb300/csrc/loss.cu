// loss.cu -- the cross entropy of target tokens under the masked softmax of
// hidden . weight^T, and its gradient (sm_103a).  The logits [rows][V] are
// never kept: their products are computed on the tensor cores tile by tile and
// folded at once, and the gradient recomputes them in pieces of the
// vocabulary.
//
//   x[t][v] = sum_d h[t][d] w[v][d]            A_t: the tokens the mask allows
//   lse[t]  = log sum_{v in A_t} exp x[t][v]
//   loss[t] = lse[t] - x[t][y_t]               0 without a target, +inf where
//                                              the mask excludes the target
//   G[t][v] = c_t (exp(x[t][v] - lse[t]) - [v = y_t]) for v in A_t, else 0
//             c_t = grad_loss[t], 0 for rows without a finite loss
//   dh      = G w          dw = G^T h
//
// product_kernel  one warp-specialised persistent kernel for all four products
//                 (a tile of A B^T per step): TMA loads into a ring of
//                 swizzled tiles, tcgen05.mma into two accumulators in tensor
//                 memory, eight warps that fold one accumulator while the next
//                 is filled.  What it does with a tile is its Fold.
// loss_kernel     merges a row's partials into lse and loss.
// prep_kernel, dhidden_kernel: the rows' coefficients and operands
//                 laid out for TMA, the sum of the hidden gradient's parts.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "bf16_rows.cuh"
#include "decode.cuh"
#include "loss.h"
#include "tcgen05.cuh"
#include "tensor_map.h"

namespace domino {
namespace {

// Tiles of a product: kRowsM rows of A a CTA and N of B.  PAIR: two CTAs make
// 2 * kRowsM rows and hold half of B each, so that a product's operands take two
// thirds of the bytes.
constexpr int kRowsM = 128, kTileK = 64, kWideN = 256, kNarrowN = 64;
constexpr int kAccs = 2;                       // accumulators of N columns: of 256, all of tensor memory
constexpr int kRingBytes = 196608;             // of operand tiles on their way
constexpr int kMaxStages = 16;                 // k blocks of them
constexpr int kFoldWarps = 8;
template <bool PAIR, int N>
struct Tile {
    static constexpr int kCtas = PAIR ? 2 : 1;
    static constexpr int kM = kRowsM * kCtas, kN = N;
    static constexpr int kRowsB = N / kCtas;           // a CTA's
    static constexpr int kBytesA = kRowsM * kTileK * 2, kBytesB = kRowsB * kTileK * 2;
    static constexpr int kColumns = N / (kFoldWarps / 4);   // a fold warp's: 32 rows, half of the columns
    static_assert(kRingBytes % (kBytesA + kBytesB) == 0 && kColumns % 32 == 0);
};
// Which tiles a launch takes: 256 x 256 of two CTAs, 128 x 256, 128 x 64.
enum Shape : int { kPair = 0, kWide = 1, kNarrow = 2 };
int shape_m(Shape s) { return s == kPair ? 2 * kRowsM : kRowsM; }
int shape_n(Shape s) { return s == kNarrow ? kNarrowN : kWideN; }
int shape_box(Shape s) { return s == kWide ? kWideN : s == kPair ? kWideN / 2 : kNarrowN; }   // rows of B a CTA loads

// Results leave through shared memory: 32 rows of 64 bytes a warp's buffer, in the 64-byte swizzle.
constexpr int kOutBytes = 32 * 64, kOutBuffers = 16 / kFoldWarps;
constexpr int kProductSmem = kRingBytes + kFoldWarps * kOutBuffers * kOutBytes + 1024;   // tiles lie on 1024-byte boundaries
constexpr int kProductThreads = 128 + 32 * kFoldWarps;
constexpr int kGroupM = 16;                    // row tiles that share a pass over the columns' tiles

// A tensor-core sum is cut, not rounded, at every step of 16 products: what it
// loses grows with the steps.  Logits of more than kDeepBlocks k blocks are
// summed in parts, each in an accumulator of its own, which are added in fp32
// (256 x 128256 x 4096: lse 1.9e-6 off in one part of 64 blocks, 4e-7 in parts of
// 16, 6e-7 of 24; 184 us in one part, 193, 192 and 192 in parts of 16, 24 and 32; 4096
// rows 2060, 2120, 2100, 2064).  G is rounded to bf16, a thousand times as much: its
// logits are summed in one, and so is a split's part of G w, over up to a whole
// piece of the vocabulary (4096 x 128256 x 4096 against 64 bits: dhidden 2.20e-3 off,
// dweight 2.18e-3, 1.66e-3 of each the results' own rounding; their lengths along the
// right ones are 1.7e-5 too short and 2.7e-5 too long: the cuts do not add up).
constexpr int kDeepBlocks = 24;

// What becomes of a tile of products.
enum ProductFold : int {
    kFoldLogSum = 0,   // rows of tokens, columns of the vocabulary: (max, sum of exp) and the target's logit
    kFoldGrad = 1,     // the same tile: G, in bf16
    kFoldHidden = 2,   // G w: added to fp32 planes
    kFoldWeight = 3,   // G^T h: the weight's gradient, in bf16
    kFoldLogSumDeep = 4,   // kFoldLogSum in parts
};

struct Product {
    CUtensorMap a, b;
    CUtensorMap to;                // where the results go, in boxes of 32 rows and 64 bytes (kFoldGrad, kFoldHidden, kFoldWeight)
    int32_t m, n;                  // valid rows and columns of the product
    int32_t m_tiles, n_tiles, splits, k_blocks;   // k_blocks: of the whole sum, shared out over the splits
    int32_t a_mn, b_mn;            // operands whose rows of memory run along k (MN-major)
    // Rows of A that a CTA loads, a multiple of 8.  Fewer than kRowsM where the product has fewer: a product then reads
    // what lies behind them in shared memory, into rows of the accumulator that nothing uses, and the ring holds more
    // k blocks (5 rows, V = 32000, 1024 wide: 16.2 us with 4 blocks on their way, 12.7 with 5).
    int32_t a_rows;
    int32_t items;                 // m_tiles * n_tiles * splits
    // kFoldLogSum, kFoldGrad
    const uint32_t* mask;          // at the first column's word; nullptr: everything allowed
    int64_t mask_words;            // of a row
    const int32_t* targets;
    int32_t column0;               // token id of column 0
    float2* part;                  // [m][part_pitch]
    int32_t part_pitch;
    float* target_logit;           // [m]
    const float* lse;
    const float* coef;             // c_t / scale
    const float* scale;            // kFoldWeight
    __nv_bfloat16* out;            // kFoldWeight: where `to` cannot be, rows off 16-byte boundaries
    int64_t ld;
    int32_t plane_rows;            // kFoldHidden: `to` is [splits][plane_rows][n]
    int32_t add;                   // kFoldHidden: to what the planes hold
    uint32_t* err;
};

struct Item {
    int32_t m, n, k0, k1, split;
};

// Row tiles in groups of kGroupM; in a group the columns' tiles one after the
// other, each with all of the group's row tiles: what CTAs read at a time is
// one column tile and a group of row tiles.
__device__ __forceinline__ Item item_at(const Product& p, int32_t i) {
    Item t;
    const int32_t tiles = p.m_tiles * p.n_tiles;
    t.split = i / tiles;
    i -= t.split * tiles;
    const int32_t group = i / (kGroupM * p.n_tiles);
    const int32_t m0 = group * kGroupM, rows = min(kGroupM, p.m_tiles - m0);
    i -= group * kGroupM * p.n_tiles;
    t.n = i / rows;
    t.m = m0 + i - t.n * rows;
    t.k0 = (int32_t)((int64_t)p.k_blocks * t.split / p.splits);
    t.k1 = (int32_t)((int64_t)p.k_blocks * (t.split + 1) / p.splits);
    return t;
}

// An operand's tile of `rows` m or n and kTileK k, from (r0, k0) on.
template <bool PAIR>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, bool mn, int rows, int32_t r0,
                                          int32_t k0, uint32_t bar) {
    if (!mn) {
        tma_load<PAIR>(dst, map, k0, r0, bar);
    } else {
        for (int c = 0; c < rows; c += 64) tma_load<PAIR>(dst + c * kTileK * 2, map, r0 + c, k0, bar);
    }
}

// Bits of the columns [c, c + 32) of a row that are allowed and below n.
__device__ __forceinline__ uint32_t allowed_word(const uint32_t* mrow, int32_t c, int32_t n) {
    if (c >= n) return 0u;
    const uint32_t word = mrow ? __ldg(mrow + (c >> 5)) : 0xFFFFFFFFu;
    return n - c < 32 ? word & ((1u << (n - c)) - 1u) : word;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ float2 mul2(float2 a, float b) {
    unsigned long long x, y, r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a.x), "f"(a.y));
    asm("mov.b64 %0, {%1, %1};" : "=l"(y) : "f"(b));
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    float2 o;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(o.x), "=f"(o.y) : "l"(r));
    return o;
}

// What a warp's lane needs beside the products of its row in a tile.
template <int COLUMNS>
struct Side {
    uint32_t word[COLUMNS / 32];        // allowed tokens
    int32_t target;                     // its column
    float lse, coef;
};

template <int FOLD, typename T>
__device__ __forceinline__ Side<T::kColumns> load_side(const Product& p, int32_t item, int row_in_tile, int half) {
    Side<T::kColumns> s;
    const Item t = item_at(p, item);
    const int32_t row = t.m * T::kM + row_in_tile, c0 = t.n * T::kN + half * T::kColumns;
    const bool on = row < p.m;
    s.target = on ? (int32_t)((uint32_t)__ldg(p.targets + row) - (uint32_t)p.column0) : -1;
    s.lse = FOLD == kFoldGrad && on ? p.lse[row] : 0.0f;
    s.coef = FOLD == kFoldGrad && on ? p.coef[row] : 0.0f;
    const uint32_t* mrow = p.mask && on ? p.mask + (int64_t)row * p.mask_words : nullptr;
    // a row that is none does not slow its warp's others down
#pragma unroll
    for (int j = 0; j < T::kColumns / 32; ++j) s.word[j] = on ? allowed_word(mrow, c0 + 32 * j, p.n) : 0xFFFFFFFFu;
    return s;
}

// 16 words (64 bytes) of each lane's row to one of the warp's buffers, and from there to (x, y).
// A buffer was read by its copy before it is written again.
__device__ __forceinline__ void put_rows(const CUtensorMap* map, int32_t x, int32_t y, bool add, uint32_t buffer, int lane,
                                         const uint32_t* w) {
    if (lane == 0) tma_wait_read<kOutBuffers - 1>();
    __syncwarp();
    put_words(buffer, lane, w);
    tma_fence();
    __syncwarp();
    if (lane == 0) {
        if (add) tma_add(map, x, y, buffer);
        else tma_store(map, x, y, buffer);
        tma_commit();
    }
}

// 32 logits of a row, those that `word` allows, into the row's (m, sum).
__device__ __forceinline__ void fold_log_sum(float* v, uint32_t word, float& m, float& sum) {
    if (!__all_sync(0xffffffffu, word == 0xFFFFFFFFu)) {
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = (word & (1u << e)) ? v[e] : -INFINITY;
    }
    float top = m;
#pragma unroll
    for (int e = 0; e < 32; e += 2) top = fmaxf(fmaxf(top, v[e]), v[e + 1]);
    const float ref = sum_ref(top);
    float2 s0 = make_float2(sum * exp_diff(m, ref), 0.0f), s1 = make_float2(0.0f, 0.0f);
    const float2 nref = make_float2(-ref, -ref);
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        const float2 d0 = mul2(add2(make_float2(v[e], v[e + 1]), nref), kLog2e);
        const float2 d1 = mul2(add2(make_float2(v[e + 2], v[e + 3]), nref), kLog2e);
        s0 = add2(s0, make_float2(ex2(d0.x), ex2(d0.y)));
        s1 = add2(s1, make_float2(ex2(d1.x), ex2(d1.y)));
    }
    s0 = add2(s0, s1);
    sum = s0.x + s0.y;
    m = top;
}

// The value at place `at` of 32 (below 32), if this row has it there.
__device__ __forceinline__ float pick(const float* v, uint32_t at) {
    float x = 0.0f;
#pragma unroll
    for (int e = 0; e < 32; ++e) x = at == (uint32_t)e ? v[e] : x;
    return x;
}

template <int FOLD, bool PAIR, int N>
__global__ void __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ Product p) {
    using T = Tile<PAIR, N>;
    constexpr int kColumns = T::kColumns, kTmemColumns = kAccs * N;
    constexpr bool kDeep = FOLD == kFoldLogSumDeep, kLogSum = FOLD == kFoldLogSum || kDeep;
    extern __shared__ unsigned char smem[];
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_acc_full[kAccs], s_acc_empty[kAccs], s_done;
    __shared__ uint32_t s_tmem, s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tiles = (smem_addr(smem) + 1023u) & ~1023u;
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const int32_t first = blockIdx.x / T::kCtas, step = gridDim.x / T::kCtas;   // items of this CTA or pair
    volatile uint32_t* failed = &s_failed;
    const uint32_t bytes_a = p.a_rows * kTileK * 2, stage_bytes = bytes_a + T::kBytesB;
    const uint32_t stages = min((uint32_t)kMaxStages, kRingBytes / stage_bytes);
    if (threadIdx.x == 0) {
        s_failed = 0u;
        for (int s = 0; s < kMaxStages; ++s) {
            bar_init(smem_addr(&s_full[s]), 1);
            bar_init(smem_addr(&s_empty[s]), 1);
        }
        for (int s = 0; s < kAccs; ++s) {
            bar_init(smem_addr(&s_acc_full[s]), 1);
            bar_init(smem_addr(&s_acc_empty[s]), kFoldWarps * T::kCtas);
        }
        bar_init(smem_addr(&s_done), 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        tma_prefetch_map(&p.a);
        tma_prefetch_map(&p.b);
    }
    if (warp == 2) tmem_alloc<PAIR>(smem_addr(&s_tmem), kTmemColumns);
    tcgen_before();
    __syncthreads();
    if constexpr (PAIR) cluster_barrier();
    tcgen_after();
    const uint32_t tmem = s_tmem;
    pdl_wait();
    pdl_trigger();

    if (warp == 0) {   // ---- loads: each CTA its part of the tiles; the first CTA's barriers count the bytes of both
        uint32_t s = 0, turn = 0, loads = 0;   // the stage, how often the ring has come round
        bool ok = true;
        for (int32_t i = first; i < p.items && ok; i += step) {
            const Item t = item_at(p, i);
            const int32_t row_a = t.m * T::kM + rank * kRowsM, row_b = t.n * N + rank * T::kRowsB;
            for (int32_t k = t.k0; k < t.k1; ++k) {
                if (!(ok = warp_wait(smem_addr(&s_empty[s]), (turn & 1u) ^ 1u, failed))) break;
                const uint32_t mine = smem_addr(&s_full[s]), a = tiles + s * stage_bytes;
                const uint32_t full = PAIR ? in_cta(mine, 0) : mine;
                if (elect_lane()) {
                    if (rank == 0) bar_expect(mine, stage_bytes * T::kCtas);
                    load_tile<PAIR>(a, &p.a, p.a_mn, kRowsM, row_a, k * kTileK, full);
                    load_tile<PAIR>(a + bytes_a, &p.b, p.b_mn, T::kRowsB, row_b, k * kTileK, full);
                }
                ++loads;
                if (++s == stages) {
                    s = 0;
                    ++turn;
                }
            }
        }
        // given up: the loads on their way write into this CTA's memory
        if (!ok && rank == 0 && lane == 0)
            for (uint32_t j = 1; j <= stages && j <= loads; ++j) {
                const uint32_t last = loads - j;   // the stages' last loads
                const uint64_t end = timer_ns() + kWaitNs;
                while (!bar_try(smem_addr(&s_full[last % stages]), (last / stages) & 1u) && timer_ns() < end) {}
            }
    } else if (warp == 1) {   // ---- products
        if (rank == 0) {
            const uint32_t desc = mma_desc(T::kM, N, p.a_mn, p.b_mn);
            // 16 k further: 32 bytes along a row of a K-major tile, 16 rows of an MN-major one (16-byte units)
            const uint32_t step_a = p.a_mn ? 2048 / 16 : 32 / 16, step_b = p.b_mn ? 2048 / 16 : 32 / 16;
            uint32_t s = 0, turn = 0, accs = 0;
            bool ok = true;
            for (int32_t i = first; i < p.items && ok; i += step) {
                const Item t = item_at(p, i);
                for (int32_t k0 = t.k0, k1; ok; k0 = k1, ++accs) {   // an accumulator each
                    k1 = kDeep ? min(t.k1, k0 + kDeepBlocks) : t.k1;
                    const uint32_t s_acc = accs % kAccs, acc = tmem + s_acc * N;
                    if (!(ok = warp_wait(smem_addr(&s_acc_empty[s_acc]), ((accs / kAccs) & 1u) ^ 1u, failed))) break;
                    tcgen_after();
                    for (int32_t k = k0; k < k1; ++k) {
                        if (!(ok = warp_wait(smem_addr(&s_full[s]), turn & 1u, failed))) break;
                        tcgen_after();
                        const uint64_t a = operand_desc(tiles + s * stage_bytes, kTileK * 128);
                        const uint64_t b = operand_desc(tiles + s * stage_bytes + bytes_a, kTileK * 128);
                        if (elect_lane()) {
#pragma unroll
                            for (int j = 0; j < kTileK / 16; ++j)
                                mma_bf16<PAIR>(acc, a + (uint64_t)(j * step_a), b + (uint64_t)(j * step_b), desc, k > k0 || j > 0);
                            mma_commit<PAIR>(smem_addr(&s_empty[s]));
                        }
                        if (++s == stages) {
                            s = 0;
                            ++turn;
                        }
                    }
                    if (ok && elect_lane()) mma_commit<PAIR>(smem_addr(&s_acc_full[s_acc]));
                    if (k1 >= t.k1) {
                        ++accs;
                        break;
                    }
                }
            }
            if (elect_lane()) mma_commit<PAIR>(smem_addr(&s_done));
        }
        // no product, and no arrival at a barrier of this CTA, may be on its way when the CTA ends
        if (lane == 0) {
            const uint64_t end = timer_ns() + 3 * kWaitNs;
            while (!bar_try(smem_addr(&s_done), 0u) && timer_ns() < end) {}
        }
    } else if (warp >= 4) {   // ---- folds
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t buffers = tiles + kRingBytes + (warp - 4) * kOutBuffers * kOutBytes;
        const int row_in_tile = rank * kRowsM + quarter * 32 + lane;
        constexpr bool kTokens = kLogSum || FOLD == kFoldGrad;
        uint32_t accs = 0, puts = 0;
        Side<kColumns> next{};
        if (kTokens && first < p.items) next = load_side<FOLD, T>(p, first, row_in_tile, half);
        float scale = 1.0f;
        if constexpr (FOLD == kFoldWeight) scale = *p.scale;
        // waits for the next accumulator; the whole warp goes on or leaves: loads from tensor memory are a warp's
        const auto filled = [&] {
            const bool ok = warp_wait(smem_addr(&s_acc_full[accs % kAccs]), (accs / kAccs) & 1u, failed);
            tcgen_after();
            return ok;
        };
        const auto columns = [&] { return tmem + (accs % kAccs) * N + half * kColumns + ((uint32_t)(quarter * 32) << 16); };
        // gives it back
        const auto emptied = [&] {
            tcgen_before();
            __syncwarp();
            const uint32_t bar = smem_addr(&s_acc_empty[accs % kAccs]);
            if (lane == 0) {
                if constexpr (PAIR) bar_arrive_cluster(in_cta(bar, 0));
                else bar_arrive(bar);
            }
            ++accs;
        };
        bool ok = true;
        for (int32_t i = first; i < p.items; i += step) {
            const Item t = item_at(p, i);
            const int32_t row = t.m * T::kM + row_in_tile, row0 = row - lane, c0 = t.n * N + half * kColumns;
            const bool on = row < p.m;
            // the next tile's are on their way while this one is folded
            const Side<kColumns> side = next;
            if (kTokens && i + step < p.items) next = load_side<FOLD, T>(p, i + step, row_in_tile, half);
            float m = -INFINITY, sum = 0.0f;
            if constexpr (kDeep) {
                float x[kColumns];
#pragma unroll
                for (int e = 0; e < kColumns; ++e) x[e] = 0.0f;
                for (int32_t k = t.k0; k < t.k1; k += kDeepBlocks) {
                    if (!(ok = filled())) break;
                    const uint32_t acc = columns();
#pragma unroll
                    for (int e = 0; e < kColumns; e += 16) tmem_add16(x + e, acc + e);
                    emptied();
                }
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < kColumns / 32; ++j) {
                    const uint32_t at = (uint32_t)side.target - (uint32_t)(c0 + 32 * j);
                    if (__any_sync(0xffffffffu, at < 32u)) {
                        const float y = pick(x + 32 * j, at);
                        if (at < 32u && on) p.target_logit[row] = y;
                    }
                    fold_log_sum(x + 32 * j, side.word[j], m, sum);
                }
                if (on) p.part[(int64_t)row * p.part_pitch + t.n * (N / kColumns) + half] = make_float2(m, sum);
                continue;
            }
            if (!(ok = filled())) break;
            const uint32_t acc = columns();
#pragma unroll 1
            for (int j = 0; j < kColumns / 32; ++j) {
                const int32_t c = c0 + 32 * j;
                if (c >= p.n && FOLD != kFoldGrad) break;   // the tile's columns beyond the last
                float v[32];
                tmem_load32(v, acc + 32 * j);
                uint32_t word = side.word[0];   // not by an index: the words stay in registers
#pragma unroll
                for (int k = 1; k < kColumns / 32; ++k) word = j == k ? side.word[k] : word;
                const uint32_t at = (uint32_t)side.target - (uint32_t)c;   // below 32: the target's place
                if constexpr (FOLD == kFoldLogSum) {
                    if (__any_sync(0xffffffffu, at < 32u)) {
                        const float x = pick(v, at);
                        if (at < 32u && on) p.target_logit[row] = x;
                    }
                    fold_log_sum(v, word, m, sum);
                } else if constexpr (FOLD == kFoldGrad) {
                    const float2 nlse = make_float2(-side.lse, -side.lse);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float2 d = mul2(add2(make_float2(v[e], v[e + 1]), nlse), kLog2e);
                        const float2 q = mul2(make_float2(ex2(d.x), ex2(d.y)), side.coef);
                        v[e] = q.x;
                        v[e + 1] = q.y;
                    }
                    if (__any_sync(0xffffffffu, at < 32u)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = at == (uint32_t)e ? v[e] - side.coef : v[e];
                    }
                    // rows without a gradient, and columns beyond the vocabulary (they are read again): zeros
                    const uint32_t keep = side.coef != 0.0f ? word : 0u;
                    if (!__all_sync(0xffffffffu, keep == 0xFFFFFFFFu)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = (keep & (1u << e)) ? v[e] : 0.0f;
                    }
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                    if (row0 < p.m) put_rows(&p.to, c, row0, false, buffers + (puts++ % kOutBuffers) * kOutBytes, lane, w);
                } else if constexpr (FOLD == kFoldHidden) {
                    // a split of a short piece may have no products: its accumulator holds an earlier tile's
                    if (row0 < p.m && (t.k0 < t.k1 || !p.add)) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t w[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) w[e] = t.k0 < t.k1 ? __float_as_uint(v[16 * h + e]) : 0u;
                            if (c + 16 * h < p.n)
                                put_rows(&p.to, c + 16 * h, t.split * p.plane_rows + row0, p.add != 0,
                                         buffers + (puts++ % kOutBuffers) * kOutBytes, lane, w);
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] *= scale;
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                    if (!p.out) {
                        if (row0 < p.m) put_rows(&p.to, c, row0, false, buffers + (puts++ % kOutBuffers) * kOutBytes, lane, w);
                    } else {   // a row after the other, a column a lane
                        const uint32_t buffer = buffers;
                        __syncwarp();
                        put_words(buffer, lane, w);
                        __syncwarp();
                        const uint32_t chunk = (uint32_t)lane >> 3, byte = (lane & 7) * 2;
                        uint16_t* to = reinterpret_cast<uint16_t*>(p.out) + (int64_t)row0 * p.ld + c + lane;
                        const int rows = c + lane < p.n ? min(32, p.m - row0) : 0;
#pragma unroll
                        for (int r0 = 0; r0 < 32; r0 += 8) {
                            uint16_t x[8];
#pragma unroll
                            for (int r = r0; r < r0 + 8; ++r)
                                asm volatile("ld.shared.u16 %0, [%1];\n"
                                             : "=h"(x[r - r0])
                                             : "r"(buffer + r * 64 + ((chunk ^ ((r >> 1) & 3)) << 4) + byte));
#pragma unroll
                            for (int r = r0; r < r0 + 8; ++r, to += p.ld)
                                if (r < rows) *to = x[r - r0];
                        }
                    }
                }
            }
            if constexpr (FOLD == kFoldLogSum) {
                if (on) p.part[(int64_t)row * p.part_pitch + t.n * (N / kColumns) + half] = make_float2(m, sum);
            }
            emptied();
        }
        if (lane == 0) tma_wait_all();
    }
    __syncwarp();
    tcgen_before();
    __syncthreads();
    if constexpr (PAIR) cluster_barrier();   // neither CTA's memory or barriers are used by the other any more
    tcgen_after();
    if (warp == 2) tmem_free<PAIR>(tmem, kTmemColumns);
    if (threadIdx.x == 0 && *failed) atomicOr(p.err, DOMINO_DEVERR_INTERNAL);
}

// Whether row t's loss is finite by its target and mask.  report: a target
// beyond the vocabulary sets the error word.
__device__ __forceinline__ bool has_target(const int32_t* targets, const uint32_t* mask, int64_t W, int32_t V, int32_t t,
                                           uint32_t* report, bool* excluded) {
    const int32_t y = __ldg(targets + t);
    *excluded = false;
    if (y < 0) return false;
    if (y >= V) {
        if (report) atomicOr(report, DOMINO_DEVERR_BAD_TOKEN);
        return false;
    }
    if (mask && !((__ldg(mask + t * W + (y >> 5)) >> (y & 31)) & 1u)) {
        *excluded = true;
        return false;
    }
    return true;
}

constexpr int kMergeThreads = 256;

// A warp per row: its partials, each a (max, sum of exp against it), into lse.
__global__ void __launch_bounds__(kMergeThreads)
    loss_kernel(const float2* part, int32_t parts, int32_t pitch, const float* target_logit, const int32_t* targets,
                const uint32_t* mask, int32_t rows, int32_t V, float* loss, float* lse, uint32_t* err) {
    pdl_wait();
    pdl_trigger();
    const int32_t row = blockIdx.x * (kMergeThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (row >= rows) return;
    float m = -INFINITY, s = 0.0f;
    for (int32_t i = lane; i < parts; i += 32) {
        const float2 a = part[(int64_t)row * pitch + i];
        const float m2 = fmaxf(m, a.x), ref = sum_ref(m2);
        s = s * exp_diff(m, ref) + a.y * exp_diff(a.x, ref);
        m = m2;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const float mo = __shfl_xor_sync(0xffffffffu, m, off), so = __shfl_xor_sync(0xffffffffu, s, off);
        const float m2 = fmaxf(m, mo), ref = sum_ref(m2);
        s = s * exp_diff(m, ref) + so * exp_diff(mo, ref);
        m = m2;
    }
    if (lane == 0) {
        // no number among the row's logits: none comes out
        const float z = isnan(s) ? s : log_sum_exp(m, s);
        bool excluded;
        const bool target = has_target(targets, mask, (V + 31) / 32, V, row, err, &excluded);
        if (lse) lse[row] = z;
        loss[row] = target ? z - target_logit[row] : excluded ? INFINITY : 0.0f;
    }
}

constexpr int kPackThreads = 256;

// Rows of bf16 to be laid out in rows of `pitch` (a multiple of 8: what TMA can
// read).  GRAD: rows without a gradient become zeros, so that what stands in them
// (a padding's NaN) meets no other row.
struct Pack {
    const __nv_bfloat16* src;
    int64_t stride;
    int32_t rows, cols;
    __nv_bfloat16* dst;
    int64_t pitch;
    bool aligned;                  // rows of src begin on 16-byte boundaries
};

// Eight values from column c on; zeros beyond the last column.  Rows off 16-byte
// boundaries are read in the 16-byte blocks that hold the values.
__device__ __forceinline__ uint4 read_eight(const Pack& p, const __nv_bfloat16* from, int32_t c) {
    if (c + 8 <= p.cols) {
        if (p.aligned) return __ldg(reinterpret_cast<const uint4*>(from + c));
        const uintptr_t at = reinterpret_cast<uintptr_t>(from + c);
        const uint4* block = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
        const uint32_t off = (uint32_t)(at & 15) / 2;
        const uint4 a = __ldg(block);
        if (off == 0) return a;
        const uint4 b = __ldg(block + 1);
        return eight_from(a, b, off);
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < p.cols) w[i / 2] |= (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(from + c + i)) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct Prep {
    Pack pack[2];                  // hidden, weight; rows 0: none
    int32_t ctas[2];               // of each
    // gradient: the rows' coefficients, by one CTA more, the first
    bool grad;
    const int32_t* targets;
    const uint32_t* mask;
    const float* grad_loss;
    int32_t rows, n_tokens;
    float* coef;
    float* scale;
    uint32_t* err;
};

__device__ __forceinline__ float row_coef(const Prep& p, int32_t t, uint32_t* report) {
    bool excluded;
    return has_target(p.targets, p.mask, (p.n_tokens + 31) / 32, p.n_tokens, t, report, &excluded) ? __ldg(p.grad_loss + t) : 0.0f;
}

// Coefficients over the largest finite one's magnitude: what G is rounded from.
// G is kept in bf16, as the tensor cores take it: the gradients are 2.2e-3 off where
// their own rounding alone makes 1.66e-3, and a second part of G for the bits that go
// would be two products more.  A coefficient that all rows share (a mean's 1 / rows)
// would be off by one rounding, the same in every entry, if it were in G; the scale
// is given back in fp32.
__device__ void make_coefs(const Prep& p) {
    __shared__ float s_top[kPackThreads / 32];
    float top = 0.0f;
    for (int32_t t = threadIdx.x; t < p.rows; t += kPackThreads) {
        const float c = row_coef(p, t, p.err);
        p.coef[t] = c;
        if (fabsf(c) <= FLT_MAX) top = fmaxf(top, fabsf(c));
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
    __syncthreads();
    top = 0.0f;
    for (int w = 0; w < kPackThreads / 32; ++w) top = fmaxf(top, s_top[w]);
    if (top == 0.0f) top = 1.0f;
    if (threadIdx.x == 0) *p.scale = top;
    for (int32_t t = threadIdx.x; t < p.rows; t += kPackThreads) p.coef[t] = p.coef[t] / top;
}

__global__ void __launch_bounds__(kPackThreads) prep_kernel(const __grid_constant__ Prep p) {
    pdl_wait();
    pdl_trigger();
    int32_t cta = blockIdx.x;
    if (p.grad && cta-- == 0) return make_coefs(p);
    const bool second = cta >= p.ctas[0];
    const Pack& k = p.pack[second];
    if (second) cta -= p.ctas[0];
    const uint32_t vectors = (uint32_t)(k.pitch / 8);   // of a row
    const int64_t n = (int64_t)k.rows * vectors, step = (int64_t)p.ctas[second] * kPackThreads;
    for (int64_t i = (int64_t)cta * kPackThreads + threadIdx.x; i < n; i += step) {
        const int32_t r = n <= UINT_MAX ? (int32_t)((uint32_t)i / vectors) : (int32_t)(i / vectors);
        const int32_t c = (int32_t)(i - (int64_t)r * vectors) * 8;
        const bool zero = p.grad && !second && row_coef(p, r, nullptr) == 0.0f;
        *reinterpret_cast<uint4*>(k.dst + r * k.pitch + c) =
            zero ? make_uint4(0, 0, 0, 0) : read_eight(k, k.src + r * k.stride, c);
    }
}

// dhidden = scale * the sum of the planes.  PARTS threads share a vector's planes
// (of one column tile as many as SMs: a chain of 152 loads, 19 with eight threads,
// would take longer than the rest of a small call).
template <int PARTS>
__global__ void __launch_bounds__(kPackThreads)
    dhidden_kernel(const float* planes, int32_t splits, int64_t plane, int32_t rows, int32_t cols, int32_t pitch,
                   const float* scale, __nv_bfloat16* out, int64_t ld) {
    constexpr int kVectors = kPackThreads / PARTS;   // a CTA's
    __shared__ float4 s_sum[PARTS][kVectors];
    pdl_wait();
    pdl_trigger();
    const int32_t vectors = pitch / 4;   // of a row of a plane
    const int64_t n = (int64_t)rows * vectors;
    const int part = threadIdx.x / kVectors, at = threadIdx.x - part * kVectors;
    const int k0 = splits * part / PARTS, k1 = splits * (part + 1) / PARTS;
    const float s = *scale;
    for (int64_t i0 = (int64_t)blockIdx.x * kVectors; i0 < n; i0 += (int64_t)gridDim.x * kVectors) {
        const int64_t i = i0 + at;
        const int32_t r = n <= UINT_MAX ? (int32_t)((uint32_t)i / (uint32_t)vectors) : (int32_t)(i / vectors);
        const int32_t c = (int32_t)(i - (int64_t)r * vectors) * 4;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (i < n) {
#pragma unroll 4
            for (int k = k0; k < k1; ++k) {
                const float4 x = *reinterpret_cast<const float4*>(planes + k * plane + (int64_t)r * pitch + c);
                v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
            }
        }
        if constexpr (PARTS > 1) {
            s_sum[part][at] = v;
            __syncthreads();
            if (part == 0)
#pragma unroll
                for (int k = 1; k < PARTS; ++k) {
                    const float4 x = s_sum[k][at];
                    v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
                }
            __syncthreads();
        }
        if (part || i >= n) continue;
        __nv_bfloat16* to = out + (int64_t)r * ld + c;
        const uint32_t lo = pack_bf16(s * v.x, s * v.y), hi = pack_bf16(s * v.z, s * v.w);
        if (c + 4 <= cols && (reinterpret_cast<uintptr_t>(to) & 7) == 0) {
            *reinterpret_cast<uint2*>(to) = make_uint2(lo, hi);
        } else {
            const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < cols) to[e] = __float2bfloat16_rn(s * x[e]);
        }
    }
}

// ---- host --------------------------------------------------------------------
cudaError_t make_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t pitch, int box_rows) {
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, rows, cols, pitch, 64, box_rows,
                      CU_TENSOR_MAP_SWIZZLE_128B);
}
cudaError_t make_out_map(CUtensorMap* map, void* base, int64_t rows, int64_t cols, int64_t pitch) {
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, rows, cols, pitch, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B);
}
cudaError_t make_plane_map(CUtensorMap* map, void* base, int64_t rows, int64_t cols, int64_t pitch) {
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, base, rows, cols, pitch, 16, 32, CU_TENSOR_MAP_SWIZZLE_64B);
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// Rows of a K-major A that a CTA loads.
int rows_loaded(Shape shape, int32_t m) { return shape == kPair ? kRowsM : std::min(kRowsM, (m + 7) / 8 * 8); }

void cut_product(Product& p, Shape shape, int32_t m, int32_t n, int64_t k, int splits) {
    p.m = m;
    p.n = n;
    p.m_tiles = ceil_div(m, shape_m(shape));
    p.n_tiles = ceil_div(n, shape_n(shape));
    p.k_blocks = ceil_div(k, kTileK);
    p.a_rows = rows_loaded(shape, m);
    p.splits = splits;
    p.items = p.m_tiles * p.n_tiles * splits;
}

template <int FOLD, bool PAIR, int N>
cudaError_t product_smem_ready() {
    constexpr int kDevices = 64;
    static std::atomic<bool> ready[kDevices];   // one array per kernel
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < kDevices && ready[dev].load())) return e;
    e = cudaFuncSetAttribute(product_kernel<FOLD, PAIR, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, kProductSmem);
    if (e == cudaSuccess && dev < kDevices) ready[dev].store(true);
    return e;
}

template <int FOLD, bool PAIR, int N>
cudaError_t launch_product_t(const LaunchEnv& env, const Product& p, cudaStream_t st) {
    if (cudaError_t e = product_smem_ready<FOLD, PAIR, N>(); e != cudaSuccess) return e;
    constexpr int kCtas = Tile<PAIR, N>::kCtas;
    const int at_once = std::max(1, env.num_sms / kCtas);
    return launch_cluster(product_kernel<FOLD, PAIR, N>, dim3((unsigned)(std::min(p.items, at_once) * kCtas)),
                          dim3(kProductThreads), kCtas, kProductSmem, st, p);
}
template <int FOLD>
cudaError_t launch_product(const LaunchEnv& env, Shape shape, const Product& p, cudaStream_t st) {
    if constexpr (FOLD != kFoldHidden)
        if (shape == kNarrow) return launch_product_t<FOLD, false, kNarrowN>(env, p, st);
    return shape == kPair ? launch_product_t<FOLD, true, kWideN>(env, p, st) : launch_product_t<FOLD, false, kWideN>(env, p, st);
}

cudaError_t launch_prep(const LaunchEnv& env, Prep& p, cudaStream_t st) {
    for (int i = 0; i < 2; ++i) {
        const Pack& k = p.pack[i];
        p.ctas[i] = (int)std::min<int64_t>((k.rows * (k.pitch / 8) + kPackThreads - 1) / kPackThreads, env.num_sms * 8);
    }
    return launch_pdl(prep_kernel, dim3((unsigned)(p.grad + p.ctas[0] + p.ctas[1])), dim3(kPackThreads), 0, st, p);
}

bool tma_ready(const void* p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0; }

// Where a call's parts lie in its workspace.
struct LossSpace {
    size_t hidden, weight, part, target_logit, coef, scale, grad, planes, end;
    int64_t pitch;        // of packed rows
    Shape logits, sums;   // the products' tiles
    int32_t part_pitch;
    int32_t piece;        // tokens of the vocabulary at a time (gradient)
    int32_t splits;       // of the hidden gradient's sum
    int32_t plane_rows;   // of each split's plane
};

// G takes at most this many bytes at a time.
constexpr int64_t kGradBytes = (int64_t)256 << 20;

// The tiles of the logits of `rows` rows and `n` tokens.  Pairs of CTAs have
// tiles of 256 rows: not where that leaves a quarter or more of the last of few
// tiles empty (GB300, us single / pairs, loss and gradient: 256 rows, V =
// 128256, 4096 wide 214, 641 / 192, 607; 300 rows, V = 32003, 1024 wide 23.1, 90 /
// 28.3, 93; 777 rows 37.9, 137 / 42.5, 134; 1024 rows, V = 65536 91.7, 277 / 79.1,
// 260; 2000 rows, V = 32003, 512 wide 60.0, 170 / 53.7, 169).  Rows off 128-byte
// lines (each of TMA's 128 bytes takes two lines) gain more by reading less: 777
// rows, 1000 wide 65.9, 167 / 62.0, 157.  Narrow tiles where every SM has at most one:
// a k block takes them nearly as long as wide ones (us wide / narrow: 300 rows, V =
// 2000, 256 wide 8.1, 21.1 / 6.3, 19.6; 64 rows, V = 8000, 4096 wide 23.6, 64.1 / 21.7,
// 54.2; two rounds of them, 64 rows, V = 12000, 512 wide 9.2, 28.0 / 12.0, 30.5).
Shape logits_shape(const LaunchEnv& env, int32_t rows, int64_t n, bool off_lines) {
    const int tiles = ceil_div(rows, kRowsM);
    if ((int64_t)tiles * ceil_div(n, kNarrowN) <= env.num_sms) return kNarrow;
    return tiles % 2 == 0 || tiles > 15 || (tiles > 1 && off_lines) ? kPair : kWide;
}

LossSpace loss_space(const LossArgs& a, const LaunchEnv& env, bool grad) {
    LossSpace s{};
    s.pitch = (a.dim + 7) / 8 * 8;
    size_t at = 0;
    const auto take = [&](size_t n) {
        const size_t p = at;
        at += align256(n);
        return p;
    };
    if (grad || !tma_ready(a.hidden, a.hidden_stride)) s.hidden = take((size_t)a.rows * s.pitch * 2);
    if (!tma_ready(a.weight, a.weight_stride)) s.weight = take((size_t)a.n_tokens * s.pitch * 2);
    if (!grad) {
        s.logits = logits_shape(env, a.rows, a.n_tokens, s.pitch % 64 != 0);
        s.part_pitch = ceil_div(a.n_tokens, shape_n(s.logits)) * (kFoldWarps / 4);
        s.part = take((size_t)a.rows * s.part_pitch * sizeof(float2));
        s.target_logit = take((size_t)a.rows * 4);
    } else {
        s.coef = take((size_t)a.rows * 4);
        s.scale = take(4);
        const int64_t most = std::max<int64_t>(kWideN, kGradBytes / 2 / a.rows / kWideN * kWideN);
        const int pieces = ceil_div(a.n_tokens, most);
        s.piece = ceil_div(ceil_div(a.n_tokens, pieces), kWideN) * kWideN;
        s.logits = logits_shape(env, a.rows, s.piece, s.pitch % 64 != 0);
        s.grad = take((size_t)a.rows * s.piece * 2);
        s.sums = a.rows > kRowsM ? kPair : kWide;
        // few tiles: their sums are split, each part into a plane of its own
        const int64_t tiles = (int64_t)ceil_div(a.rows, shape_m(s.sums)) * ceil_div(a.dim, kWideN);
        s.splits = (int)std::max<int64_t>(1, std::min<int64_t>(env.num_sms / (s.sums == kPair ? 2 : 1) / tiles, s.piece / kTileK / 2));
        s.plane_rows = ceil_div(a.rows, shape_m(s.sums)) * shape_m(s.sums);
        s.planes = take((size_t)s.splits * s.plane_rows * s.pitch * 4);
    }
    s.end = at;
    return s;
}

// The weight (and without a gradient the hidden rows) as TMA can read it: in place, or to be laid out by `prep`.
struct Operand {
    const void* p;
    int64_t stride;
};
Operand operand(Pack& pack, const void* p, int64_t stride, int32_t rows, int32_t cols, void* to, int64_t pitch, bool always) {
    const bool ready = tma_ready(p, stride);
    if (ready && !always) return {p, stride};
    pack = Pack{(const __nv_bfloat16*)p, stride, rows, cols, (__nv_bfloat16*)to, pitch, ready};
    return {to, pitch};
}

}  // namespace

size_t loss_workspace(const LossArgs& a, const LaunchEnv& env, bool grad) {
    return few_rows(a) ? few_workspace(a, env, grad) : loss_space(a, env, grad).end;
}

cudaError_t launch_loss_merge(const LossArgs& a, const float2* part, int32_t parts, const float* target_logit,
                              cudaStream_t st) {
    return launch_pdl(loss_kernel, dim3((unsigned)ceil_div(a.rows, kMergeThreads / 32)), dim3(kMergeThreads), 0, st, part,
                      parts, parts, target_logit, a.targets, a.mask, a.rows, a.n_tokens, a.loss, a.lse, a.err);
}

bool loss_fits(const LossArgs& a) {
    // tiles are counted in 32 bits
    return (int64_t)ceil_div(a.rows, kRowsM) * ceil_div(std::max(a.n_tokens, a.dim), kNarrowN) < ((int64_t)1 << 28);
}

cudaError_t launch_token_loss(const LossArgs& a, const LaunchEnv& env, void* space, cudaStream_t st) {
    if (few_rows(a)) return launch_few_loss(a, env, space, st);
    const LossSpace s = loss_space(a, env, false);
    char* ws = (char*)space;
    Prep prep{};
    const Operand h = operand(prep.pack[0], a.hidden, a.hidden_stride, a.rows, a.dim, ws + s.hidden, s.pitch, false);
    const Operand w = operand(prep.pack[1], a.weight, a.weight_stride, a.n_tokens, a.dim, ws + s.weight, s.pitch, false);
    cudaError_t e = cudaSuccess;
    if (prep.pack[0].rows || prep.pack[1].rows) e = launch_prep(env, prep, st);
    if (e != cudaSuccess) return e;
    Product p{};
    if ((e = make_map(&p.a, h.p, a.rows, a.dim, h.stride, rows_loaded(s.logits, a.rows))) != cudaSuccess) return e;
    if ((e = make_map(&p.b, w.p, a.n_tokens, a.dim, w.stride, shape_box(s.logits))) != cudaSuccess) return e;
    cut_product(p, s.logits, a.rows, a.n_tokens, a.dim, 1);
    p.mask = a.mask;
    p.mask_words = (a.n_tokens + 31) / 32;
    p.targets = a.targets;
    p.part = (float2*)(ws + s.part);
    p.part_pitch = s.part_pitch;
    p.target_logit = (float*)(ws + s.target_logit);
    p.err = a.err;
    e = p.k_blocks > kDeepBlocks ? launch_product<kFoldLogSumDeep>(env, s.logits, p, st)
                                 : launch_product<kFoldLogSum>(env, s.logits, p, st);
    if (e != cudaSuccess) return e;
    return launch_loss_merge(a, p.part, s.part_pitch, p.target_logit, st);
}

cudaError_t launch_token_loss_grad(const LossArgs& a, const LaunchEnv& env, void* space, cudaStream_t st) {
    if (few_rows(a)) return launch_few_loss_grad(a, env, space, st);
    const LossSpace s = loss_space(a, env, true);
    char* ws = (char*)space;
    Prep prep{};
    const Operand h = operand(prep.pack[0], a.hidden, a.hidden_stride, a.rows, a.dim, ws + s.hidden, s.pitch, true);
    const Operand w = operand(prep.pack[1], a.weight, a.weight_stride, a.n_tokens, a.dim, ws + s.weight, s.pitch, false);
    prep.grad = true;
    prep.targets = a.targets;
    prep.mask = a.mask;
    prep.grad_loss = a.grad_loss;
    prep.rows = a.rows;
    prep.n_tokens = a.n_tokens;
    prep.coef = (float*)(ws + s.coef);
    prep.scale = (float*)(ws + s.scale);
    prep.err = a.err;
    cudaError_t e = launch_prep(env, prep, st);
    if (e != cudaSuccess) return e;
    for (int32_t v0 = 0; v0 < a.n_tokens; v0 += s.piece) {
        const int32_t n = std::min(s.piece, a.n_tokens - v0), width = ceil_div(n, kWideN) * kWideN;
        const char* wp = (const char*)w.p + (int64_t)v0 * w.stride * 2;
        Product g{};   // G of the piece, [rows][width]
        if ((e = make_map(&g.a, h.p, a.rows, a.dim, h.stride, rows_loaded(s.logits, a.rows))) != cudaSuccess) return e;
        if ((e = make_map(&g.b, wp, n, a.dim, w.stride, shape_box(s.logits))) != cudaSuccess) return e;
        cut_product(g, s.logits, a.rows, n, a.dim, 1);
        g.mask = a.mask ? a.mask + v0 / 32 : nullptr;
        g.mask_words = (a.n_tokens + 31) / 32;
        g.targets = a.targets;
        g.column0 = v0;
        g.lse = a.lse;
        g.coef = prep.coef;
        if ((e = make_out_map(&g.to, ws + s.grad, a.rows, width, width)) != cudaSuccess) return e;
        g.err = a.err;
        if ((e = launch_product<kFoldGrad>(env, s.logits, g, st)) != cudaSuccess) return e;
        Product d{};   // its part of the hidden gradient
        if ((e = make_map(&d.a, ws + s.grad, a.rows, width, width, rows_loaded(s.sums, a.rows))) != cudaSuccess) return e;
        if ((e = make_map(&d.b, wp, n, a.dim, w.stride, 64)) != cudaSuccess) return e;
        cut_product(d, s.sums, a.rows, a.dim, n, s.splits);
        d.b_mn = 1;
        d.plane_rows = s.plane_rows;
        e = make_plane_map(&d.to, ws + s.planes, (int64_t)s.splits * s.plane_rows, a.dim, s.pitch);
        if (e != cudaSuccess) return e;
        d.add = v0 > 0;
        d.err = a.err;
        if ((e = launch_product<kFoldHidden>(env, s.sums, d, st)) != cudaSuccess) return e;
        // few tiles: the fold of a wide one, not its products, is the longer part (31 x 1760 x 219 8.5 us)
        const bool few = (int64_t)ceil_div(n, kRowsM) * ceil_div(a.dim, kNarrowN) <= env.num_sms;
        const Shape shape_w = few ? kNarrow : n > kRowsM ? kPair : kWide;
        Product g2{};   // the piece's rows of the weight's gradient
        if ((e = make_map(&g2.a, ws + s.grad, a.rows, width, width, 64)) != cudaSuccess) return e;
        if ((e = make_map(&g2.b, h.p, a.rows, a.dim, h.stride, 64)) != cudaSuccess) return e;
        cut_product(g2, shape_w, n, a.dim, a.rows, 1);
        g2.a_mn = g2.b_mn = 1;
        g2.a_rows = kRowsM;   // its loads are of 64 rows of m each
        __nv_bfloat16* rows = (__nv_bfloat16*)a.dweight + (int64_t)v0 * a.dweight_stride;
        if (tma_ready(a.dweight, a.dweight_stride)) {
            if ((e = make_out_map(&g2.to, rows, n, a.dim, a.dweight_stride)) != cudaSuccess) return e;
        } else {
            g2.out = rows;
            g2.ld = a.dweight_stride;
        }
        g2.scale = prep.scale;
        g2.err = a.err;
        if ((e = launch_product<kFoldWeight>(env, shape_w, g2, st)) != cudaSuccess) return e;
    }
    const int parts = s.splits >= 8 ? 8 : 1;
    const int64_t cells = (int64_t)a.rows * (s.pitch / 4);
    return launch_pdl(parts > 1 ? dhidden_kernel<8> : dhidden_kernel<1>,
                      dim3((unsigned)std::min<int64_t>(ceil_div(cells, kPackThreads / parts), env.num_sms * 8)),
                      dim3(kPackThreads), 0, st, (const float*)(ws + s.planes), s.splits, (int64_t)s.plane_rows * s.pitch, a.rows,
                      a.dim, (int32_t)s.pitch, (const float*)prep.scale, (__nv_bfloat16*)a.dhidden, a.dhidden_stride);
}

}  // namespace domino
