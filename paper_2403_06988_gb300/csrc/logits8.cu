// logits8.cu -- the logits of hidden states and a weight in e4m3 codes with a scale for
// each 128 values along a row, of one hidden row and of 128 weight rows (sm_103a):
//
//   x[t][v] = sum_b sh[t][b] sw[v / 128][b] sum_{k in b} h[t][k] w[v][k]     b: blocks of 128 k
//
// logits8_kernel  warp-specialised and persistent: TMA loads into a ring of swizzled
//                 tiles (128 k a row: a block), tcgen05.mma of a block's products into an
//                 accumulator in tensor memory of its own, and eight warps that add it,
//                 scaled, to sums in their registers while the next is filled.  A warp's
//                 columns lie in one block of 128 weight rows, so that a block of k costs
//                 each of its rows one scale.
//
// Few rows: bound by HBM (64 x 128256 x 4096 90 us, 6.2 TB/s).  Many: by the folds.  A block
// of 128 x 256 products takes the tensor cores 512 cycles, its 32 KB from L2 about 640, and
// the fold's 32768 fused products on 128 lanes 256, between waits that two warps a scheduler
// do not hide: 970 cycles in all (2048 x 38912 x 4096 252 us, 2.6 PFLOP/s; with a quarter of
// the fused products, timed alone, 214).  Larger calls are held by the power cap too: 2048 x
// 128256 x 4096 850 to 905 us, 2.4 to 2.5 PFLOP/s; of values that are nearly alike 800.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "norm.h"
#include "tcgen05.cuh"
#include "tensor_map.h"
#include "walk_common.cuh"

namespace domino {
namespace {

// Tiles: kRowsM rows of hidden states a CTA and N of the weight.  PAIR: two CTAs make 2 * kRowsM rows and hold half of
// the weight's each.
constexpr int kRowsM = 128, kTileK = 128, kWideN = 256, kHalfN = 128, kNarrowN = 64;
constexpr int kRingBytes = 196608;             // of operand tiles on their way
constexpr int kMaxStages = 16;                 // blocks of k of them
constexpr int kFoldWarps = 8;
// Warps that issue products, each every other accumulator's: one takes 980 cycles for a block's waits, products and commits
// (2048 x 38912 x 4096 281 us, with two of them 262).
constexpr int kIssuers = 2;
template <bool PAIR, int N>
struct Tile {
    static constexpr int kCtas = PAIR ? 2 : 1;
    static constexpr int kM = kRowsM * kCtas;
    // A block's products of 256 columns are made, and folded, in two parts, each in an accumulator of its own, so that a fold
    // has the time of three parts' products and not of one tile's (2048 x 38912 x 4096: 250 us, whole tiles in two
    // accumulators 273).
    static constexpr int kParts = N == kWideN ? 2 : 1, kPartN = N / kParts, kAccs = 4;
    static constexpr int kRowsB = N / kCtas;                // a CTA's
    static constexpr int kBytesB = kRowsB * kTileK;
    static constexpr int kColumns = N / (kFoldWarps / 4);   // a fold warp's: 32 rows, half of the columns
    static constexpr int kFolds = kFoldWarps / kParts;      // fold warps of a part
    static_assert(kColumns % 32 == 0 && 128 % kColumns == 0 && kAccs * kPartN <= 512);
};
// Registers of a thread: the fold warps' sums of 128 columns and what is on its way take more than an equal share (with 168
// for all, loads of 16 columns and none ahead: 273 us where this takes 250; sixteen warps of 64 columns 263; 216 for 224
// alike).  The shares' sum is within what the CTA is launched with (smem_ready looks).
constexpr int kFoldRegs = 224, kOtherRegs = 56;

// Results leave through shared memory: 32 rows of 64 bytes a warp's buffer, in the 64-byte swizzle.
constexpr int kOutBytes = 32 * 64, kOutBuffers = 2;
constexpr int kSmem8 = kRingBytes + kFoldWarps * kOutBuffers * kOutBytes + 1024;   // tiles lie on 1024-byte boundaries
constexpr int kThreads = 128 + 32 * kFoldWarps;
constexpr int kGroupM = 16;                    // row tiles that share a pass over the columns' tiles

struct Product8 {
    CUtensorMap a, b;
    CUtensorMap to;                // the logits, in boxes of 32 rows and 64 bytes
    int32_t m, n;
    int32_t m_tiles, n_tiles, k_blocks;
    int32_t a_rows;                // that a CTA loads, a multiple of 8: what lies behind them goes into rows that nothing uses
    int32_t items;                 // m_tiles * n_tiles
    const float* row_scales;       // [m][k_blocks]
    const float* column_scales;    // [ceil(n / 128)][k_blocks]
    void* out;                     // where `to` cannot be, rows off 16-byte boundaries
    int64_t ld;
    uint32_t* err;
};

struct Item {
    int32_t m, n;
};
// Row tiles in groups; in a group the columns' tiles one after the other, each with all of the group's row tiles.
__device__ __forceinline__ Item item_at(const Product8& p, int32_t i) {
    Item t;
    const int32_t group = i / (kGroupM * p.n_tiles);
    const int32_t m0 = group * kGroupM, rows = min(kGroupM, p.m_tiles - m0);
    i -= group * kGroupM * p.n_tiles;
    t.n = i / rows;
    t.m = m0 + i - t.n * rows;
    return t;
}

// x + c v of two values, each rounded once
__device__ __forceinline__ float2 add_scaled(float2 x, float2 v, float c) {
    unsigned long long a, b, d, r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(a) : "f"(v.x), "f"(v.y));
    asm("mov.b64 %0, {%1, %1};" : "=l"(b) : "f"(c));
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x.x), "f"(x.y));
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(d));
    float2 o;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(o.x), "=f"(o.y) : "l"(r));
    return o;
}

// 64 bytes of each of 32 rows, the first at (x, y), x in values.
template <bool BF16>
__device__ __forceinline__ void put_out(const Product8& p, int32_t x, int32_t y, uint32_t buffers, uint32_t puts, int lane,
                                        const uint32_t (&w)[16]) {
    const uint32_t buffer = buffers + (puts % kOutBuffers) * kOutBytes;
    if (!p.out) {
        if (lane == 0) tma_wait_read<kOutBuffers - 1>();   // the copy from this buffer before
        __syncwarp();
        put_words(buffer, lane, w);
        tma_fence();
        __syncwarp();
        if (lane == 0) {
            tma_store(&p.to, x, y, buffer);
            tma_commit();
        }
        return;
    }
    // a row after the other (fp32: two), a column a lane
    __syncwarp();
    put_words(buffer, lane, w);
    __syncwarp();
    constexpr int kCols = BF16 ? 32 : 16, kAtOnce = 32 / kCols;
    const int col = lane % kCols, sub = lane / kCols;
    const uint32_t chunk = (uint32_t)col * (BF16 ? 2 : 4) >> 4, byte = (uint32_t)col * (BF16 ? 2 : 4) & 15u;
    const int64_t at = (int64_t)y * p.ld + x + col;
    const int rows = x + col < p.n ? min(32, p.m - y) : 0;
#pragma unroll 8
    for (int r0 = 0; r0 < 32; r0 += kAtOnce) {
        const int r = r0 + sub;
        const uint32_t from = buffer + r * 64 + ((chunk ^ ((r >> 1) & 3)) << 4) + byte;
        if constexpr (BF16) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(v) : "r"(from));
            if (r < rows) static_cast<uint16_t*>(p.out)[at + r * p.ld] = v;
        } else {
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(v) : "r"(from));
            if (r < rows) static_cast<uint32_t*>(p.out)[at + r * p.ld] = v;
        }
    }
}

template <bool BF16, bool PAIR, int N>
__global__ void __launch_bounds__(kThreads, 1) logits8_kernel(const __grid_constant__ Product8 p) {
    using T = Tile<PAIR, N>;
    constexpr int kColumns = T::kColumns, kAccs = T::kAccs, kTmemColumns = kAccs * T::kPartN;
    extern __shared__ unsigned char smem[];
    __shared__ __align__(8) uint64_t s_full[kMaxStages], s_empty[kMaxStages], s_acc_full[kAccs], s_acc_empty[kAccs], s_done;
    __shared__ uint32_t s_tmem, s_failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tiles = (smem_addr(smem) + 1023u) & ~1023u;
    const uint32_t rank = PAIR ? cluster_rank() : 0u;
    const int32_t first = blockIdx.x / T::kCtas, step = gridDim.x / T::kCtas;   // items of this CTA or pair
    volatile uint32_t* failed = &s_failed;
    const uint32_t bytes_a = p.a_rows * kTileK, stage_bytes = bytes_a + T::kBytesB;
    const uint32_t stages = min((uint32_t)kMaxStages, kRingBytes / stage_bytes);
    if (threadIdx.x == 0) {
        s_failed = 0u;
        for (int s = 0; s < kMaxStages; ++s) {
            bar_init(smem_addr(&s_full[s]), 1);
            bar_init(smem_addr(&s_empty[s]), T::kParts);
        }
        for (int s = 0; s < kAccs; ++s) {
            bar_init(smem_addr(&s_acc_full[s]), 1);
            bar_init(smem_addr(&s_acc_empty[s]), T::kFolds * T::kCtas);
        }
        bar_init(smem_addr(&s_done), kIssuers);
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

    if (warp < 4) {
        if constexpr (T::kParts == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kOtherRegs));
        if (warp == 0) {   // ---- loads: each CTA its part of the tiles; the first CTA's barriers count the bytes of both
            uint32_t s = 0, turn = 0, loads = 0;   // the stage, how often the ring has come round
            bool ok = true;
            for (int32_t i = first; i < p.items && ok; i += step) {
                const Item t = item_at(p, i);
                const int32_t row_a = t.m * T::kM + rank * kRowsM, row_b = t.n * N;
                for (int32_t k = 0; k < p.k_blocks; ++k) {
                    if (!(ok = warp_wait(smem_addr(&s_empty[s]), (turn & 1u) ^ 1u, failed))) break;
                    const uint32_t mine = smem_addr(&s_full[s]), a = tiles + s * stage_bytes;
                    const uint32_t full = PAIR ? in_cta(mine, 0) : mine;
                    if (elect_lane()) {
                        if (rank == 0) bar_expect(mine, stage_bytes * T::kCtas);
                        tma_load<PAIR>(a, &p.a, k * kTileK, row_a, full);
                        if constexpr (PAIR) {   // half of each part's rows
    #pragma unroll
                            for (int h = 0; h < T::kParts; ++h)
                                tma_load<PAIR>(a + bytes_a + h * (T::kBytesB / T::kParts), &p.b, k * kTileK,
                                               row_b + h * T::kPartN + rank * (T::kPartN / 2), full);
                        } else {
                            tma_load<PAIR>(a + bytes_a, &p.b, k * kTileK, row_b, full);
                        }
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
        } else if (warp <= kIssuers) {   // ---- products: a part of a block of k each an accumulator
            if (rank == 0) {
                constexpr uint32_t desc = mma_desc8(T::kM, T::kPartN);
                // the warp's: every kIssuers-th accumulator, of the same part of every block where there are two
                const int64_t blocks = (int64_t)((p.items - first + step - 1) / step) * p.k_blocks;
                const uint32_t h = T::kParts == 2 ? warp - 1 : 0;
                constexpr uint32_t kStep = kIssuers / T::kParts;
                uint32_t s = T::kParts == 2 ? 0 : warp - 1, turn = 0, u = warp - 1;
                for (int64_t block = s; block < blocks; block += kStep, u += kIssuers) {
                    if (s >= stages) {
                        s -= stages;
                        ++turn;
                    }
                    const uint32_t s_acc = u % kAccs, acc = tmem + s_acc * T::kPartN;
                    if (!warp_wait(smem_addr(&s_acc_empty[s_acc]), ((u / kAccs) & 1u) ^ 1u, failed)) break;
                    if (!warp_wait(smem_addr(&s_full[s]), turn & 1u, failed)) break;
                    tcgen_after();
                    const uint64_t a = operand_desc(tiles + s * stage_bytes, 0);
                    const uint64_t b = operand_desc(tiles + s * stage_bytes + bytes_a + h * (T::kBytesB / T::kParts), 0);
                    if (elect_lane()) {
    #pragma unroll
                        for (int j = 0; j < kTileK / 32; ++j)   // 32 k: 32 bytes further, in 16-byte units
                            mma_e4m3<PAIR>(acc, a + (uint64_t)(j * 2), b + (uint64_t)(j * 2), desc, j > 0);
                        mma_commit<PAIR>(smem_addr(&s_acc_full[s_acc]));
                        mma_commit<PAIR>(smem_addr(&s_empty[s]));
                    }
                    s += kStep;
                }
                if (elect_lane()) mma_commit<PAIR>(smem_addr(&s_done));
            }
            // no product, and no arrival at a barrier of this CTA, may be on its way when the CTA ends
            if (lane == 0) {
                const uint64_t end = timer_ns() + 3 * kWaitNs;
                while (!bar_try(smem_addr(&s_done), 0u) && timer_ns() < end) {}
            }
        }
    } else {   // ---- folds
        if constexpr (T::kParts == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kFoldRegs));
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t buffers = tiles + kRingBytes + (warp - 4) * kOutBuffers * kOutBytes;
        const int row_in_tile = rank * kRowsM + quarter * 32 + lane;
        uint32_t accs = 0, puts = 0;
        bool ok = true;
        for (int32_t i = first; i < p.items; i += step) {
            const Item t = item_at(p, i);
            const int32_t row = t.m * T::kM + row_in_tile, row0 = row - lane, c0 = t.n * N + half * kColumns;
            const bool some = row0 < p.m && c0 < p.n;   // of the warp's
            const float* rs = p.row_scales + (int64_t)min(row, p.m - 1) * p.k_blocks;
            const float* cs = p.column_scales + (int64_t)(min(c0, p.n - 1) / 128) * p.k_blocks;
            float2 x[kColumns / 2];
#pragma unroll
            for (int e = 0; e < kColumns / 2; ++e) x[e] = make_float2(0.0f, 0.0f);
            float next_r = __ldg(rs), next_c = __ldg(cs);
            for (int32_t k = 0; k < p.k_blocks; ++k) {
                const float c = next_r * next_c;
                if (k + 1 < p.k_blocks) {
                    next_r = __ldg(rs + k + 1);
                    next_c = __ldg(cs + k + 1);
                }
                // the block's accumulator: of the warp's half where there are two
                const uint32_t turns = accs * T::kParts + (T::kParts == 2 ? half : 0), s_acc = turns % kAccs;
                ++accs;
                if (!(ok = warp_wait(smem_addr(&s_acc_full[s_acc]), (turns / kAccs) & 1u, failed))) break;
                tcgen_after();
                const uint32_t acc = tmem + s_acc * T::kPartN + (T::kParts == 2 ? 0 : half * kColumns) + ((uint32_t)(quarter * 32) << 16);
                const auto emptied = [&] {
                    tcgen_before();
                    __syncwarp();
                    if (lane == 0) {
                        const uint32_t bar = smem_addr(&s_acc_empty[s_acc]);
                        if constexpr (PAIR) bar_arrive_cluster(in_cta(bar, 0));
                        else bar_arrive(bar);
                    }
                };
                if (!some) {
                    emptied();
                    continue;
                }
                // 32 columns are added while the next are on their way
                uint32_t v[2][32];
                tmem_fetch32(v[0], acc);
#pragma unroll
                for (int j = 0; j < kColumns / 32; ++j) {
                    tmem_wait32(v[j & 1]);
                    if (j + 1 < kColumns / 32) tmem_fetch32(v[(j + 1) & 1], acc + 32 * (j + 1));
                    else emptied();
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        x[16 * j + e] = add_scaled(x[16 * j + e], make_float2(__uint_as_float(v[j & 1][2 * e]), __uint_as_float(v[j & 1][2 * e + 1])), c);
                }
            }
            if (!ok) break;
            if (!some) continue;
#pragma unroll
            for (int j = 0; j < kColumns; j += BF16 ? 32 : 16) {
                if (c0 + j >= p.n) break;
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if constexpr (BF16) {
                        const __nv_bfloat162 v = __floats2bfloat162_rn(x[j / 2 + e].x, x[j / 2 + e].y);
                        w[e] = *reinterpret_cast<const uint32_t*>(&v);
                    } else {
                        w[e] = __float_as_uint(e & 1 ? x[(j + e) / 2].y : x[(j + e) / 2].x);
                    }
                }
                put_out<BF16>(p, c0 + j, row0, buffers, puts++, lane, w);
            }
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

// ---- host ----------------------------------------------------------------------
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

enum Shape : int { kPair = 0, kWide = 1, kNarrow = 2, kHalf = 3 };   // 256 x 256 of two CTAs, 128 x 256, 128 x 64, 128 x 128
int shape_m(Shape s) { return s == kPair ? 2 * kRowsM : kRowsM; }
int shape_n(Shape s) { return s == kNarrow ? kNarrowN : s == kHalf ? kHalfN : kWideN; }
int shape_box(Shape s) { return s == kWide ? kWideN : s == kPair ? kWideN / 4 : s == kHalf ? kHalfN : kNarrowN; }   // rows of the weight of a load

// Narrow tiles where every SM has at most one (us narrow / wide: 1 x 1000 x 64 3.0, 4.9; 128 x 8000 x 4096 11.6, 19.7; more
// than one round of them, 64 x 32000 x 1024 13.5, 10.7; 64 x 128256 x 4096 111, 97).  Up to 128 rows are bound by the bytes
// that all SMs together read: tiles of 128 columns where their last round is the shorter one (us wide / half: 64 x 128256 x
// 4096 97, 90; 1 x 50000 x 512 12.9, 11.6; else 100 x 30000 x 4096 27.8, 30.0).  Pairs read two thirds of the bytes
// from L2; not where they leave a quarter or more of few tiles' rows empty (us pair / wide: 2048 x 38912 x 4096 250, 258;
// 390 x 100000 x 2048 94, 97; 256 rows alike; 300 x 32000 x 1024 24, 19; 777 x 50000 x 1024 57, 54).
Shape shape_of(const Logits8Args& a, const LaunchEnv& env) {
    const int tiles = ceil_div(a.rows, kRowsM);
    if ((int64_t)tiles * ceil_div(a.n_tokens, kNarrowN) <= env.num_sms) return kNarrow;
    if (tiles == 1 && ceil_div(ceil_div(a.n_tokens, kHalfN), env.num_sms) < 2 * ceil_div(ceil_div(a.n_tokens, kWideN), env.num_sms))
        return kHalf;
    return tiles % 2 == 0 || tiles > 15 ? kPair : kWide;
}

cudaError_t make_map8(CUtensorMap* map, const uint8_t* base, int64_t rows, int64_t cols, int64_t pitch, int box_rows) {
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, base, rows, cols, pitch, kTileK, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <bool BF16, bool PAIR, int N>
cudaError_t smem_ready() {
    constexpr int kDevices = 64;
    static std::atomic<bool> ready[kDevices];   // one array per kernel
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < kDevices && ready[dev].load())) return e;
    e = cudaFuncSetAttribute(logits8_kernel<BF16, PAIR, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem8);
    cudaFuncAttributes attr;
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&attr, logits8_kernel<BF16, PAIR, N>);
    // a CTA launched with fewer registers than its warps' shares would wait for ever
    if (e == cudaSuccess && Tile<PAIR, N>::kParts == 2 && attr.numRegs * kThreads < kFoldRegs * 32 * kFoldWarps + kOtherRegs * 128)
        e = cudaErrorLaunchOutOfResources;
    if (e == cudaSuccess && dev < kDevices) ready[dev].store(true);
    return e;
}

template <bool BF16, bool PAIR, int N>
cudaError_t launch_t(const LaunchEnv& env, const Product8& p, cudaStream_t st) {
    if (cudaError_t e = smem_ready<BF16, PAIR, N>(); e != cudaSuccess) return e;
    constexpr int kCtas = Tile<PAIR, N>::kCtas;
    const int at_once = std::max(1, env.num_sms / kCtas);
    return launch_cluster(logits8_kernel<BF16, PAIR, N>, dim3((unsigned)(std::min(p.items, at_once) * kCtas)), dim3(kThreads), kCtas,
                          kSmem8, st, p);
}
template <bool BF16>
cudaError_t launch_shape(const LaunchEnv& env, Shape shape, const Product8& p, cudaStream_t st) {
    if (shape == kNarrow) return launch_t<BF16, false, kNarrowN>(env, p, st);
    if (shape == kHalf) return launch_t<BF16, false, kHalfN>(env, p, st);
    return shape == kPair ? launch_t<BF16, true, kWideN>(env, p, st) : launch_t<BF16, false, kWideN>(env, p, st);
}

}  // namespace

bool logits8_fits(const Logits8Args& a) {
    // tiles are counted in 32 bits
    return (int64_t)ceil_div(a.rows, kRowsM) * ceil_div(a.n_tokens, kNarrowN) < ((int64_t)1 << 28);
}

cudaError_t launch_logits8(const Logits8Args& a, const LaunchEnv& env, cudaStream_t st) {
    const Shape shape = shape_of(a, env);
    const bool bf16 = a.dtype == DOMINO_DTYPE_BF16;
    const int size = bf16 ? 2 : 4;
    Product8 p{};
    p.m = a.rows;
    p.n = a.n_tokens;
    p.m_tiles = ceil_div(a.rows, shape_m(shape));
    p.n_tiles = ceil_div(a.n_tokens, shape_n(shape));
    p.k_blocks = ceil_div(a.dim, kTileK);
    p.a_rows = shape == kPair ? kRowsM : std::min(kRowsM, (a.rows + 7) / 8 * 8);
    p.items = p.m_tiles * p.n_tiles;
    p.row_scales = a.hidden_scales;
    p.column_scales = a.weight_scales;
    p.err = a.err;
    cudaError_t e = make_map8(&p.a, a.hidden, a.rows, a.dim, a.hidden_stride, p.a_rows);
    if (e == cudaSuccess) e = make_map8(&p.b, a.weight, a.n_tokens, a.dim, a.weight_stride, shape_box(shape));
    if (e != cudaSuccess) return e;
    if (reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.logits_stride * size % 16 == 0) {
        e = encode_map(&p.to, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, size, a.logits, a.rows,
                       a.n_tokens, a.logits_stride, 64 / size, 32, CU_TENSOR_MAP_SWIZZLE_64B);
        if (e != cudaSuccess) return e;
    } else {
        p.out = a.logits;
        p.ld = a.logits_stride;
    }
    return bf16 ? launch_shape<true>(env, shape, p, st) : launch_shape<false>(env, shape, p, st);
}

}  // namespace domino
