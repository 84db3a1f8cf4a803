// quantize8.cu -- a matrix in e4m3 codes with a scale for each 1 x 128 or 128 x 128
// values (sm_103a): rows of hidden states that do not come from a norm in codes, or a
// weight.  Bound by HBM: a value is read once and kept until its block's largest is known.
#include <algorithm>

#include "norm.h"
#include "values8.cuh"

namespace domino {
namespace {

constexpr int kThreads8 = 256;
constexpr int kHalves = kThreads8 / kBlockLanes;     // of a CTA: sixteen lanes take 128 values of a row
constexpr int kTogether8 = 4;                        // pieces of 128 values of sixteen lanes, read together
constexpr int kTileRows = 128, kPerHalf = kTileRows / kHalves;
constexpr int64_t kFarCodes = (int64_t)64 << 20;

template <bool BF16, bool ALIGNED>
__global__ void __launch_bounds__(kThreads8) rows_kernel(const __grid_constant__ Quantize8Args a, const int64_t pieces, const bool far) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & (kBlockLanes - 1), half = threadIdx.x / kBlockLanes;
    const int32_t blocks = (a.dim + kBlock8 - 1) / kBlock8;
    Vec8<BF16, ALIGNED> v[kTogether8];
    int32_t row[kTogether8], c[kTogether8];
#pragma unroll
    for (int j = 0; j < kTogether8; ++j) {
        const int64_t i = ((int64_t)blockIdx.x * kTogether8 + j) * kHalves + half;
        row[j] = (int32_t)(pieces <= UINT_MAX ? (uint32_t)i / (uint32_t)blocks : i / blocks);
        c[j] = i < pieces ? (int32_t)(i - (int64_t)row[j] * blocks) * kBlock8 + lane * kN : a.dim;
        v[j].load((const char*)a.x + row[j] * a.stride * (BF16 ? 2 : 4), c[j], a.dim);
    }
#pragma unroll
    for (int j = 0; j < kTogether8; ++j) {
        float f[kN];
        v[j].get(f);
        const float top = fmaxf(block_largest(largest(f)), kLeast8);
        if (c[j] >= a.dim) continue;
        if (lane == 0) a.scales[(int64_t)row[j] * blocks + c[j] / kBlock8] = scale_of(top);
        store_codes(a.codes + row[j] * a.codes_stride, c[j], a.dim, f, kMost8 / top, far);
    }
}

// A tile of 128 rows and 128 columns a CTA.
template <bool BF16, bool ALIGNED>
__global__ void __launch_bounds__(kThreads8) tiles_kernel(const __grid_constant__ Quantize8Args a, const bool far) {
    __shared__ float s_top[kThreads8 / 32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & (kBlockLanes - 1), half = threadIdx.x / kBlockLanes;
    const int32_t blocks = (a.dim + kBlock8 - 1) / kBlock8;
    const int32_t tile = blockIdx.x / blocks, block = blockIdx.x - tile * blocks;
    const int32_t c = block * kBlock8 + lane * kN;
    Vec8<BF16, ALIGNED> v[kPerHalf];
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < kPerHalf; ++j) {
        const int64_t row = (int64_t)tile * kTileRows + j * kHalves + half;
        v[j].load((const char*)a.x + row * a.stride * (BF16 ? 2 : 4), c, row < a.rows ? a.dim : 0);
    }
#pragma unroll
    for (int j = 0; j < kPerHalf; ++j) {
        float f[kN];
        v[j].get(f);
        v[j].keep();
        top = fmaxf(top, largest(f));
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads8 / 32; ++w) top = fmaxf(top, s_top[w]);
    top = fmaxf(top, kLeast8);
    if (threadIdx.x == 0) a.scales[(int64_t)tile * blocks + block] = scale_of(top);
    const float by = kMost8 / top;
#pragma unroll
    for (int j = 0; j < kPerHalf; ++j) {
        const int64_t row = (int64_t)tile * kTileRows + j * kHalves + half;
        float f[kN];
        v[j].get(f);
        if (row < a.rows) store_codes(a.codes + row * a.codes_stride, c, a.dim, f, by, far);
    }
}

template <bool BF16, bool ALIGNED>
cudaError_t launch_t(const Quantize8Args& a, cudaStream_t st) {
    const bool far = (int64_t)a.rows * a.dim >= kFarCodes;
    const int64_t blocks = (a.dim + kBlock8 - 1) / kBlock8;
    if (a.block == 1) {
        const int64_t pieces = a.rows * blocks, per_cta = kHalves * kTogether8;
        return launch_pdl(rows_kernel<BF16, ALIGNED>, dim3((unsigned)((pieces + per_cta - 1) / per_cta)), dim3(kThreads8), 0, st, a,
                          pieces, far);
    }
    const int64_t tiles = (a.rows + (int64_t)kTileRows - 1) / kTileRows;
    return launch_pdl(tiles_kernel<BF16, ALIGNED>, dim3((unsigned)(tiles * blocks)), dim3(kThreads8), 0, st, a, far);
}

}  // namespace

cudaError_t launch_quantize8(const Quantize8Args& a, const LaunchEnv&, cudaStream_t st) {
    const bool aligned = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.stride * (a.dtype == DOMINO_DTYPE_BF16 ? 2 : 4) % 16 == 0;
    if (a.dtype == DOMINO_DTYPE_BF16) return aligned ? launch_t<true, true>(a, st) : launch_t<true, false>(a, st);
    return aligned ? launch_t<false, true>(a, st) : launch_t<false, false>(a, st);
}

}  // namespace domino
