// loss_few.cu -- the cross entropy of loss.cu and its gradient for up to four
// rows of tokens (scoring single tokens, the smallest training steps).  With
// so few rows the products are bound by reading the weight (and writing its
// gradient) once, which the tensor cores' 128-row tiles would not speed up:
// the dot products run in fp32 on the CUDA cores, and weight rows that no
// row's mask allows are not read.
//
// few_logits_kernel  a warp takes a block of tokens against all rows: 32 sums
//                    a lane, which one transposing reduction over the lanes
//                    turns into one logit a lane.  Folded into (max, sum of exp), or
//                    into G (fp32).
// few_sums_kernel    a thread keeps eight columns: over a strip of tokens it adds
//                    G w to its sums and writes G^T h.
// few_hidden_kernel  the strips' sums, in their order.
#include <cuda_bf16.h>

#include <algorithm>

#include "bf16_rows.cuh"
#include "decode.cuh"
#include "loss.h"

namespace domino {
namespace {

constexpr int kFewThreads = 256, kFewWarps = kFewThreads / 32;
constexpr int kFewLoads = 8;              // of a lane in flight

struct FewCall {
    LossArgs a;
    int64_t mask_words;
    int32_t block, blocks;                // tokens a warp takes at a time
    bool grad;
    float2* part;                         // [rows][gridDim.x]
    float* target_logit;                  // [rows]
    float* g;                             // [rows][n_tokens]
};

// Eight consecutive bf16 of a row as fp32, zeros beyond the row's end.  ALIGNED:
// rows begin on 16-byte boundaries and have whole vectors.  Else they are read in
// the 16-byte blocks that hold the values, and shifted.
template <bool ALIGNED>
struct Cols : Eight {};
template <>
struct Cols<true> {
    uint4 u;
    __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int32_t) { u = __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void get(float (&f)[kN]) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
};

// Sums over the warp of 32 values a lane: value l comes out in lane l.
__device__ __forceinline__ float transpose_sum(float (&acc)[32], int lane) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
        const bool up = lane & s;
#pragma unroll
        for (int i = 0; i < s; ++i) {
            const float keep = up ? acc[i + s] : acc[i], send = up ? acc[i] : acc[i + s];
            acc[i] = keep + __shfl_xor_sync(0xffffffffu, send, s);
        }
    }
    return acc[0];
}

// TN rows of tokens (those beyond the call's are not read).  ROWS: weight rows read together, 1 (blocks of one token, the
// loads unrolled along the row), 4, or 8 (rows of up to 256 values).
template <int TN, int ROWS, bool ALIGNED>
__global__ void __launch_bounds__(kFewThreads, 2) few_logits_kernel(const __grid_constant__ FewCall c) {
    constexpr int kR = 32 / TN;                              // lane l: row l / kR, token l % kR of the block
    constexpr bool SINGLE = ROWS == 1;
    constexpr int kRows = ROWS, kLoads = ALIGNED ? kFewLoads : kFewLoads / 2, kSteps = kLoads > kRows ? kLoads / kRows : 1;
    __shared__ float2 s_part[kFewWarps][TN];
    const LossArgs& a = c.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t = lane / kR, r = lane % kR;
    const __nv_bfloat16* hidden = (const __nv_bfloat16*)a.hidden;
    const __nv_bfloat16* weight = (const __nv_bfloat16*)a.weight;
    pdl_wait();
    pdl_trigger();
    const bool row_on = t < a.rows;
    const uint32_t* mrow = a.mask && row_on ? a.mask + t * c.mask_words : nullptr;
    int32_t target = row_on ? __ldg(a.targets + t) : -1;
    float coef = 0.0f, lse = 0.0f;
    if (target >= a.n_tokens) {
        if (blockIdx.x == 0 && warp == 0 && c.grad) atomicOr(a.err, DOMINO_DEVERR_BAD_TOKEN);
        target = -1;
    }
    if (c.grad && target >= 0 && (!mrow || (__ldg(mrow + (target >> 5)) >> (target & 31)) & 1u)) {
        coef = __ldg(a.grad_loss + t);
        lse = a.lse[t];
    }
    const bool use = row_on && (!c.grad || coef != 0.0f);
    float m = -INFINITY, sum = 0.0f;
    for (int32_t b = blockIdx.x * kFewWarps + warp; b < c.blocks; b += gridDim.x * kFewWarps) {
        const int32_t v0 = b * c.block, v = v0 + r;
        const bool here = row_on && r < c.block && v < a.n_tokens;
        const bool ok = here && use && (!mrow || (__ldg(mrow + (v >> 5)) >> (v & 31)) & 1u);
        uint32_t need = __ballot_sync(0xffffffffu, ok);      // of the block's tokens, by any row
#pragma unroll
        for (int k = kR; k < 32; k <<= 1) need |= need >> k;
        if (kR < 32) need &= (1u << (kR & 31)) - 1u;
        float acc[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
#pragma unroll
        for (int r0 = 0; r0 < (SINGLE ? 1 : kR); r0 += kRows) {
            if (!((need >> r0) & ((1u << kRows) - 1u))) continue;
            for (int32_t c0 = lane * kN; c0 < a.dim; c0 += 32 * kN * kSteps) {
                Cols<ALIGNED> w[kSteps][kRows];
#pragma unroll
                for (int u = 0; u < kSteps; ++u)
#pragma unroll
                    for (int k = 0; k < kRows; ++k) {
                        const int32_t at = c0 + u * 32 * kN;
                        w[u][k].zero();
                        if (at < a.dim && ((need >> (r0 + k)) & 1u))
                            w[u][k].load(weight + (int64_t)(v0 + r0 + k) * a.weight_stride + at, a.dim - at);
                    }
#pragma unroll
                for (int u = 0; u < kSteps; ++u) {
                    const int32_t at = c0 + u * 32 * kN;
                    if (at >= a.dim) break;
                    Cols<ALIGNED> h[TN];
#pragma unroll
                    for (int i = 0; i < TN; ++i) {
                        h[i].zero();
                        if (i < a.rows) h[i].load(hidden + i * a.hidden_stride + at, a.dim - at);
                    }
                    float x[kRows][kN];
#pragma unroll
                    for (int k = 0; k < kRows; ++k) w[u][k].get(x[k]);
#pragma unroll
                    for (int i = 0; i < TN; ++i) {
                        float y[kN];
                        h[i].get(y);
#pragma unroll
                        for (int k = 0; k < kRows; ++k)
#pragma unroll
                            for (int e = 0; e < kN; ++e) acc[i * kR + r0 + k] = fmaf(x[k][e], y[e], acc[i * kR + r0 + k]);
                    }
                }
            }
        }
        float x = 0.0f;
        if (need) {
            if constexpr (SINGLE) {
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    float s = acc[i * kR];
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
                    x = t == i ? s : x;
                }
            } else {
                x = transpose_sum(acc, lane);
            }
        }
        if (c.grad) {
            if (here) c.g[(int64_t)t * a.n_tokens + v] = ok ? coef * (exp_diff(x, lse) - (v == target ? 1.0f : 0.0f)) : 0.0f;
        } else if (ok) {
            const float m2 = fmaxf(m, x), ref = sum_ref(m2);
            sum = sum * exp_diff(m, ref) + exp_diff(x, ref);
            m = m2;
            if (v == target) c.target_logit[t] = x;
        }
    }
    if (c.grad) return;
    const auto merge = [&](float mo, float so) {
        const float m2 = fmaxf(m, mo), ref = sum_ref(m2);
        sum = sum * exp_diff(m, ref) + so * exp_diff(mo, ref);
        m = m2;
    };
#pragma unroll
    for (int off = kR / 2; off > 0; off >>= 1)
        merge(__shfl_xor_sync(0xffffffffu, m, off), __shfl_xor_sync(0xffffffffu, sum, off));
    if (r == 0) s_part[warp][t] = make_float2(m, sum);
    __syncthreads();
    if (warp == 0 && r == 0 && row_on) {
        for (int k = 1; k < kFewWarps; ++k) merge(s_part[k][t].x, s_part[k][t].y);
        c.part[(int64_t)t * gridDim.x + blockIdx.x] = make_float2(m, sum);
    }
}

constexpr int kSumsThreads = 128;          // at most: a warp per 256 columns
constexpr int kSumsTokens = 64;           // whose G lies in shared memory at a time
constexpr int kSumsLoads = 8;

struct FewSums {
    LossArgs a;
    const float* g;                       // [rows][n_tokens]
    int32_t strip;                        // tokens of a CTA
    int32_t pitch;                        // of the planes' rows, a multiple of kN
    float* planes;                        // [strips][rows][pitch]
    bool aligned_out;
};

template <int TN, bool ALIGNED>
__global__ void __launch_bounds__(kSumsThreads) few_sums_kernel(const __grid_constant__ FewSums c) {
    __shared__ float s_g[kSumsTokens][TN];
    const LossArgs& a = c.a;
    const __nv_bfloat16* weight = (const __nv_bfloat16*)a.weight;
    __nv_bfloat16* dweight = (__nv_bfloat16*)a.dweight;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int32_t col = (blockIdx.y * blockDim.x + threadIdx.x) * kN, left = a.dim - col;
    const bool on = left > 0;
    const int32_t lo = blockIdx.x * c.strip, hi = min(a.n_tokens, lo + c.strip);
    // rows without a gradient have no part in dweight, whatever they hold: their G is 0
    float h[TN][kN], acc[TN][kN];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int e = 0; e < kN; ++e) h[i][e] = acc[i][e] = 0.0f;
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        if (i >= a.rows || !on) break;
        const int32_t y = __ldg(a.targets + i);
        const bool given = y >= 0 && y < a.n_tokens &&
                           (!a.mask || (__ldg(a.mask + (int64_t)i * ((a.n_tokens + 31) / 32) + (y >> 5)) >> (y & 31)) & 1u);
        if (given && __ldg(a.grad_loss + i) != 0.0f) {
            Cols<ALIGNED> x;
            x.load((const __nv_bfloat16*)a.hidden + i * a.hidden_stride + col, left);
            x.get(h[i]);
        }
    }
    constexpr int kLoads = ALIGNED ? kSumsLoads : kSumsLoads / 2;
    for (int32_t v0 = lo; v0 < hi; v0 += kSumsTokens) {
        __syncthreads();
        for (int k = threadIdx.x; k < kSumsTokens * TN; k += blockDim.x) {
            const int i = k / kSumsTokens, v = k - i * kSumsTokens;
            s_g[v][i] = i < a.rows && v0 + v < hi ? c.g[(int64_t)i * a.n_tokens + v0 + v] : 0.0f;
        }
        __syncthreads();
        const int n = min(kSumsTokens, hi - v0);
        for (int k0 = 0; k0 < n; k0 += kLoads) {
            Cols<ALIGNED> w[kLoads];
            uint32_t any = 0;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                w[j].zero();
                if (k0 + j < n) {
                    bool some = false;
#pragma unroll
                    for (int i = 0; i < TN; ++i) some |= s_g[k0 + j][i] != 0.0f;
                    any |= (some ? 1u : 0u) << j;
                    if (some && on) w[j].load(weight + (int64_t)(v0 + k0 + j) * a.weight_stride + col, left);
                }
            }
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                if (k0 + j >= n) break;
                float out[kN];
#pragma unroll
                for (int e = 0; e < kN; ++e) out[e] = 0.0f;
                if ((any >> j) & 1u) {
                    float x[kN];
                    w[j].get(x);
#pragma unroll
                    for (int i = 0; i < TN; ++i) {
                        const float g = s_g[k0 + j][i];
#pragma unroll
                        for (int e = 0; e < kN; ++e) {
                            acc[i][e] = fmaf(g, x[e], acc[i][e]);
                            out[e] = fmaf(g, h[i][e], out[e]);
                        }
                    }
                }
                uint32_t o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __nv_bfloat162 p = __floats2bfloat162_rn(out[2 * e], out[2 * e + 1]);
                    o[e] = *reinterpret_cast<const uint32_t*>(&p);
                }
                __nv_bfloat16* to = dweight + (int64_t)(v0 + k0 + j) * a.dweight_stride + col;
                if (c.aligned_out) {
                    if (on) __stcs(reinterpret_cast<uint4*>(to), make_uint4(o[0], o[1], o[2], o[3]));
                } else {
                    store_any(to, o, left, lane);
                }
            }
        }
    }
    if (!on) return;
#pragma unroll
    for (int i = 0; i < TN; ++i) {
        if (i >= a.rows) break;
        float4* plane = reinterpret_cast<float4*>(c.planes + ((int64_t)blockIdx.x * a.rows + i) * c.pitch + col);
        plane[0] = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
        plane[1] = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
    }
}

constexpr int kHiddenThreads = 1024, kHiddenParts = kHiddenThreads / 32;   // that share a column's strips

__global__ void __launch_bounds__(kHiddenThreads)
    few_hidden_kernel(const float* planes, int32_t strips, int32_t rows, int32_t dim, int32_t pitch, __nv_bfloat16* out, int64_t ld) {
    __shared__ float s_sum[kHiddenParts][32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int32_t i = blockIdx.y, col = blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (col < dim) {
        const int32_t lo = (int32_t)((int64_t)strips * part / kHiddenParts), hi = (int32_t)((int64_t)strips * (part + 1) / kHiddenParts);
#pragma unroll 8
        for (int32_t s = lo; s < hi; ++s) sum += planes[((int64_t)s * rows + i) * pitch + col];
    }
    s_sum[part][lane] = sum;
    __syncthreads();
    if (part == 0 && col < dim) {
#pragma unroll
        for (int k = 1; k < kHiddenParts; ++k) sum += s_sum[k][lane];
        out[i * ld + col] = __float2bfloat16_rn(sum);
    }
}

// ---- host ----------------------------------------------------------------------
bool rows_aligned(const void* p, int64_t stride, int32_t dim) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0 && dim % 8 == 0;
}
// Both operands' rows on 16-byte boundaries, in whole vectors.
bool vectors(const LossArgs& a) {
    return rows_aligned(a.hidden, a.hidden_stride, a.dim) && rows_aligned(a.weight, a.weight_stride, a.dim);
}

struct FewSpace {
    int padded;              // rows, to 1, 2 or 4
    int32_t block, blocks, ctas, threads, stretches, strip, strips, pitch;
    size_t target_logit, g, planes, end;
};

FewSpace few_space(const LossArgs& a, const LaunchEnv& env, bool grad) {
    FewSpace s{};
    for (s.padded = 1; s.padded < a.rows; s.padded *= 2) {}
    // blocks of as many tokens as give every warp one; of one token where that is fewer than are read together
    const int most = 32 / s.padded, warps = env.num_sms * 2 * kFewWarps;
    s.block = most;
    while (s.block > 1 && a.n_tokens / s.block < warps) s.block /= 2;
    if (s.block < 4) s.block = 1;
    s.blocks = (a.n_tokens + s.block - 1) / s.block;
    s.ctas = std::min((s.blocks + kFewWarps - 1) / kFewWarps, env.num_sms * 2);
    size_t at = 0;
    const auto take = [&](size_t n) {
        const size_t p = at;
        at += (n + 255) & ~(size_t)255;
        return p;
    };
    if (!grad) {
        take((size_t)a.rows * s.ctas * sizeof(float2));   // part, at 0
        s.target_logit = take((size_t)a.rows * 4);
    } else {
        s.threads = std::min(kSumsThreads, (a.dim + 32 * kN - 1) / (32 * kN) * 32);
        s.stretches = (a.dim + s.threads * kN - 1) / (s.threads * kN);
        const int want = std::max(1, env.num_sms * 4 * (kSumsThreads / s.threads) / s.stretches);
        s.pitch = (a.dim + kN - 1) / kN * kN;
        s.strip = std::max(16, (a.n_tokens + want - 1) / want);
        s.strips = (a.n_tokens + s.strip - 1) / s.strip;
        s.g = take((size_t)a.rows * a.n_tokens * 4);
        s.planes = take((size_t)s.strips * a.rows * s.pitch * 4);
    }
    s.end = at;
    return s;
}

template <int TN, int ROWS>
cudaError_t launch_logits_v(const FewCall& c, int ctas, bool vec, cudaStream_t st) {
    const dim3 grid((unsigned)ctas), block(kFewThreads);
    return vec ? launch_pdl(few_logits_kernel<TN, ROWS, true>, grid, block, 0, st, c)
               : launch_pdl(few_logits_kernel<TN, ROWS, false>, grid, block, 0, st, c);
}
template <int TN>
cudaError_t launch_few_t(const FewCall& c, int ctas, bool vec, cudaStream_t st) {
    if (c.block == 1) return launch_logits_v<TN, 1>(c, ctas, vec, st);
    // off 16-byte boundaries eight rows' two blocks each do not fit the registers
    if (vec && c.block >= 8 && c.a.dim <= 32 * kN)
        return launch_pdl(few_logits_kernel<TN, 8, true>, dim3((unsigned)ctas), dim3(kFewThreads), 0, st, c);
    return launch_logits_v<TN, 4>(c, ctas, vec, st);
}
cudaError_t launch_few(const FewCall& c, const FewSpace& s, cudaStream_t st) {
    const bool vec = vectors(c.a);
    switch (s.padded) {
        case 1: return launch_few_t<1>(c, s.ctas, vec, st);
        case 2: return launch_few_t<2>(c, s.ctas, vec, st);
        default: return launch_few_t<4>(c, s.ctas, vec, st);
    }
}

template <int TN>
cudaError_t launch_sums_t(const FewSums& c, dim3 grid, int threads, bool vec, cudaStream_t st) {
    return vec ? launch_pdl(few_sums_kernel<TN, true>, grid, dim3((unsigned)threads), 0, st, c)
               : launch_pdl(few_sums_kernel<TN, false>, grid, dim3((unsigned)threads), 0, st, c);
}

FewCall few_call(const LossArgs& a, const FewSpace& s) {
    FewCall c{};
    c.a = a;
    c.mask_words = (a.n_tokens + 31) / 32;
    c.block = s.block;
    c.blocks = s.blocks;
    return c;
}

}  // namespace

// One or two rows: as fast as the tensor cores over dense masks (GB300, us few / tensor cores, loss and gradient together: 2
// rows, V = 2000, 256 wide 18.5 / 21.2, V = 32000, 1024 wide 53 / 61, V = 128256, 2048 wide 376 / 352, 4096 wide 726 / 657),
// and weight rows that no mask allows are not read (V = 128256, 2048 wide, sparse masks 123 / 353).  Three and four rows
// without a mask only where the launches are what counts (4 rows, V = 2000, 512 wide 20 / 23, V = 5000, 2048 wide 39 / 42, V =
// 20000, 1024 wide 58 / 44).  With one, sparse masks decide, unless the weight is so large that a dense one would cost twice
// (V = 20000, 1024 wide 38 / 45, 3 rows, V = 14000, 2048 wide 44 / 62; dense: V = 32000, 1024 wide 84 / 61, V = 20000, 4096
// wide 225 / 133); off 16-byte boundaries the tensor cores' operands are laid out first, which takes longer than the products
// of a large weight (4 rows, V = 39587, 1001 wide 86 / 143, V = 128256, 2049 wide 690 / 904; V = 20001, 333 wide 56 / 46).
bool few_rows(const LossArgs& a) {
    if (a.rows <= 2 || a.rows > 4) return a.rows <= 2;
    const int64_t values = (int64_t)a.n_tokens * a.dim;
    if (!a.mask) return vectors(a) && values <= (10 << 20);
    return vectors(a) ? values <= (28 << 20) : values > (1 << 24);
}

size_t few_workspace(const LossArgs& a, const LaunchEnv& env, bool grad) { return few_space(a, env, grad).end; }

cudaError_t launch_few_loss(const LossArgs& a, const LaunchEnv& env, void* space, cudaStream_t st) {
    const FewSpace s = few_space(a, env, false);
    FewCall c = few_call(a, s);
    c.part = (float2*)space;
    c.target_logit = (float*)((char*)space + s.target_logit);
    if (cudaError_t e = launch_few(c, s, st); e != cudaSuccess) return e;
    return launch_loss_merge(a, c.part, s.ctas, c.target_logit, st);
}

cudaError_t launch_few_loss_grad(const LossArgs& a, const LaunchEnv& env, void* space, cudaStream_t st) {
    const FewSpace s = few_space(a, env, true);
    FewCall c = few_call(a, s);
    c.grad = true;
    c.g = (float*)((char*)space + s.g);
    if (cudaError_t e = launch_few(c, s, st); e != cudaSuccess) return e;
    FewSums f{};
    f.a = a;
    f.g = c.g;
    f.strip = s.strip;
    f.planes = (float*)((char*)space + s.planes);
    f.pitch = s.pitch;
    f.aligned_out = rows_aligned(a.dweight, a.dweight_stride, a.dim);
    const bool vec = vectors(a);
    const dim3 grid((unsigned)s.strips, (unsigned)s.stretches);
    cudaError_t e;
    switch (s.padded) {
        case 1: e = launch_sums_t<1>(f, grid, s.threads, vec, st); break;
        case 2: e = launch_sums_t<2>(f, grid, s.threads, vec, st); break;
        default: e = launch_sums_t<4>(f, grid, s.threads, vec, st);
    }
    if (e != cudaSuccess) return e;
    return launch_pdl(few_hidden_kernel, dim3((unsigned)((a.dim + 31) / 32), (unsigned)a.rows), dim3(kHiddenThreads), 0, st,
                      (const float*)f.planes, s.strips, a.rows, a.dim, s.pitch, (__nv_bfloat16*)a.dhidden, a.dhidden_stride);
}

}  // namespace domino
