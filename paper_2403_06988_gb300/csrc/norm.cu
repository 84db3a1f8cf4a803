// norm.cu -- the root-mean-square norm of a stream with the residual's addition, its
// output in the stream's type or in e4m3 codes with a scale for each 128 values, and
// its gradient (sm_103a).
//
//   h    = x + residual, rounded to the stream's type
//   rstd = (mean(h^2) + eps)^(-1/2)
//   y    = h rstd w
//   with g = w dy, c = rstd^2 mean(g h):
//   dx   = rstd (g - c h) + dsum              (of x and of the residual alike)
//   dw   = sum over the rows of dy h rstd
//
// All of it is bound by HBM: a row is read once, kept in registers between its sum of
// squares and its use, and written once.  Sums are fp32; y, the codes, dx and dw are
// rounded once each.  Products and sums are fused where the code says so and nowhere
// else.  The norm's rows give the same bits at any alignment, and so do the gradient's of
// fp32 and of more than 8192 columns; other bf16 rows of the gradient are divided otherwise
// on 16-byte boundaries than off them, which orders its sums otherwise.
#include <algorithm>
#include <atomic>

#include "norm.h"
#include "values8.cuh"

namespace domino {
namespace {

constexpr int kRowThreads8 = 512;         // of a row, at most
constexpr int kFewThreads = 256;          // of a row that they can hold
constexpr int kCtaThreads = 128;          // of a CTA, at least: short rows share one
constexpr int kMaxVectors = 4;            // of a thread, in registers
constexpr int32_t kLongRow = kRowThreads8 * kMaxVectors * kN;   // longer rows are read twice
constexpr int64_t kFarOut = (int64_t)64 << 20;                  // outputs of half of the L2 or more are written past it

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}

// The sum over a row's threads (blockDim.x, a multiple of 32), the same in each; every thread of the CTA calls it.
// `part` is used again only after another barrier.
__device__ __forceinline__ float row_sum(float v, float (*part)[kRowThreads8 / 32]) {
    v = warp_sum(v);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.y][threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < warps; ++w) s += part[threadIdx.y][w];
    return s;
}

template <bool BF16>
__device__ __forceinline__ char* at_row(const void* p, int64_t row, int64_t stride) {
    return (char*)p + row * stride * (BF16 ? 2 : 4);
}

// Eight values of h, x or the rounded sum, as their bits: bf16 in four words.
template <bool BF16>
struct Held {
    uint32_t w[BF16 ? 4 : 8];
    __device__ __forceinline__ void set(const float (&h)[kN]) {
        if constexpr (BF16) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack2(h[2 * e], h[2 * e + 1]);
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) w[e] = __float_as_uint(h[e]);
        }
    }
    __device__ __forceinline__ void get(float (&h)[kN]) const {
        if constexpr (BF16) {
#pragma unroll
            for (int e = 0; e < 4; ++e) h[2 * e] = bf16_lo(w[e]), h[2 * e + 1] = bf16_hi(w[e]);
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) h[e] = __uint_as_float(w[e]);
        }
    }
    // From now on get() unpacks again.
    __device__ __forceinline__ void keep() {
        if constexpr (BF16) asm volatile("" : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]));
    }
};
template <bool BF16, bool ALIGNED>
__device__ __forceinline__ Held<BF16> held(const Vec8<BF16, ALIGNED>& x, const Vec8<BF16, ALIGNED>& r, bool residual) {
    Held<BF16> out;
    float h[kN];
    x.get(h);
    if (residual) {
        float f[kN];
        r.get(f);
        add8(h, f);
    }
    out.set(h);   // without a residual the bits that were read
    return out;
}

// Eight values of y out: h rstd w, as values or as codes.
template <bool BF16, bool ALIGNED, bool CODES>
__device__ __forceinline__ void put_norm(const NormArgs& a, int32_t row, int32_t c, const float (&h)[kN],
                                         const VecOf<BF16, ALIGNED>& weight, float rstd, bool far, int lane) {
    float y[kN], w[kN];
    weight.get(w);
#pragma unroll
    for (int e = 0; e < kN; ++e) y[e] = h[e];
    mul8(y, rstd);
    mul8(y, w);
    if constexpr (CODES) {
        const float top = fmaxf(block_largest(largest(y)), kLeast8);
        if ((lane & (kBlockLanes - 1)) == 0 && c < a.dim)
            a.scales[(int64_t)row * ((a.dim + kBlock8 - 1) / kBlock8) + c / kBlock8] = scale_of(top);
        store_codes(a.codes + (int64_t)row * a.codes_stride, c, a.dim, y, kMost8 / top, far);
    } else {
        store8<BF16, ALIGNED>(at_row<BF16>(a.y, row, a.y_stride), c, a.dim, y, far, lane);
    }
}

__device__ __forceinline__ float root_of(float sum, const NormArgs& a) {
    return __frsqrt_rn(__fadd_rn(__fdiv_rn(sum, (float)a.dim), a.eps));
}

// blockDim.y rows a CTA, of blockDim.x threads with VECTORS times eight values each.
// Registers of bf16 rows on 16-byte boundaries are held down so that an SM has 1024 to 2048 threads (16384 rows, us in codes,
// held down / not: 8192 wide 137, 150; 4096 73, 77; 2048 44, 51; fp32 and rows off the boundaries lose by it).
template <bool BF16, bool ALIGNED, int VECTORS>
constexpr int kNormThreads = BF16 && ALIGNED && VECTORS <= 2 ? kFewThreads : kRowThreads8;
template <bool BF16, bool ALIGNED, int VECTORS>
constexpr int kNormCtas = !(BF16 && ALIGNED) ? 0 : VECTORS == 1 ? 8 : VECTORS == 2 ? 6 : 2;   // 0: as many as there are
template <bool BF16, bool ALIGNED, bool CODES, int VECTORS>
__global__ void __launch_bounds__(kNormThreads<BF16, ALIGNED, VECTORS>, kNormCtas<BF16, ALIGNED, VECTORS>)
    norm_kernel(const __grid_constant__ NormArgs a, const bool far) {
    __shared__ float s_part[kCtaThreads / 32][kRowThreads8 / 32];
    const int lane = threadIdx.x & 31;
    const int32_t row = blockIdx.x * blockDim.y + threadIdx.y;
    const bool on = row < a.rows;
    pdl_wait();
    pdl_trigger();
    Vec8<BF16, ALIGNED> vx[VECTORS], vr[VECTORS];
    VecOf<BF16, ALIGNED> w[VECTORS];
    Held<BF16> v[VECTORS];
    const int32_t dim = on ? a.dim : 0;
    const char* x = at_row<BF16>(a.x, row, a.x_stride);
    const char* r = a.residual ? at_row<BF16>(a.residual, row, a.residual_stride) : nullptr;
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
        const int32_t c = (threadIdx.x + j * blockDim.x) * kN;
        vx[j].load(x, c, dim);
        if (r) vr[j].load(r, c, dim);
    }
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) w[j].load(a.weight, (threadIdx.x + j * blockDim.x) * kN, a.dim);
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
        float h[kN];
        v[j] = held(vx[j], vr[j], r != nullptr);
        v[j].get(h);
        v[j].keep();
        square8(s, h);
    }
    const float rstd = root_of(row_sum(s.x + s.y, s_part), a);
    if (!on) return;   // whole warps
    if (!CODES && a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
        const int32_t c = (threadIdx.x + j * blockDim.x) * kN;
        float h[kN];
        v[j].get(h);
        if (a.sum) store8<BF16, ALIGNED>(at_row<BF16>(a.sum, row, a.sum_stride), c, a.dim, h, far, lane);
        put_norm<BF16, ALIGNED, CODES>(a, row, c, h, w[j], rstd, far, lane);
    }
}

// Rows of more than kLongRow values: a CTA each, the sum read again.
template <bool BF16, bool ALIGNED, bool CODES>
__global__ void __launch_bounds__(kRowThreads8) norm_long_kernel(const __grid_constant__ NormArgs a, const bool far) {
    __shared__ float s_part[1][kRowThreads8 / 32];
    const int lane = threadIdx.x & 31;
    const int32_t row = blockIdx.x, steps = (a.dim + kRowThreads8 * kN - 1) / (kRowThreads8 * kN);
    pdl_wait();
    pdl_trigger();
    const char* x = at_row<BF16>(a.x, row, a.x_stride);
    const char* r = a.residual ? at_row<BF16>(a.residual, row, a.residual_stride) : nullptr;
    char* sum = a.sum ? at_row<BF16>(a.sum, row, a.sum_stride) : nullptr;
    float2 s = make_float2(0.0f, 0.0f);
    for (int32_t j = 0; j < steps; ++j) {
        const int32_t c = (threadIdx.x + j * kRowThreads8) * kN;
        Vec8<BF16, ALIGNED> vx, vr;
        float h[kN];
        vx.load(x, c, a.dim);
        if (r) vr.load(r, c, a.dim);
        held(vx, vr, r != nullptr).get(h);
        if (sum) store8<BF16, ALIGNED>(sum, c, a.dim, h, false, lane);
        square8(s, h);
    }
    const float rstd = root_of(row_sum(s.x + s.y, s_part), a);   // its barrier: the sum is written
    if (!CODES && a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    for (int32_t j = 0; j < steps; ++j) {
        const int32_t c = (threadIdx.x + j * kRowThreads8) * kN;
        Vec8<BF16, ALIGNED> v;
        VecOf<BF16, ALIGNED> w;
        float h[kN];
        v.load(sum ? sum : x, c, a.dim);
        w.load(a.weight, c, a.dim);
        v.get(h);
        put_norm<BF16, ALIGNED, CODES>(a, row, c, h, w, rstd, far, lane);
    }
}

// ---- gradient ------------------------------------------------------------------
// Eight columns of a row: their part of dw, and of the row's sums of g h, of the even columns and of the odd ones.  PAIRS:
// two values an instruction, the same roundings (bf16 rows; fp32 ones lie in single registers: 16384 x 4096 191 us, 226 in
// pairs).
template <bool PAIRS>
__device__ __forceinline__ void first_pass(const float (&h)[kN], const float (&dy)[kN], const float (&w)[kN], float rstd,
                                           float (&dw)[kN], float2& s) {
    if constexpr (PAIRS) {
        float n[kN], g[kN];
#pragma unroll
        for (int e = 0; e < kN; ++e) n[e] = h[e], g[e] = dy[e];
        mul8(n, rstd);
        fma8(dw, dy, n, dw);
        mul8(g, w);
        dot8(s, g, h);
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            dw[e] = __fmaf_rn(dy[e], __fmul_rn(h[e], rstd), dw[e]);
            float& sum = e & 1 ? s.y : s.x;
            sum = __fmaf_rn(__fmul_rn(dy[e], w[e]), h[e], sum);
        }
    }
}
// Their part of dx, in dy's place: rstd (dy w - h c).
template <bool PAIRS>
__device__ __forceinline__ void second_pass(const float (&h)[kN], float (&dy)[kN], const float (&w)[kN], float rstd, float c) {
    if constexpr (PAIRS) {
        mul8(dy, w);
        fma8(dy, h, -c, dy);
        mul8(dy, rstd);
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e) dy[e] = __fmul_rn(rstd, __fmaf_rn(h[e], -c, __fmul_rn(dy[e], w[e])));
    }
}

constexpr int kGradThreads = 256;         // of a row, at most
constexpr int kGradVectors = 4;
constexpr int32_t kGradLongRow = kGradThreads * kGradVectors * kN;

// A CTA's blockDim.y strips of rows.
struct Strip {
    int32_t row0, row1, most;   // most: rows of the longest strip, all take part in the barriers
    __device__ __forceinline__ Strip(int32_t rows, int32_t strips) {
        const int32_t i = blockIdx.x * blockDim.y + threadIdx.y;
        row0 = i < strips ? (int32_t)((int64_t)rows * i / strips) : 0;
        row1 = i < strips ? (int32_t)((int64_t)rows * (i + 1) / strips) : 0;
        most = (rows + strips - 1) / strips;
    }
};

// A CTA's rows (blockDim.y strips of them, threads as in norm_kernel) one after the other; the strip's part of dw stays
// in registers and goes to parts[strip][pitch].
// (Registers of fp32 rows off 16-byte boundaries are held down: 8000 x 333 19.4 us, else 21.3.)
template <bool BF16, bool ALIGNED, int VECTORS>
__global__ void __launch_bounds__(kGradThreads, !BF16 && !ALIGNED && VECTORS == 1 ? 3 : 0) norm_grad_kernel(const __grid_constant__ NormGradArgs a, float* parts,
                                                                 const int32_t strips, const int32_t pitch, const bool far) {
    __shared__ float s_part[2][kCtaThreads / 32][kRowThreads8 / 32];
    const int lane = threadIdx.x & 31;
    const Strip t(a.rows, strips);
    pdl_wait();
    pdl_trigger();
    VecOf<BF16, ALIGNED> w[VECTORS];
    float dw[VECTORS][kN];
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
        w[j].load(a.weight, (threadIdx.x + j * blockDim.x) * kN, a.dim);
#pragma unroll
        for (int e = 0; e < kN; ++e) dw[j][e] = 0.0f;
    }
    for (int32_t i = 0; i < t.most; ++i) {
        const int32_t row = t.row0 + i;
        const bool on = row < t.row1;
        const int32_t dim = on ? a.dim : 0;
        const char* ph = at_row<BF16>(a.h, row, a.h_stride);
        const char* pd = at_row<BF16>(a.dy, row, a.dy_stride);
        Vec8<BF16, ALIGNED> vh[VECTORS], vd[VECTORS], vs[VECTORS];
        float2 s = make_float2(0.0f, 0.0f);
        const float rstd = on ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
            const int32_t c = (threadIdx.x + j * blockDim.x) * kN;
            vh[j].load(ph, c, dim);
            vd[j].load(pd, c, dim);
            if (a.dsum) vs[j].load(at_row<BF16>(a.dsum, row, a.dsum_stride), c, dim);
        }
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
            float h[kN], g[kN], u[kN];
            vh[j].get(h);
            vd[j].get(g);
            w[j].get(u);
            vh[j].keep();
            vd[j].keep();
            w[j].keep();
            if (a.dsum) vs[j].keep();
            first_pass<BF16>(h, g, u, rstd, dw[j], s);
        }
        const float c1 = __fmul_rn(__fmul_rn(__fdiv_rn(row_sum(s.x + s.y, s_part[i & 1]), (float)a.dim), rstd), rstd);
        if (!on) continue;
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
            float h[kN], g[kN], u[kN];
            vh[j].get(h);
            vd[j].get(g);
            w[j].get(u);
            second_pass<BF16>(h, g, u, rstd, c1);
            if (a.dsum) {
                vs[j].get(h);
                add8(g, h);
            }
            store8<BF16, ALIGNED>(at_row<BF16>(a.dx, row, a.dx_stride), (threadIdx.x + j * blockDim.x) * kN, a.dim, g, far, lane);
        }
    }
    if (t.row0 >= t.row1) return;
    const int32_t strip = blockIdx.x * blockDim.y + threadIdx.y;
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
        const int32_t c = (threadIdx.x + j * blockDim.x) * kN;
        if (c >= pitch) continue;
        float4* to = reinterpret_cast<float4*>(parts + (int64_t)strip * pitch + c);
        to[0] = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
        to[1] = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
    }
}

// ---- bf16: the next rows on their way ---------------------------------------------
// A thread's own vectors of the strip's next rows come to shared memory by asynchronous copies, and it alone reads them:
// no barrier guards them, and what is on its way takes no registers (16384 x 4096: 99 us, without 123; 1024 wide 40 and
// 46; 300 x 4096 7.2 and 8.0; all before the steps below).  fp32 rows take twice the memory, which then holds one CTA an SM: 300 us, without
// 191.
// Rows in shared memory: one in use, the others on their way.  Of the widest two, so that an SM holds two CTAs (16384 x
// 8192: 178 us, with three 249).
template <int VECTORS>
constexpr int kAhead = VECTORS == 4 ? 2 : 3;
template <int VECTORS>
constexpr int kStreamCtas = VECTORS == 1 ? 4 : VECTORS == 2 ? 3 : 2;   // of kGradThreads, of an SM, by their registers
constexpr int kStreamBytes = 220 * 1024;  // of an SM

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
// All but the last PENDING groups of this thread have come.
template <int PENDING>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;\n" ::"n"(PENDING) : "memory");
}

// A thread's vectors of three rows (h, dy, dsum), kAhead times; neighbouring threads' lie side by side.
template <int VECTORS>
struct Ahead {
    uint32_t base, threads;
    __device__ __forceinline__ Ahead(const void* smem) {
        threads = blockDim.x * blockDim.y;
        base = (uint32_t)__cvta_generic_to_shared(smem) + (threadIdx.y * blockDim.x + threadIdx.x) * 16;
    }
    __device__ __forceinline__ uint32_t at(int slot, int array, int j) const {
        return base + (uint32_t)((slot * 3 + array) * VECTORS + j) * threads * 16;
    }
    __device__ __forceinline__ void copy(int slot, int array, const char* row, int32_t dim) const {
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
            const int32_t c = (threadIdx.x + j * blockDim.x) * kN;
            if (c < dim) copy16(at(slot, array, j), row + (int64_t)c * 2);
        }
    }
    __device__ __forceinline__ Vec8<true, true> read(int slot, int array, int j, int32_t dim) const {
        Vec8<true, true> v;
        v.left = dim - (int32_t)(threadIdx.x + j * blockDim.x) * kN;
        v.u = make_uint4(0u, 0u, 0u, 0u);
        if (v.left > 0)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n"
                         : "=r"(v.u.x), "=r"(v.u.y), "=r"(v.u.z), "=r"(v.u.w)
                         : "r"(at(slot, array, j))
                         : "memory");
        return v;
    }
};

template <int VECTORS>
__global__ void __launch_bounds__(kGradThreads, kStreamCtas<VECTORS>) norm_grad_stream_kernel(const __grid_constant__ NormGradArgs a, float* parts,
                                                                        const int32_t strips, const int32_t pitch, const bool far) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float s_part[2][kCtaThreads / 32][kRowThreads8 / 32];
    const int lane = threadIdx.x & 31;
    const Strip t(a.rows, strips);
    const Ahead<VECTORS> ahead(smem);
    pdl_wait();
    pdl_trigger();
    const auto fetch = [&](int32_t i) {
        const int32_t row = t.row0 + i;
        if (row < t.row1) {
            ahead.copy(i % kAhead<VECTORS>, 0, at_row<true>(a.h, row, a.h_stride), a.dim);
            ahead.copy(i % kAhead<VECTORS>, 1, at_row<true>(a.dy, row, a.dy_stride), a.dim);
            if (a.dsum) ahead.copy(i % kAhead<VECTORS>, 2, at_row<true>(a.dsum, row, a.dsum_stride), a.dim);
        }
        copies_done();
    };
#pragma unroll
    for (int i = 0; i < kAhead<VECTORS> - 1; ++i) fetch(i);
    VecOf<true, true> w[VECTORS];
    float dw[VECTORS][kN];
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
        w[j].load(a.weight, (threadIdx.x + j * blockDim.x) * kN, a.dim);
#pragma unroll
        for (int e = 0; e < kN; ++e) dw[j][e] = 0.0f;
    }
    float next = t.row0 < t.row1 ? a.rstd[t.row0] : 0.0f;
    for (int32_t i = 0; i < t.most; ++i) {
        const int32_t row = t.row0 + i;
        const bool on = row < t.row1;
        const float rstd = next;
        if (row + 1 < t.row1) next = a.rstd[row + 1];
        fetch(i + kAhead<VECTORS> - 1);   // where row i - 1 was
        copies_wait<kAhead<VECTORS> - 1>();
        const int slot = i % kAhead<VECTORS>;
        float2 s = make_float2(0.0f, 0.0f);
        if (on) {
#pragma unroll
            for (int j = 0; j < VECTORS; ++j) {
                float h[kN], g[kN], u[kN];
                ahead.read(slot, 0, j, a.dim).get(h);
                ahead.read(slot, 1, j, a.dim).get(g);
                w[j].keep();
                w[j].get(u);
                first_pass<true>(h, g, u, rstd, dw[j], s);
            }
        }
        const float c1 = __fmul_rn(__fmul_rn(__fdiv_rn(row_sum(s.x + s.y, s_part[i & 1]), (float)a.dim), rstd), rstd);
        if (!on) continue;
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
            float h[kN], g[kN], u[kN];
            ahead.read(slot, 0, j, a.dim).get(h);
            ahead.read(slot, 1, j, a.dim).get(g);
            w[j].keep();
            w[j].get(u);
            second_pass<true>(h, g, u, rstd, c1);
            if (a.dsum) {
                ahead.read(slot, 2, j, a.dim).get(h);
                add8(g, h);
            }
            store8<true, true>(at_row<true>(a.dx, row, a.dx_stride), (threadIdx.x + j * blockDim.x) * kN, a.dim, g, far, lane);
        }
    }
    if (t.row0 >= t.row1) return;
    const int32_t strip = blockIdx.x * blockDim.y + threadIdx.y;
#pragma unroll
    for (int j = 0; j < VECTORS; ++j) {
        const int32_t c = (threadIdx.x + j * blockDim.x) * kN;
        if (c >= pitch) continue;
        float4* to = reinterpret_cast<float4*>(parts + (int64_t)strip * pitch + c);
        to[0] = make_float4(dw[j][0], dw[j][1], dw[j][2], dw[j][3]);
        to[1] = make_float4(dw[j][4], dw[j][5], dw[j][6], dw[j][7]);
    }
}

// Rows of more than kGradLongRow values: the rows' sums first, then columns by strips of rows, a thread eight columns.
template <bool BF16, bool ALIGNED>
__global__ void __launch_bounds__(kRowThreads8) norm_grad_sums_kernel(const __grid_constant__ NormGradArgs a, float* sums) {
    __shared__ float s_part[1][kRowThreads8 / 32];
    pdl_wait();
    pdl_trigger();
    const int32_t row = blockIdx.x;
    float2 s = make_float2(0.0f, 0.0f);
    for (int32_t c = threadIdx.x * kN; c < a.dim; c += kRowThreads8 * kN) {
        Vec8<BF16, ALIGNED> vh, vd;
        VecOf<BF16, ALIGNED> vw;
        float h[kN], g[kN], w[kN];
        vh.load(at_row<BF16>(a.h, row, a.h_stride), c, a.dim);
        vd.load(at_row<BF16>(a.dy, row, a.dy_stride), c, a.dim);
        vw.load(a.weight, c, a.dim);
        vh.get(h);
        vd.get(g);
        vw.get(w);
        mul8(g, w);
        dot8(s, g, h);
    }
    const float sum = row_sum(s.x + s.y, s_part), rstd = a.rstd[row];
    if (threadIdx.x == 0) sums[row] = __fmul_rn(__fmul_rn(__fdiv_rn(sum, (float)a.dim), rstd), rstd);
}
template <bool BF16, bool ALIGNED>
__global__ void __launch_bounds__(kGradThreads) norm_grad_long_kernel(const __grid_constant__ NormGradArgs a, const float* sums,
                                                                      float* parts, const int32_t strips, const int32_t pitch,
                                                                      const bool far) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int32_t c = (blockIdx.x * kGradThreads + threadIdx.x) * kN, strip = blockIdx.y;
    const int32_t row0 = (int32_t)((int64_t)a.rows * strip / strips), row1 = (int32_t)((int64_t)a.rows * (strip + 1) / strips);
    float w[kN], dw[kN];
    VecOf<BF16, ALIGNED> vw;
    vw.load(a.weight, c, a.dim);
    vw.get(w);
#pragma unroll
    for (int e = 0; e < kN; ++e) dw[e] = 0.0f;
    for (int32_t row = row0; row < row1; ++row) {
        Vec8<BF16, ALIGNED> vh, vd, vs;
        float h[kN], g[kN], ds[kN];
        const float rstd = a.rstd[row], c1 = sums[row];
        vh.load(at_row<BF16>(a.h, row, a.h_stride), c, a.dim);
        vd.load(at_row<BF16>(a.dy, row, a.dy_stride), c, a.dim);
        if (a.dsum) {
            vs.load(at_row<BF16>(a.dsum, row, a.dsum_stride), c, a.dim);
            vs.get(ds);
        }
        vh.get(h);
        vd.get(g);
        float2 none = make_float2(0.0f, 0.0f);
        first_pass<BF16>(h, g, w, rstd, dw, none);
        second_pass<BF16>(h, g, w, rstd, c1);
        if (a.dsum) add8(g, ds);
        store8<BF16, ALIGNED>(at_row<BF16>(a.dx, row, a.dx_stride), c, a.dim, g, far, lane);
    }
    if (c >= pitch) return;
    float4* to = reinterpret_cast<float4*>(parts + (int64_t)strip * pitch + c);
    to[0] = make_float4(dw[0], dw[1], dw[2], dw[3]);
    to[1] = make_float4(dw[4], dw[5], dw[6], dw[7]);
}

// dw: the strips' parts, added in an order that their number fixes.  LANES times four columns a CTA, so that few columns too
// give many SMs some of the sum.
constexpr int kJoinThreads = 512;
template <bool BF16, int LANES>
__global__ void __launch_bounds__(kJoinThreads) norm_join_kernel(const float* parts, const int32_t strips, const int32_t pitch,
                                                                 const int32_t dim, void* dweight) {
    constexpr int kGroups = kJoinThreads / LANES;
    __shared__ float4 s_sum[kGroups][LANES];
    pdl_wait();
    pdl_trigger();
    const int at = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int32_t c = (blockIdx.x * LANES + at) * 4;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < pitch) {
#pragma unroll 8
        for (int32_t k = group; k < strips; k += kGroups) {
            const float4 x = *reinterpret_cast<const float4*>(parts + (int64_t)k * pitch + c);
            v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
        }
    }
    s_sum[group][at] = v;
#pragma unroll
    for (int n = kGroups / 2; n > 0; n >>= 1) {
        __syncthreads();
        if (group < n) {
            const float4 x = s_sum[group + n][at];
            v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
            s_sum[group][at] = v;
        }
    }
    if (group) return;
    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (c + e >= dim) break;
        if constexpr (BF16) static_cast<__nv_bfloat16*>(dweight)[c + e] = __float2bfloat16_rn(f[e]);
        else static_cast<float*>(dweight)[c + e] = f[e];
    }
}

// ---- host ----------------------------------------------------------------------
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

bool on16(const void* p, int64_t stride, int dtype) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * (dtype == DOMINO_DTYPE_BF16 ? 2 : 4) % 16 == 0;
}

// Threads of a row and the vectors that each holds.
struct Cut {
    int threads, vectors, rows;   // rows of a CTA
};
Cut cut_row(int32_t dim, int most_threads) {
    const int vectors = ceil_div(dim, kN);
    Cut c{0, 1, 1};
    while (vectors > most_threads * c.vectors && c.vectors < kMaxVectors) c.vectors *= 2;
    c.threads = std::min(most_threads, ceil_div(ceil_div(vectors, c.vectors), 32) * 32);
    c.rows = std::max(1, kCtaThreads / c.threads);
    return c;
}

template <bool BF16, bool ALIGNED, bool CODES>
cudaError_t launch_norm_t(const NormArgs& a, cudaStream_t st) {
    const bool far = (int64_t)a.rows * a.dim * (CODES ? 1 : BF16 ? 2 : 4) >= kFarOut;
    if (a.dim > kLongRow)
        return launch_pdl(norm_long_kernel<BF16, ALIGNED, CODES>, dim3((unsigned)a.rows), dim3(kRowThreads8), 0, st, a, far);
    // 256 threads a row where they can hold it: a CTA's row waits at one barrier, and smaller CTAs wait less (16384 x 4096
    // bf16: norm 78 us, in codes 77; with 512 threads 102 and 102, before registers were held down)
    const Cut c = cut_row(a.dim, a.dim <= kFewThreads * kMaxVectors * kN ? kFewThreads : kRowThreads8);
    const dim3 grid((unsigned)ceil_div(a.rows, c.rows)), block((unsigned)c.threads, (unsigned)c.rows);
    switch (c.vectors) {
        case 1: return launch_pdl(norm_kernel<BF16, ALIGNED, CODES, 1>, grid, block, 0, st, a, far);
        case 2: return launch_pdl(norm_kernel<BF16, ALIGNED, CODES, 2>, grid, block, 0, st, a, far);
        default: return launch_pdl(norm_kernel<BF16, ALIGNED, CODES, 4>, grid, block, 0, st, a, far);
    }
}
template <bool BF16, bool ALIGNED>
cudaError_t launch_norm_c(const NormArgs& a, cudaStream_t st) {
    return a.codes ? launch_norm_t<BF16, ALIGNED, true>(a, st) : launch_norm_t<BF16, ALIGNED, false>(a, st);
}

struct GradCut {
    Cut cut;
    int32_t strips, pitch;
    size_t sums;          // bytes of the rows' sums (long rows)
    int stream;           // bytes of a CTA of the kernel that fetches ahead; 0: the other
};
bool grad_aligned(const NormGradArgs& a) {
    return on16(a.h, a.h_stride, a.dtype) && on16(a.dy, a.dy_stride, a.dtype) && on16(a.dx, a.dx_stride, a.dtype) &&
           on16(a.weight, 0, a.dtype) && (!a.dsum || on16(a.dsum, a.dsum_stride, a.dtype));
}
GradCut cut_grad(const NormGradArgs& a, const LaunchEnv& env) {
    GradCut g{cut_row(a.dim, kGradThreads), 0, ceil_div(a.dim, kN) * kN, 0, 0};
    const bool lng = a.dim > kGradLongRow;
    if (lng) g.sums = ((size_t)a.rows * 4 + 255) / 256 * 256;
    if (!lng && a.dtype == DOMINO_DTYPE_BF16 && grad_aligned(a)) {
        // as many vectors a thread as there are, up to four: fewer warps share a row's sum (16384 rows, us, four / one: 4096
        // wide 95, 98 with two; 2048 54, 60; 1024 33, 39)
        const int vectors = ceil_div(a.dim, kN);
        g.cut.vectors = vectors > 64 ? 4 : vectors > 32 ? 2 : 1;
        g.cut.threads = ceil_div(ceil_div(vectors, g.cut.vectors), 32) * 32;
        g.cut.rows = std::max(1, kCtaThreads / g.cut.threads);
        const int ctas = g.cut.vectors == 1 ? kStreamCtas<1> : g.cut.vectors == 2 ? kStreamCtas<2> : kStreamCtas<4>;
        const int threads = g.cut.threads * g.cut.rows;
        g.stream = (g.cut.vectors == 4 ? kAhead<4> : kAhead<1>) * 3 * g.cut.vectors * threads * 16;
        const int per_sm = std::max(1, std::min(kStreamBytes / g.stream, ctas * kGradThreads / threads));
        g.strips = (int32_t)std::min<int64_t>(a.rows, (int64_t)per_sm * env.num_sms * g.cut.rows);
        return g;
    }
    // strips of rows: as many as the SMs hold at once (768 threads each, by their registers), and not so many that their
    // parts of dw take longer than the rows (8000 x 1001 bf16: 34 us with six an SM, 42 with four; 16384 x 4096 fp32 alike)
    const int threads = g.cut.threads * g.cut.rows;
    const int64_t ctas = lng ? (int64_t)env.num_sms * 4 / ceil_div(a.dim, kGradThreads * kN)
                             : (int64_t)env.num_sms * std::max(4, 768 / threads) * g.cut.rows;
    g.strips = (int32_t)std::max<int64_t>(1, std::min<int64_t>(a.rows, ctas));
    return g;
}

template <int VECTORS>
cudaError_t launch_grad_stream(const NormGradArgs& a, const GradCut& g, float* parts, bool far, cudaStream_t st) {
    static std::atomic<bool> ready[64];   // more than 48 KB of shared memory: raised once per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !ready[dev].load()) {
        e = cudaFuncSetAttribute(norm_grad_stream_kernel<VECTORS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamBytes);
        if (e != cudaSuccess) return e;
        if (dev < 64) ready[dev].store(true);
    }
    return launch_pdl(norm_grad_stream_kernel<VECTORS>, dim3((unsigned)ceil_div(g.strips, g.cut.rows)),
                      dim3((unsigned)g.cut.threads, (unsigned)g.cut.rows), (size_t)g.stream, st, a, parts, g.strips, g.pitch, far);
}

template <bool BF16, bool ALIGNED>
cudaError_t launch_grad_t(const NormGradArgs& a, const LaunchEnv& env, void* space, cudaStream_t st) {
    const GradCut g = cut_grad(a, env);
    const bool far = (int64_t)a.rows * a.dim * (BF16 ? 2 : 4) >= kFarOut;
    float* parts = (float*)((char*)space + g.sums);
    cudaError_t e;
    if (a.dim > kGradLongRow) {
        float* sums = (float*)space;
        e = launch_pdl(norm_grad_sums_kernel<BF16, ALIGNED>, dim3((unsigned)a.rows), dim3(kRowThreads8), 0, st, a, sums);
        if (e != cudaSuccess) return e;
        e = launch_pdl(norm_grad_long_kernel<BF16, ALIGNED>, dim3((unsigned)ceil_div(a.dim, kGradThreads * kN), (unsigned)g.strips),
                       dim3(kGradThreads), 0, st, a, (const float*)sums, parts, g.strips, g.pitch, far);
    } else if constexpr (BF16 && ALIGNED) {   // as cut_grad divides them
        switch (g.cut.vectors) {
            case 1: e = launch_grad_stream<1>(a, g, parts, far, st); break;
            case 2: e = launch_grad_stream<2>(a, g, parts, far, st); break;
            default: e = launch_grad_stream<4>(a, g, parts, far, st);
        }
    } else {
        const dim3 grid((unsigned)ceil_div(g.strips, g.cut.rows)), block((unsigned)g.cut.threads, (unsigned)g.cut.rows);
        switch (g.cut.vectors) {
            case 1: e = launch_pdl(norm_grad_kernel<BF16, ALIGNED, 1>, grid, block, 0, st, a, parts, g.strips, g.pitch, far); break;
            case 2: e = launch_pdl(norm_grad_kernel<BF16, ALIGNED, 2>, grid, block, 0, st, a, parts, g.strips, g.pitch, far); break;
            default: e = launch_pdl(norm_grad_kernel<BF16, ALIGNED, 4>, grid, block, 0, st, a, parts, g.strips, g.pitch, far);
        }
    }
    if (e != cudaSuccess) return e;
    const bool few = ceil_div(a.dim, 8) * 2 <= env.num_sms;   // 16384 x 256 bf16 15.0 us, in wide CTAs 19.5
    return launch_pdl(few ? norm_join_kernel<BF16, 2> : norm_join_kernel<BF16, 8>, dim3((unsigned)ceil_div(a.dim, few ? 8 : 32)),
                      dim3(kJoinThreads), 0, st, (const float*)parts, g.strips, g.pitch, a.dim, a.dweight);
}

}  // namespace

cudaError_t launch_norm(const NormArgs& a, const LaunchEnv&, cudaStream_t st) {
    bool aligned = on16(a.x, a.x_stride, a.dtype) && on16(a.weight, 0, a.dtype);
    if (a.residual) aligned = aligned && on16(a.residual, a.residual_stride, a.dtype);
    if (a.sum) aligned = aligned && on16(a.sum, a.sum_stride, a.dtype);
    if (!a.codes) aligned = aligned && on16(a.y, a.y_stride, a.dtype);
    if (a.dtype == DOMINO_DTYPE_BF16) return aligned ? launch_norm_c<true, true>(a, st) : launch_norm_c<true, false>(a, st);
    return aligned ? launch_norm_c<false, true>(a, st) : launch_norm_c<false, false>(a, st);
}

size_t norm_grad_workspace(const NormGradArgs& a, const LaunchEnv& env) {
    const GradCut g = cut_grad(a, env);
    return g.sums + (size_t)g.strips * g.pitch * 4;
}

cudaError_t launch_norm_grad(const NormGradArgs& a, const LaunchEnv& env, void* space, cudaStream_t st) {
    const bool aligned = grad_aligned(a);
    if (a.dtype == DOMINO_DTYPE_BF16) return aligned ? launch_grad_t<true, true>(a, env, space, st) : launch_grad_t<true, false>(a, env, space, st);
    return aligned ? launch_grad_t<false, true>(a, env, space, st) : launch_grad_t<false, false>(a, env, space, st);
}

}  // namespace domino
