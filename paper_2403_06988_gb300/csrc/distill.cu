// distill.cu -- the Kullback-Leibler divergence of a teacher's top logits from
// a student's masked softmax, and its gradient (sm_103a).
//
//   q     = softmax of x[v] / tau over the tokens that the mask allows
//   p     = softmax of t[i] / tau over the row's entries: those whose id is a
//           token that the mask allows and whose logits, the teacher's and the
//           student's, are not -inf; of equal ids the first
//   loss  = tau^2 sum_i p_i (ln p_i - ln q_{id_i})         0 without entries
//   dx[v] = g tau (q_v - sum_{i: id_i = v} p_i)            0 without entries
//
// The student's logits are read once and, for the gradient, written once: HBM
// bounds both.  One CTA per row, or a cluster of up to 8 that share out the
// row's tokens while the rows alone leave SMs idle.  16-byte vectors without an
// allowed token are not read.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "decode.cuh"
#include "loss.h"

namespace cg = cooperative_groups;

namespace domino {
namespace {

constexpr int kDistillThreads = 512;
constexpr int kDistillWarps = kDistillThreads / 32;
constexpr int kDistillMaxSlices = 8;
// Two vectors a thread and four CTAs an SM (us of the loss, and of both; 2048 rows, V = 128256 bf16 / 301 rows, V = 50001, masks): 99,
// 271 / 12.4, 25.8; four vectors and three CTAs 100, 267 / 15.5, 30.3; one vector 112, 295 / 12.4, 28.2; four and the
// next four on their way, which leaves room for fewer warps, 190, 358 / 18.0, 31.0.
constexpr int kDistillCtas = 4, kDistillUnroll = 2;
constexpr int kDistillSlots = 2 * kDistillMaxK;                        // of the table of ids
constexpr int kDistillEntries = kDistillMaxK / kDistillThreads;        // a thread's

struct DistillCall {
    DistillArgs a;
    int32_t W;
    int32_t slices, slice;       // CTAs per row; tokens of each (a multiple of 32)
    int32_t slots;               // of the table of ids: a power of two, twice the entries or more
    float inv_tau, k;            // 1 / tau; log2(e) / tau
};

struct DistillShared {
    int32_t id[kDistillSlots];
    int32_t first[kDistillSlots];
    float red[2 * kDistillWarps];
    float2 part;                 // the slice's (max, sum)
    float lse;
};

template <bool BF16>
struct Vec {
    static constexpr int kN = BF16 ? 8 : 4;
    float v[kN];
    __device__ __forceinline__ void set(const uint4& u) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            } else {
                v[i] = __uint_as_float(w[i]);
            }
        }
    }
    __device__ __forceinline__ uint4 get() const {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&b);
            } else {
                w[i] = __float_as_uint(v[i]);
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <bool BF16>
__device__ __forceinline__ float load_at(const void* row, int64_t t) {
    if constexpr (BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[t]);
    else return reinterpret_cast<const float*>(row)[t];
}
template <bool BF16>
__device__ __forceinline__ void store_at(void* row, int64_t t, float x) {
    if constexpr (BF16) reinterpret_cast<__nv_bfloat16*>(row)[t] = __float2bfloat16_rn(x);
    else reinterpret_cast<float*>(row)[t] = x;
}

// Bits of the tokens [t, t + n) of a row that are allowed (n <= 8, t + n <= V).
__device__ __forceinline__ uint32_t allowed_bits(const uint32_t* mrow, int32_t t, int n) {
    const uint32_t all = (1u << n) - 1u;
    if (!mrow) return all;
    const int32_t w = t >> 5, off = t & 31;
    uint32_t bits = __ldg(mrow + w) >> off;
    if (off + n > 32) bits |= __ldg(mrow + w + 1) << (32 - off);
    return bits & all;
}

// x / tau as a product with the inverse (a rounding more than a division), rounded to fp32 wherever it is used: lse holds the
// largest one's rounding, and a difference from lse that kept the product's other bits (one fma) would be off by up to half a
// unit in lse's last place, above zero too: exp of it passes all bounds where that unit is large (logits that ban a token, 1e9
// and more).
__device__ __forceinline__ float scaled(float x, const DistillCall& c) { return __fmul_rn(x, c.inv_tau); }

__device__ __forceinline__ float2 merge(float2 a, float2 b, float k) {
    const float m = fmaxf(a.x, b.x), ref = sum_ref(m);
    return make_float2(m, a.y * ex2((a.x - ref) * k) + b.y * ex2((b.x - ref) * k));
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}
// of the CTA, for every thread; ends with a barrier
template <bool MAX>
__device__ __forceinline__ float cta_reduce(float x, float* red) {
    x = MAX ? warp_max(x) : warp_sum(x);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    x = red[threadIdx.x & (kDistillWarps - 1)];
    x = MAX ? warp_max(x) : warp_sum(x) * (kDistillWarps / 32.0f);   // each of 16 twice
    __syncthreads();
    return x;
}

// A thread's entries of the row's teacher list: p (0: no entry), the teacher's
// and the student's log-probabilities' numerators.
struct Entries {
    int32_t id[kDistillEntries];
    float p[kDistillEntries], logp[kDistillEntries], x[kDistillEntries];
    bool any;
};

template <bool BF16>
__device__ void read_entries(Entries& e, const DistillCall& c, int32_t row, const void* xrow, const uint32_t* mrow,
                             DistillShared& sh, bool report) {
    const DistillArgs& a = c.a;
    const int slots = c.slots;
    for (int i = threadIdx.x; i < slots; i += kDistillThreads) {
        sh.id[i] = -1;
        sh.first[i] = INT_MAX;
    }
    __syncthreads();
    uint32_t slot[kDistillEntries];
    float t[kDistillEntries];
#pragma unroll
    for (int j = 0; j < kDistillEntries; ++j) {
        const int32_t i = threadIdx.x + j * kDistillThreads;
        e.id[j] = -1;
        if (i >= a.k) continue;
        const int32_t id = __ldg(a.ids + (int64_t)row * a.k + i);
        if (id >= a.n_tokens && report) atomicOr(a.err, DOMINO_DEVERR_BAD_TOKEN);
        if (id < 0 || id >= a.n_tokens || !allowed_bits(mrow, id, 1)) continue;
        const float x = load_at<BF16>(xrow, id);
        t[j] = a.teacher_dtype == DOMINO_DTYPE_BF16 ? load_at<true>(a.teacher, (int64_t)row * a.k + i)
                                                    : load_at<false>(a.teacher, (int64_t)row * a.k + i);
        if (x == -INFINITY || t[j] == -INFINITY) continue;
        e.id[j] = id;
        e.x[j] = x;
        // the first entry of an id: its place in a table of ids
        uint32_t h = ((uint32_t)id * 2654435761u >> 16) & (slots - 1);
        while (true) {
            const int32_t old = atomicCAS(&sh.id[h], -1, id);
            if (old == -1 || old == id) break;
            h = (h + 1) & (slots - 1);
        }
        atomicMin(&sh.first[h], i);
        slot[j] = h;
    }
    __syncthreads();
    float top = -INFINITY;
    bool any = false;
#pragma unroll
    for (int j = 0; j < kDistillEntries; ++j) {
        if (e.id[j] >= 0 && sh.first[slot[j]] != threadIdx.x + j * kDistillThreads) e.id[j] = -1;
        if (e.id[j] >= 0) {
            top = fmaxf(top, t[j]);
            any = true;
        }
    }
    e.any = __syncthreads_or(any);
    top = sum_ref(cta_reduce<true>(top, sh.red));
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kDistillEntries; ++j) {
        e.p[j] = 0.0f;
        if (e.id[j] < 0) continue;
        e.logp[j] = (t[j] - top) * c.inv_tau;
        e.p[j] = ex2((t[j] - top) * c.k);
        sum += e.p[j];
    }
    sum = cta_reduce<false>(sum, sh.red);
    const float inv = 1.0f / sum, ln = logf(sum);
#pragma unroll
    for (int j = 0; j < kDistillEntries; ++j)
        if (e.id[j] >= 0) {
            e.p[j] *= inv;
            e.logp[j] -= ln;
        }
}

__device__ __forceinline__ float2 scale2(float2 a, float b) { return fma2(a, b, 0.0f); }

// The vectors that a thread reads together, and which of their tokens are allowed.
template <bool BF16>
struct Batch {
    uint4 u[kDistillUnroll];
    uint32_t bits[kDistillUnroll];
    // vectors n = i, i + kDistillThreads, ... of the slice's, the first at token `head`
    template <bool KEEP>
    __device__ __forceinline__ void load(const char* xrow, const uint32_t* mrow, int32_t head, int32_t vectors, int32_t i, bool any) {
        constexpr int kN = Vec<BF16>::kN;
#pragma unroll
        for (int j = 0; j < kDistillUnroll; ++j) {
            const int32_t n = i + j * kDistillThreads;
            bits[j] = n < vectors && any ? allowed_bits(mrow, head + n * kN, kN) : 0u;
            u[j] = make_uint4(0, 0, 0, 0);
            const uint4* p = reinterpret_cast<const uint4*>(xrow + (int64_t)(head + n * kN) * (BF16 ? 2 : 4));
            if (bits[j]) u[j] = KEEP ? *p : __ldcs(p);
        }
    }
    __device__ __forceinline__ bool full() const {
        uint32_t all = bits[0];
#pragma unroll
        for (int j = 1; j < kDistillUnroll; ++j) all &= bits[j];
        return all == (1u << Vec<BF16>::kN) - 1u;
    }
};

// Tokens [t0, t1) of a row in vectors on the 16-byte boundaries of `base`:
// [t0, head) and [tail, t1) lie outside of them.
struct Cut {
    int32_t head, tail;
};
template <bool BF16>
__device__ __forceinline__ Cut cut_slice(const void* base, int32_t t0, int32_t t1) {
    constexpr int kSize = BF16 ? 2 : 4;
    const uintptr_t p = reinterpret_cast<uintptr_t>(base) + (uintptr_t)t0 * kSize;
    Cut c;
    c.head = min(t1, t0 + (int32_t)(((16 - (p & 15)) & 15) / kSize));
    c.tail = c.head + (t1 - c.head) / Vec<BF16>::kN * Vec<BF16>::kN;
    return c;
}

template <bool BF16, bool GRAD>
__global__ void __launch_bounds__(kDistillThreads, kDistillCtas) distill_kernel(const __grid_constant__ DistillCall c) {
    __shared__ DistillShared sh;
    const DistillArgs& a = c.a;
    constexpr int kN = Vec<BF16>::kN, kSize = BF16 ? 2 : 4;
    const int tid = threadIdx.x;
    // the gradient begins with the rows that the loss has read last: they may still be in L2
    const int32_t at = blockIdx.x / c.slices, slice = blockIdx.x - at * c.slices, row = GRAD ? a.rows - 1 - at : at;
    pdl_wait();
    pdl_trigger();
    const char* xrow = (const char*)a.logits + (int64_t)row * a.stride * kSize;
    const uint32_t* mrow = a.mask ? a.mask + (int64_t)row * c.W : nullptr;
    const int32_t t0 = min(a.n_tokens, slice * c.slice), t1 = min(a.n_tokens, t0 + c.slice);
    const Cut cut = cut_slice<BF16>(xrow, t0, t1);
    const int32_t vectors = (cut.tail - cut.head) / kN;
    Entries e;

    if constexpr (!GRAD) {
        float2 acc = make_float2(-INFINITY, 0.0f);   // (max, sum of exp against it)
        const auto fold1 = [&](int32_t t) {
            if (allowed_bits(mrow, t, 1)) acc = merge(acc, make_float2(load_at<BF16>(xrow, t), 1.0f), c.k);
        };
        for (int32_t t = t0 + tid; t < cut.head; t += kDistillThreads) fold1(t);
        for (int32_t t = cut.tail + tid; t < t1; t += kDistillThreads) fold1(t);
        constexpr int32_t kStep = kDistillThreads * kDistillUnroll;
        for (int32_t i = tid; i < vectors; i += kStep) {
            Batch<BF16> now;
            now.template load<true>(xrow, mrow, cut.head, vectors, i, true);
            Vec<BF16> x[kDistillUnroll];
            float top = acc.x;
            const bool full = now.full();
#pragma unroll
            for (int j = 0; j < kDistillUnroll; ++j) {
                x[j].set(now.u[j]);
                if (!full) {
#pragma unroll
                    for (int b = 0; b < kN; ++b) x[j].v[b] = (now.bits[j] >> b) & 1u ? x[j].v[b] : -INFINITY;
                }
#pragma unroll
                for (int b = 0; b < kN; b += 2) top = fmaxf(fmaxf(top, x[j].v[b]), x[j].v[b + 1]);
            }
            const float ref = sum_ref(top);
            const float2 nref = make_float2(-ref, -ref);
            float2 s0 = make_float2(acc.y * ex2((acc.x - ref) * c.k), 0.0f), s1 = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < kDistillUnroll; ++j) {
                if (now.bits[j] == 0u) continue;
#pragma unroll
                for (int b = 0; b < kN; b += 4) {
                    const float2 d0 = scale2(add2(make_float2(x[j].v[b], x[j].v[b + 1]), nref), c.k);
                    const float2 d1 = scale2(add2(make_float2(x[j].v[b + 2], x[j].v[b + 3]), nref), c.k);
                    s0 = add2(s0, make_float2(ex2(d0.x), ex2(d0.y)));
                    s1 = add2(s1, make_float2(ex2(d1.x), ex2(d1.y)));
                }
            }
            s0 = add2(s0, s1);
            acc = make_float2(top, s0.x + s0.y);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1)
            acc = merge(acc, make_float2(__shfl_xor_sync(0xffffffffu, acc.x, off), __shfl_xor_sync(0xffffffffu, acc.y, off)), c.k);
        if ((tid & 31) == 0) {
            sh.red[2 * (tid >> 5)] = acc.x;
            sh.red[2 * (tid >> 5) + 1] = acc.y;
        }
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kDistillWarps; ++w) acc = merge(acc, make_float2(sh.red[2 * w], sh.red[2 * w + 1]), c.k);
            sh.part = acc;
        }
        if (c.slices > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            cluster.sync();
            if (slice == 0 && tid == 0)
                for (int s = 1; s < c.slices; ++s) acc = merge(acc, *cluster.map_shared_rank(&sh.part, s), c.k);
            cluster.sync();
            if (slice) return;
        }
        if (tid == 0) sh.lse = isnan(acc.y) ? acc.y : log_sum_exp(scaled(acc.x, c), acc.y);
        __syncthreads();
        const float lse = sh.lse;
        read_entries<BF16>(e, c, row, xrow, mrow, sh, true);
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kDistillEntries; ++j)
            if (e.id[j] >= 0 && e.p[j] != 0.0f) sum += e.p[j] * (e.logp[j] - (scaled(e.x[j], c) - lse));
        sum = cta_reduce<false>(sum, sh.red);
        if (tid == 0) {
            if (a.lse) a.lse[row] = lse;
            a.loss[row] = e.any ? a.temperature * a.temperature * sum : 0.0f;
        }
    } else {
        char* drow = (char*)a.dlogits + (int64_t)row * a.dstride * kSize;
        const float lse = a.lse[row];
        read_entries<BF16>(e, c, row, xrow, mrow, sh, slice == 0);
        // the entries' logits have been read by every CTA of the row before any is written over
        if (c.slices > 1) cg::this_cluster().sync();
        const float g = e.any ? __ldg(a.grad_loss + row) * a.temperature : 0.0f;
        const auto q = [&](float x) { return ex2((scaled(x, c) - lse) * kLog2e); };
        const auto grad1 = [&](int32_t t) {
            store_at<BF16>(drow, t, g != 0.0f && allowed_bits(mrow, t, 1) ? g * q(load_at<BF16>(xrow, t)) : 0.0f);
        };
        // a gradient whose rows lie otherwise against 16-byte boundaries than the logits' is written one by one
        const bool same = ((reinterpret_cast<uintptr_t>(xrow) ^ reinterpret_cast<uintptr_t>(drow)) & 15) == 0;
        const int32_t head = same ? cut.head : t1, tail = same ? cut.tail : t1;
        for (int32_t t = t0 + tid; t < head; t += kDistillThreads) grad1(t);
        for (int32_t t = tail + tid; t < t1; t += kDistillThreads) grad1(t);
        constexpr int32_t kStep = kDistillThreads * kDistillUnroll;
        const bool any = g != 0.0f;
        const float2 nlse = make_float2(-lse, -lse);
        for (int32_t i = tid; same && i < vectors; i += kStep) {
            Batch<BF16> now;
            now.template load<false>(xrow, mrow, cut.head, vectors, i, any);
            const bool full = now.full();
#pragma unroll
            for (int j = 0; j < kDistillUnroll; ++j) {
                const int32_t n = i + j * kDistillThreads;
                if (n >= vectors) break;
                uint4 out = make_uint4(0, 0, 0, 0);
                if (now.bits[j]) {
                    Vec<BF16> x;
                    x.set(now.u[j]);
#pragma unroll
                    for (int b = 0; b < kN; b += 2) {
                        const float2 d = scale2(add2(scale2(make_float2(x.v[b], x.v[b + 1]), c.inv_tau), nlse), kLog2e);
                        const float2 y = scale2(make_float2(ex2(d.x), ex2(d.y)), g);
                        x.v[b] = y.x;
                        x.v[b + 1] = y.y;
                    }
                    if (!full) {
#pragma unroll
                        for (int b = 0; b < kN; ++b) x.v[b] = (now.bits[j] >> b) & 1u ? x.v[b] : 0.0f;
                    }
                    out = x.get();
                }
                __stcs(reinterpret_cast<uint4*>(drow + (int64_t)(cut.head + n * kN) * kSize), out);
            }
        }
        __syncthreads();
        // the entries' tokens of this slice again, with the teacher's part
#pragma unroll
        for (int j = 0; j < kDistillEntries; ++j)
            if (e.id[j] >= t0 && e.id[j] < t1 && g != 0.0f)
                store_at<BF16>(drow, e.id[j], g * (q(e.x[j]) - e.p[j]));
    }
}

template <bool BF16, bool GRAD>
cudaError_t launch(const DistillCall& c, cudaStream_t st) {
    return launch_cluster(distill_kernel<BF16, GRAD>, dim3((unsigned)c.a.rows * (unsigned)c.slices), dim3(kDistillThreads),
                          c.slices, 0, st, c);
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& a, const LaunchEnv& env, bool grad, cudaStream_t st) {
    DistillCall c{};
    c.a = a;
    c.W = (a.n_tokens + 31) / 32;
    int s = 1;
    while (s < kDistillMaxSlices && (int64_t)a.rows * s * 2 <= env.num_sms * 2 && a.n_tokens > 4096 * s) s *= 2;
    c.slices = s;
    c.slice = ((a.n_tokens + s - 1) / s + 31) / 32 * 32;
    for (c.slots = 64; c.slots < 2 * a.k; c.slots *= 2) {}
    c.inv_tau = 1.0f / a.temperature;
    c.k = kLog2e / a.temperature;
    if (a.dtype == DOMINO_DTYPE_BF16) return grad ? launch<true, true>(c, st) : launch<true, false>(c, st);
    return grad ? launch<false, true>(c, st) : launch<false, false>(c, st);
}

}  // namespace domino
