// embed.cu -- rows of an embedding table for a list of tokens, and the table's
// gradient (sm_103a).
//
//   out[i]  = scale W[tokens[i]]              zeros for tokens below 0
//   dW[v]   = scale sum_{i: tokens[i] = v} g[i]
//
// Both are bound by HBM.  The gradient sorts the tokens (stable, so that a
// row's sum is always made in the same order) and sums runs of equal
// tokens in fp32: a CTA per chunk of the sorted list and stretch of columns; a
// run that crosses chunks is kept in parts, which a second pass joins in order.
// One cluster sorts while the others write the table's zeros.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "bf16_rows.cuh"
#include "loss.h"
#include "walk_common.cuh"

namespace cg = cooperative_groups;

namespace domino {
namespace {

constexpr int kEmbedThreads = 256;
// Pieces of a thread: 16384 x 4096 bf16 39.7 us with four, 37.0 with two, 41.6 with one (32 x 4096 2.9, 2.1, 1.9).
constexpr int kEmbedUnroll = 2;
constexpr int64_t kFarBytes = (int64_t)64 << 20;

template <bool BF16>
__device__ __forceinline__ uint4 scaled(const uint4& u, float scale) {
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(w[i] << 16) * scale,
                                                           __uint_as_float(w[i] & 0xFFFF0000u) * scale);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        } else {
            w[i] = __float_as_uint(__uint_as_float(w[i]) * scale);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A thread takes kEmbedUnroll pieces (16-byte vectors, or with !VEC single fp32
// values) of the output's `per_row` a row, a grid's width apart.  far: an output of half the L2 or more is written past it
// (37.0 -> 35.3 us).
template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedArgs a, const uint32_t per_row, const int64_t pieces, const bool far) {
    pdl_wait();
    pdl_trigger();
    constexpr int kSize = BF16 ? 2 : 4;
    const int64_t width = (int64_t)gridDim.x * kEmbedThreads;
    int64_t at[kEmbedUnroll];
    uint4 u[kEmbedUnroll];
#pragma unroll
    for (int j = 0; j < kEmbedUnroll; ++j) {
        const int64_t i = (int64_t)blockIdx.x * kEmbedThreads + threadIdx.x + j * width;
        at[j] = -1;
        u[j] = make_uint4(0, 0, 0, 0);
        if (i >= pieces) continue;
        const uint32_t r = pieces <= UINT_MAX ? (uint32_t)i / per_row : (uint32_t)(i / per_row);
        const uint32_t c = (uint32_t)(i - (int64_t)r * per_row);
        const int32_t t = __ldg(a.tokens + r);
        at[j] = (int64_t)r * a.out_stride + (int64_t)c * (VEC ? 16 / kSize : 1);
        if (t >= 0 && t < a.n_tokens) {
            const int64_t from = (int64_t)t * a.weight_stride + (int64_t)c * (VEC ? 16 / kSize : 1);
            if constexpr (VEC) u[j] = __ldg(reinterpret_cast<const uint4*>((const char*)a.weight + from * kSize));
            else u[j].x = __float_as_uint(__ldg((const float*)a.weight + from));
        } else if (t >= a.n_tokens && c == 0) {
            atomicOr(a.err, DOMINO_DEVERR_BAD_TOKEN);
        }
    }
#pragma unroll
    for (int j = 0; j < kEmbedUnroll; ++j) {
        if (at[j] < 0) continue;
        if constexpr (VEC) {
            uint4* to = reinterpret_cast<uint4*>((char*)a.out + at[j] * kSize);
            const uint4 x = scaled<BF16>(u[j], a.scale);
            if (far) __stcs(to, x);
            else *to = x;
        } else {
            ((float*)a.out)[at[j]] = __uint_as_float(u[j].x) * a.scale;
        }
    }
}

// bf16 rows off 16-byte boundaries: a warp takes 256 columns of a row.
__global__ void __launch_bounds__(kEmbedThreads) embed_any_kernel(const EmbedArgs a, const int32_t stretches) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t i = (int64_t)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5);
    const int32_t r = (int32_t)(i / stretches), c = (int32_t)(i - (int64_t)r * stretches) * 256 + lane * kN;
    if (r >= a.n) return;
    const int32_t t = __ldg(a.tokens + r), left = a.dim - c;
    if (t >= a.n_tokens && c == 0) atomicOr(a.err, DOMINO_DEVERR_BAD_TOKEN);
    Eight x;
    x.zero();
    if (t >= 0 && t < a.n_tokens && left > 0) x.load((const __nv_bfloat16*)a.weight + (int64_t)t * a.weight_stride + c, left);
    float v[kN];
    x.get(v);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k] * a.scale, v[2 * k + 1] * a.scale);
        w[k] = *reinterpret_cast<const uint32_t*>(&b);
    }
    store_any((__nv_bfloat16*)a.out + (int64_t)r * a.out_stride + c, w, left, lane);
}

// ---- the list sorted by token ---------------------------------------------------
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortCtas = 8;               // one cluster
constexpr int kSortBits = 8;               // at most, of a token id per pass
constexpr int kSortBins = 1 << kSortBits;
constexpr int kCountTokens = 1024, kCountParts = 16, kCountEntries = kSortThreads / kCountParts;
static_assert(kCountTokens <= kSortWarps * kSortBins);

struct SortArgs {
    const int32_t* tokens;
    int32_t n, n_tokens;
    int32_t passes, bits;      // bits per pass
    int32_t ctas;
    uint2* a;                  // [n] {token (n_tokens: none), place in the list}
    uint2* b;                  // [n]
    uint32_t* err;
    // the table to be cleared by the clusters after the first: fill_rows rows of fill_bytes (one row where
    // they follow each other), each a multiple of fill_size
    char* fill;
    int64_t fill_pitch, fill_bytes, fill_rows;
    int32_t fill_size;
};

// Zeros to bytes [0, n) at p, by threads `at`, `at` + step, ...
__device__ __forceinline__ void clear(char* p, int64_t n, int size, int64_t at, int64_t step) {
    int64_t head = (int64_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15);
    head = head < n ? head : n;
    const int64_t vectors = (n - head) / 16, tail = head + 16 * vectors;
    for (int64_t i = at; i < vectors; i += step) __stcs(reinterpret_cast<uint4*>(p + head) + i, make_uint4(0, 0, 0, 0));
    const int64_t edge = (head + n - tail) / size;   // values beside the vectors
    for (int64_t i = at; i < edge; i += step) {
        char* q = i * size < head ? p + i * size : p + tail + (i * size - head);
        if (size == 2) *reinterpret_cast<uint16_t*>(q) = 0;
        else *reinterpret_cast<uint32_t*>(q) = 0u;
    }
}

// Up to kCountTokens tokens: counted, a CTA for every kCountEntries of them (192
// tokens 2.8 us, by digits 6.8; the whole gradient of 4000 tokens x 1001 28.1 us, by digits 23.4).  More:
// stable least-significant-digit radix sort by one cluster.  The list is cut
// into one strip per warp.  A pass counts the strips' digits, turns the counts
// into places (all smaller digits first, then the same digit of earlier CTAs
// and warps), and moves every strip in order.  The last pass ends in `a`.
__global__ void __launch_bounds__(kSortThreads) sort_kernel(const SortArgs s) {
    __shared__ __align__(16) uint32_t count[kSortWarps][kSortBins];
    __shared__ uint32_t total[kSortBins], base[kSortBins], warp_sum[kSortBins / 32];
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
    pdl_wait();
    pdl_trigger();
    if (cta >= s.ctas) {
        const int64_t threads = (int64_t)(gridDim.x - s.ctas) * kSortThreads, at = (int64_t)(cta - s.ctas) * kSortThreads + tid;
        if (s.fill_rows == 1) clear(s.fill, s.fill_bytes, s.fill_size, at, threads);
        else
            for (int64_t r = at / 32; r < s.fill_rows; r += threads / 32) clear(s.fill + r * s.fill_pitch, s.fill_bytes, s.fill_size, lane, 32);
        return;
    }
    if (s.n == 0) return;
    if (s.n <= kCountTokens) {   // an entry's place is the number of entries before it: kCountParts threads an entry
        uint32_t* keys = &count[0][0];
        for (int j = tid; j < (s.n + 3) / 4 * 4; j += kSortThreads) {
            uint32_t key = ~0u;
            if (j < s.n) {
                const int32_t t = __ldg(s.tokens + j);
                if (t >= s.n_tokens && cta == 0) atomicOr(s.err, DOMINO_DEVERR_BAD_TOKEN);
                key = (uint32_t)(t < 0 || t >= s.n_tokens ? s.n_tokens : t);
            }
            keys[j] = key;
        }
        __syncthreads();
        const int at = cta * kCountEntries + tid / kCountParts, part = tid % kCountParts;
        const uint32_t key = at < s.n ? keys[at] : 0u;
        uint32_t place = 0;
        for (int j = 4 * part; j < s.n; j += 4 * kCountParts) {
            const uint4 k = *reinterpret_cast<const uint4*>(keys + j);
            place += (k.x < key || (k.x == key && j < at)) + (k.y < key || (k.y == key && j + 1 < at)) +
                     (k.z < key || (k.z == key && j + 2 < at)) + (k.w < key || (k.w == key && j + 3 < at));
        }
#pragma unroll
        for (int off = kCountParts / 2; off > 0; off >>= 1) place += __shfl_xor_sync(0xffffffffu, place, off);
        if (part == 0 && at < s.n) s.a[place] = make_uint2(key, (uint32_t)at);
        return;
    }
    const int64_t strips = (int64_t)s.ctas * kSortWarps, strip = (int64_t)cta * kSortWarps + warp;
    const int32_t lo = (int32_t)(s.n * strip / strips), hi = (int32_t)(s.n * (strip + 1) / strips);
    const uint32_t bins = 1u << s.bits, digit_mask = bins - 1u;
    for (int pass = 0; pass < s.passes; ++pass) {
        const int shift = pass * s.bits;
        // passes alternate between the buffers, the last into `a`
        uint2* to = (s.passes - pass) & 1 ? s.a : s.b;
        const uint2* from = (s.passes - pass) & 1 ? s.b : s.a;
        const auto entry = [&](int32_t i) {
            if (pass) return from[i];
            int32_t t = __ldg(s.tokens + i);
            if (t >= s.n_tokens) atomicOr(s.err, DOMINO_DEVERR_BAD_TOKEN);
            if (t < 0 || t >= s.n_tokens) t = s.n_tokens;
            return make_uint2((uint32_t)t, (uint32_t)i);
        };
        for (uint32_t i = lane; i < bins; i += 32) count[warp][i] = 0u;
        __syncwarp();
        for (int32_t i = lo + lane; i < hi; i += 32) atomicAdd(&count[warp][(entry(i).x >> shift) & digit_mask], 1u);
        __syncthreads();
        if (tid < (int)bins) {   // before each warp's: the CTA's earlier warps'
            uint32_t n[kSortWarps], sum = 0;   // read before any is written: the reads do not wait for one another
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) n[w] = count[w][tid];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                count[w][tid] = sum;
                sum += n[w];
            }
            total[tid] = sum;
        }
        cluster.sync();
        uint32_t all = 0, before = 0;
        if (tid < (int)bins) {
            uint32_t n[kSortCtas];
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) n[c] = c < s.ctas ? *cluster.map_shared_rank(&total[tid], c) : 0u;
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) {
                all += n[c];
                if (c < cta) before += n[c];
            }
        }
        uint32_t scan = all;   // of the bins: smaller digits
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, scan, off);
            if (lane >= off) scan += x;
        }
        if (lane == 31 && warp < kSortBins / 32) warp_sum[warp] = scan;
        __syncthreads();
        if (tid < (int)bins) {
            uint32_t smaller = scan - all;
#pragma unroll
            for (int w = 0; w < kSortBins / 32; ++w) smaller += w < warp ? warp_sum[w] : 0u;
            base[tid] = smaller + before;
        }
        __syncthreads();
        for (int32_t i0 = lo; i0 < hi; i0 += 32) {
            const int32_t i = i0 + lane;
            const bool on = i < hi;
            uint2 e = make_uint2(0u, 0u);
            if (on) e = entry(i);
            const uint32_t d = on ? (e.x >> shift) & digit_mask : bins;
            const uint32_t peers = __match_any_sync(0xffffffffu, d);
            const uint32_t rank = __popc(peers & ((1u << lane) - 1u));
            uint32_t place = 0;
            if (on) place = base[d] + count[warp][d] + rank;
            __syncwarp();
            if (on && rank == 0) count[warp][d] += __popc(peers);
            __syncwarp();
            if (on) to[place] = e;
        }
        __threadfence();
        cluster.sync();   // also: the others have read this CTA's totals
    }
}

// ---- sums of runs -----------------------------------------------------------------
constexpr int kSumThreads = 128;
constexpr int kSumUnroll = 8;
constexpr int kSumChunk = 32;              // of the sorted list whose places are in shared memory at a time

struct SumArgs {
    EmbedArgs a;
    const uint2* order;
    int32_t chunk, chunks;
    int32_t stretches;         // of the columns, kSumThreads pieces each
    int32_t pitch;             // dim, rounded up to 8
    float* part;               // [chunks][2][pitch]: the run that began before the chunk; the one that goes on after it
};

// A thread's columns: VEC: a 16-byte vector; else one fp32 value, or eight bf16 at any alignment.
template <bool BF16, bool VEC>
struct Piece {
    static constexpr int kCols = BF16 ? 8 : VEC ? 4 : 1;
    float v[kCols];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kCols; ++i) v[i] = 0.0f;
    }
    // as it lies in memory
    using Raw = std::conditional_t<BF16 && !VEC, Eight, uint4>;
    static __device__ __forceinline__ Raw nothing() {
        Raw r;
        if constexpr (BF16 && !VEC) r.zero();
        else r = make_uint4(0u, 0u, 0u, 0u);
        return r;
    }
    // value i of p, the row's end `left` values further
    static __device__ __forceinline__ Raw fetch(const void* p, int64_t i, int32_t left) {
        Raw r;
        if constexpr (VEC) r = __ldcs(reinterpret_cast<const uint4*>((const char*)p + i * (BF16 ? 2 : 4)));
        else if constexpr (BF16) r.load((const __nv_bfloat16*)p + i, left);
        else r = make_uint4(__float_as_uint(((const float*)p)[i]), 0u, 0u, 0u);
        return r;
    }
    __device__ __forceinline__ void add(const Raw& r) {
        if constexpr (BF16 && !VEC) {
            float x[kN];
            r.get(x);
#pragma unroll
            for (int k = 0; k < kCols; ++k) v[k] += x[k];
        } else {
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int k = 0; k < (VEC ? 4 : 1); ++k) {
                if constexpr (BF16) {
                    v[2 * k] += __uint_as_float(w[k] << 16);
                    v[2 * k + 1] += __uint_as_float(w[k] & 0xFFFF0000u);
                } else {
                    v[k] += __uint_as_float(w[k]);
                }
            }
        }
    }
    // every thread of the warp calls it (left <= 0: nothing of its own)
    __device__ __forceinline__ void store(void* p, int64_t i, int32_t left) const {
        if constexpr (BF16) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
                w[k] = *reinterpret_cast<const uint32_t*>(&b);
            }
            if constexpr (!VEC) store_any((__nv_bfloat16*)p + i, w, left, threadIdx.x & 31);
            else if (left > 0) *reinterpret_cast<uint4*>((__nv_bfloat16*)p + i) = make_uint4(w[0], w[1], w[2], w[3]);
        } else if (left > 0) {
            if constexpr (VEC) *reinterpret_cast<float4*>((float*)p + i) = make_float4(v[0], v[1], v[2], v[3]);
            else ((float*)p)[i] = v[0];
        }
    }
};

// One row's sum is complete: scaled, with what dW holds where asked for, rounded once.
template <bool BF16, bool VEC>
__device__ __forceinline__ void finish_row(const EmbedArgs& a, uint32_t token, int32_t c, Piece<BF16, VEC> sum) {
    const int64_t at = (int64_t)token * a.dweight_stride + c;
    const int32_t left = a.dim - c;
#pragma unroll
    for (int i = 0; i < sum.kCols; ++i) sum.v[i] *= a.scale;
    if (a.add && left > 0) sum.add(Piece<BF16, VEC>::fetch(a.dweight, at, left));
    sum.store(a.dweight, at, left);
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const SumArgs s) {
    using P = Piece<BF16, VEC>;
    const EmbedArgs& a = s.a;
    pdl_wait();
    pdl_trigger();
    const int32_t chunk = blockIdx.x / s.stretches, stretch = blockIdx.x - chunk * s.stretches;
    const int32_t c = (stretch * kSumThreads + threadIdx.x) * P::kCols;
    const bool on = c < a.dim;
    const int32_t lo = chunk * s.chunk, hi = min(a.n, lo + s.chunk);
    const uint32_t none = (uint32_t)a.n_tokens;
    // entry lo - 1 + i; none outside of the list
    __shared__ uint2 s_order[kSumChunk + 2];
    const auto stage = [&](int32_t from) {
        const int32_t i = from - 1 + (int32_t)threadIdx.x;
        if (threadIdx.x < kSumChunk + 2) s_order[threadIdx.x] = i >= 0 && i < a.n ? s.order[i] : make_uint2(none, 0u);
        __syncthreads();
    };
    stage(lo);
    const uint32_t before = s_order[0].x;
    float* part = s.part + (int64_t)chunk * 2 * s.pitch + c;
    P sum;
    sum.zero();
    uint32_t token = s_order[1].x;
    bool first = true;   // the chunk's first run
    const auto flush = [&](bool last, uint32_t after) {
        if (token == none) return;
        const bool head = first && token == before;
        if (head || (last && token == after)) {
            float* to = head ? part : part + s.pitch;
            if (on)
#pragma unroll
                for (int i = 0; i < P::kCols; ++i) to[i] = sum.v[i];
        } else {
            finish_row<BF16, VEC>(a, token, c, sum);
        }
    };
    constexpr int kUnroll = BF16 && !VEC ? kSumUnroll / 2 : kSumUnroll;   // two loads each
    for (int32_t b0 = lo; b0 < hi; b0 += kSumChunk) {
        if (b0 > lo) {
            __syncthreads();
            stage(b0);
        }
        const int n = min(kSumChunk, hi - b0);
        for (int j0 = 0; j0 < n; j0 += kUnroll) {
            typename P::Raw g[kUnroll];
#pragma unroll
            for (int j = 0; j < kUnroll; ++j) {
                g[j] = P::nothing();
                if (on && j0 + j < n && s_order[1 + j0 + j].x != none)
                    g[j] = P::fetch(a.grad, (int64_t)s_order[1 + j0 + j].y * a.grad_stride + c, a.dim - c);
            }
#pragma unroll
            for (int j = 0; j < kUnroll; ++j) {
                if (j0 + j >= n) break;
                const uint32_t t = s_order[1 + j0 + j].x;
                if (t != token) {
                    flush(false, none);
                    first = false;
                    token = t;
                    sum.zero();
                }
                sum.add(g[j]);
            }
        }
        if (b0 + n == hi) flush(true, s_order[1 + n].x);
    }
}

// The runs that cross chunks: each by the CTAs of the chunk that it begins in; one
// look at the first tokens of 32 following chunks, then their sums, eight at a
// time.  (Groups of threads for the eights: four times the threads of the many CTAs
// that have no such run, 16384 tokens x 4096 11 -> 20 us.)

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kSumThreads) join_kernel(const SumArgs s) {
    using P = Piece<BF16, VEC>;
    const EmbedArgs& a = s.a;
    pdl_wait();
    pdl_trigger();
    const int32_t chunk = blockIdx.x / s.stretches, stretch = blockIdx.x - chunk * s.stretches;
    const int lane = threadIdx.x & 31;
    const int32_t c = (stretch * kSumThreads + threadIdx.x) * P::kCols;
    const int32_t lo = chunk * s.chunk, hi = lo + s.chunk;
    if (hi >= a.n) return;
    const bool on = c < a.dim;
    const uint32_t token = s.order[hi - 1].x;
    if (token == (uint32_t)a.n_tokens || s.order[hi].x != token) return;         // no run goes on after the chunk
    if (s.order[lo].x == token && lo > 0 && s.order[lo - 1].x == token) return;   // it began before the chunk
    P sum;
    sum.zero();
    const float* part = s.part + (int64_t)chunk * 2 * s.pitch + c;
    if (on)
#pragma unroll
        for (int i = 0; i < P::kCols; ++i) sum.v[i] = part[s.pitch + i];
    for (int32_t k = chunk + 1; k < s.chunks; k += 32) {
        // the chunks that begin with the token: the first `more` of the 32 (the list is sorted)
        const bool same = k + lane < s.chunks && s.order[(int64_t)(k + lane) * s.chunk].x == token;
        const int more = __popc(__ballot_sync(0xffffffffu, same));
#pragma unroll 2
        for (int j0 = 0; j0 < more; j0 += kSumUnroll) {
            float v[kSumUnroll][P::kCols];
#pragma unroll
            for (int j = 0; j < kSumUnroll; ++j)
#pragma unroll
                for (int i = 0; i < P::kCols; ++i)
                    v[j][i] = on && j0 + j < more ? part[(int64_t)(k + j0 + j - chunk) * 2 * s.pitch + i] : 0.0f;
#pragma unroll
            for (int j = 0; j < kSumUnroll; ++j)
#pragma unroll
                for (int i = 0; i < P::kCols; ++i) sum.v[i] += v[j][i];
        }
        if (more < 32) break;
    }
    finish_row<BF16, VEC>(a, token, c, sum);
}

// ---- host --------------------------------------------------------------------------
bool vectors_fit(const void* p, int64_t stride, int32_t dim, int size) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && (int64_t)dim * size % 16 == 0;
}

template <bool BF16, bool VEC>
cudaError_t launch_rows(const EmbedArgs& a, cudaStream_t st) {
    const uint32_t per_row = (uint32_t)(VEC ? a.dim * (BF16 ? 2 : 4) / 16 : a.dim);
    const int64_t pieces = (int64_t)a.n * per_row;
    const int64_t ctas = (pieces + kEmbedThreads * kEmbedUnroll - 1) / (kEmbedThreads * kEmbedUnroll);
    if (ctas > INT_MAX) return cudaErrorInvalidValue;
    return launch_pdl(embed_kernel<BF16, VEC>, dim3((unsigned)ctas), dim3(kEmbedThreads), 0, st, a, per_row, pieces,
                      (int64_t)a.n * a.dim * (BF16 ? 2 : 4) >= kFarBytes);
}

struct EmbedSpace {
    size_t a, b, part, end;
    int32_t chunk, chunks;
};
// Chunks of the sorted list: one round of loads each while that gives the SMs no more than eight CTAs (100 of 5000 tokens,
// 256 wide: 6.7 us with chunks of 32), at most 4096 in all (a run that crosses chunks is joined by one CTA).
EmbedSpace embed_space(const EmbedArgs& a, const LaunchEnv& env) {
    EmbedSpace s{};
    s.chunk = kSumUnroll;
    const int64_t stretches = (a.dim + kSumThreads * 4 - 1) / (kSumThreads * 4);
    while ((s.chunk < kSumChunk && a.n * stretches > (int64_t)s.chunk * env.num_sms * 8) || (int64_t)s.chunk * 4096 < a.n)
        s.chunk *= 2;
    s.chunks = (a.n + s.chunk - 1) / s.chunk;
    const auto align = [](size_t n) { return (n + 255) & ~(size_t)255; };
    s.b = align((size_t)a.n * sizeof(uint2));
    s.part = 2 * s.b;
    s.end = s.part + align((size_t)s.chunks * 2 * (((size_t)a.dim + 7) / 8 * 8) * 4);
    return s;
}

template <bool BF16, bool VEC>
cudaError_t launch_sums(const EmbedArgs& a, const SumArgs& in, cudaStream_t st) {
    SumArgs s = in;
    constexpr int kCols = Piece<BF16, VEC>::kCols;
    s.stretches = (a.dim + kSumThreads * kCols - 1) / (kSumThreads * kCols);
    const dim3 grid((unsigned)s.chunks * (unsigned)s.stretches);
    cudaError_t e = launch_pdl(sum_kernel<BF16, VEC>, grid, dim3(kSumThreads), 0, st, s);
    if (e != cudaSuccess || s.chunks == 1) return e;
    return launch_pdl(join_kernel<BF16, VEC>, grid, dim3(kSumThreads), 0, st, s);
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs& a, const LaunchEnv&, cudaStream_t st) {
    const bool bf16 = a.dtype == DOMINO_DTYPE_BF16;
    const int size = bf16 ? 2 : 4;
    const bool vec = vectors_fit(a.weight, a.weight_stride, a.dim, size) && vectors_fit(a.out, a.out_stride, a.dim, size);
    if (bf16 && !vec) {
        const int32_t stretches = (a.dim + 255) / 256;
        const int64_t ctas = ((int64_t)a.n * stretches + kEmbedThreads / 32 - 1) / (kEmbedThreads / 32);
        if (ctas > INT_MAX) return cudaErrorInvalidValue;
        return launch_pdl(embed_any_kernel, dim3((unsigned)ctas), dim3(kEmbedThreads), 0, st, a, stretches);
    }
    if (bf16) return launch_rows<true, true>(a, st);
    return vec ? launch_rows<false, true>(a, st) : launch_rows<false, false>(a, st);
}

size_t embed_workspace(const EmbedArgs& a, const LaunchEnv& env) { return embed_space(a, env).end; }

cudaError_t launch_embed_grad(const EmbedArgs& a, const LaunchEnv& env, void* space, cudaStream_t st) {
    const bool bf16 = a.dtype == DOMINO_DTYPE_BF16;
    const int size = bf16 ? 2 : 4;
    if (a.n == 0 && a.add) return cudaSuccess;
    const EmbedSpace sp = embed_space(a, env);
    char* ws = (char*)space;
    SortArgs so{};
    so.tokens = a.tokens;
    so.n = a.n;
    so.n_tokens = a.n_tokens;
    int bits = 1;   // of the ids 0..n_tokens
    while ((a.n_tokens >> bits) > 0) ++bits;
    so.passes = (bits + kSortBits - 1) / kSortBits;
    so.bits = (bits + so.passes - 1) / so.passes;
    so.ctas = kSortCtas;
    while (so.ctas > 1 && a.n <= so.ctas / 2 * kSortThreads) so.ctas /= 2;
    int cluster = so.ctas;
    if (a.n <= kCountTokens) {
        so.ctas = (a.n + kCountEntries - 1) / kCountEntries;
        cluster = 1;
    }
    so.a = (uint2*)(ws + sp.a);
    so.b = (uint2*)(ws + sp.b);
    so.err = a.err;
    int ctas = so.ctas;
    if (!a.add) {
        const bool flat = a.dweight_stride == a.dim;
        so.fill = (char*)a.dweight;
        so.fill_size = size;
        so.fill_rows = flat ? 1 : a.n_tokens;
        so.fill_pitch = a.dweight_stride * size;
        so.fill_bytes = (int64_t)a.dim * size * (flat ? a.n_tokens : 1);
        ctas += 2 * env.num_sms / cluster * cluster;
    }
    cudaError_t e = launch_cluster(sort_kernel, dim3((unsigned)ctas), dim3(kSortThreads), cluster, 0, st, so);
    if (e != cudaSuccess || a.n == 0) return e;
    SumArgs s{};
    s.a = a;
    s.order = so.a;
    s.chunk = sp.chunk;
    s.chunks = sp.chunks;
    s.pitch = (a.dim + 7) / 8 * 8;
    s.part = (float*)(ws + sp.part);
    const bool vec = vectors_fit(a.grad, a.grad_stride, a.dim, size) && vectors_fit(a.dweight, a.dweight_stride, a.dim, size);
    if (bf16) return vec ? launch_sums<true, true>(a, s, st) : launch_sums<true, false>(a, s, st);
    return vec ? launch_sums<false, true>(a, s, st) : launch_sums<false, false>(a, s, st);
}

}  // namespace domino
