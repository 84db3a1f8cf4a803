// penalized.cu -- the decode of given masks with penalties for what a row has said and
// biases (sm_103a): a row's logits changed at the tokens of its history and its biases,
// then the masked argmax / log-sum-exp / log-probabilities, or a Gumbel-max draw.
//
//   n > 0: x = x > 0 ? x / repetition : x repetition     n: times in the history
//   c > 0: x = (x - frequency c) - presence              c: of them beyond the prompt
//   x = x + bias
//
// Few of a row's tokens change.  A CTA (or each of a cluster's that share out the row's
// mask words) marks them in a bit map in shared memory, takes them out of the mask and
// decodes the rest as decode.cuh does, bound by HBM; the marked ones, numbered by the
// set bits before them, get a counter each, then their logit, and are folded on their
// own.  Whole-number atomics only: the results are the same on every run.
//
// 256 x 128256 bf16, a third of the rows dense, histories of up to 4096 tokens: 28 us, of which
// the decode alone takes 24 (the bytes' floor is 10.6): most SMs have two of the 256 rows, and a
// row's fold waits for its loads and for its own results (the SMs issue in half of the
// cycles).  More CTAs a row cost more than they share out: 32 us with two, 52 with four.  One
// row is a chain of five latencies of memory and ten barriers: 7.9 us.  Draws: 96 us, 89 with
// histories of up to 64 tokens (greedy 24); one row 8.7.
#include <algorithm>
#include <atomic>

#include "decode.cuh"
#include "norm.h"

namespace domino {
namespace {

// Mask words of a row at a time, at most: 131072 tokens, most vocabularies whole.  More go in two parts (160 x 131072 24 us,
// with log-probabilities, for which each part is made again, 44; x 152064 33 and 65), unless two CTAs share them out (128 x
// 152064 20 and 33).
constexpr int kSegmentWords = 4096;
constexpr int kBiasEach = kMaxBias / kDecodeThreads;
// Of a CTA, at most.  Long histories take an SM for a row rather than more parts of it: 100 x 128256 with 16000 tokens each 36
// us, in parts that leave room for two CTAs an SM 132.
constexpr int kPenalizedSmem = 212 * 1024;
constexpr int kQuads = kSegmentWords / 4 / kDecodeThreads;   // four mask words each, of a thread
constexpr int kHeld = 8;                   // history tokens a thread keeps, of each 512
static_assert(kQuads == 2 && kBiasEach * kDecodeThreads == kMaxBias);

struct Rows {
    const void* logits;
    int64_t stride;
    const uint32_t* mask;          // nullptr: every token allowed
    domino_penalties p;
    int32_t V, W;
    int32_t slices, slice_words;   // CTAs per row, mask words of each (a multiple of 4)
    int32_t segment, places;       // mask words at a time (a multiple of 4), changed tokens in them at most
    int32_t* argmax;
    float* lse;
    float* logprobs;
    SampleArgs sample;
    uint32_t* err;
};

// Shared memory of a segment: mask words between zero words, changed tokens' words, the number of changed tokens before
// each word, the changed tokens' places and values, the decode's lists.
struct Layout {
    int mask, changed, before, place, value, list, end;
};
__host__ __device__ inline Layout layout(int segment, int places) {
    Layout l;
    l.mask = 16;
    l.changed = l.mask + segment * 4 + 16;
    l.before = l.changed + segment * 4;
    l.value = (l.before + segment * 2 + 15) & ~15;   // segment: a multiple of 4, places of 8
    l.place = l.value + places * 4;
    l.list = l.place + places * 4;
    l.end = l.list + kDecodeListBytes;
    return l;
}

// A segment of a row: mask words w0, .. w0 + n - 1.
struct Segment {
    uint32_t* mask;
    uint32_t* changed;
    uint16_t* before;
    uint32_t* value;
    uint32_t* place;               // from the segment's first token on
    int w0, n;
    int total;                     // changed tokens that are allowed

    // The number of token t, or -1: not in this segment, not changed or not allowed.
    __device__ __forceinline__ int number(int32_t t) const {
        const uint32_t j = (uint32_t)(t >> 5) - (uint32_t)w0;
        if (t < 0 || j >= (uint32_t)n) return -1;
        const uint32_t word = changed[j], bit = 1u << (t & 31);
        return word & bit ? before[j] + __popc(word & (bit - 1u)) : -1;
    }
    // Marks token t.
    __device__ __forceinline__ void mark(int32_t t, int32_t V, uint32_t* report) const {
        if (t >= V) {
            if (report) atomicOr(report, DOMINO_DEVERR_BAD_TOKEN);
            return;
        }
        const uint32_t j = (uint32_t)(t >> 5) - (uint32_t)w0;
        if (t >= 0 && j < (uint32_t)n) atomicOr(changed + j, 1u << (t & 31));
    }
};

// The segment's masks, its changed tokens and their values.  Every thread of the CTA calls it, with shared memory that
// nothing reads any more; it ends with a barrier.  report: the first time for a row.
template <bool BF16>
__device__ __forceinline__ void make_segment(Segment& g, const Rows& a, int r, int len, const char* lrow, uint32_t* report, int tid) {
    __shared__ int s_sum[kQuads][kDecodeWarps];
    const int lane = tid & 31, warp = tid >> 5;
    const uint32_t* mrow = a.mask ? a.mask + (int64_t)r * a.W + g.w0 : nullptr;
    const int32_t* hist = a.p.history_dev + (int64_t)r * a.p.history_len;
    const int32_t* ids = a.p.bias_ids_dev + (int64_t)r * a.p.n_bias;
    const int n_bias = a.p.n_bias;
    // the first tokens of the history and the ids are on their way beside the masks, and stay for the second pass
    int32_t held[kHeld], id[kBiasEach];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        const int i = tid + k * kDecodeThreads;
        held[k] = i < len ? __ldg(hist + i) : -1;
    }
#pragma unroll
    for (int k = 0; k < kBiasEach; ++k) {
        const int i = tid + k * kDecodeThreads;
        id[k] = i < n_bias ? __ldg(ids + i) : -1;
    }
    uint4 m4[kQuads];
    const bool quads = mrow && (reinterpret_cast<uintptr_t>(mrow) & 15) == 0 && (g.n & 3) == 0;
    const int rounds = (g.n + 4 * kDecodeThreads - 1) / (4 * kDecodeThreads);
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
        const int j = (tid + k * kDecodeThreads) * 4;
        m4[k] = make_uint4(0u, 0u, 0u, 0u);
        if (j >= g.n) continue;
        if (quads) {
            m4[k] = __ldg(reinterpret_cast<const uint4*>(mrow + j));
        } else {
            m4[k].x = mrow ? __ldg(mrow + j) : 0xFFFFFFFFu;
            if (j + 1 < g.n) m4[k].y = mrow ? __ldg(mrow + j + 1) : 0xFFFFFFFFu;
            if (j + 2 < g.n) m4[k].z = mrow ? __ldg(mrow + j + 2) : 0xFFFFFFFFu;
            if (j + 3 < g.n) m4[k].w = mrow ? __ldg(mrow + j + 3) : 0xFFFFFFFFu;
        }
    }
#pragma unroll
    for (int k = 0; k < kQuads; ++k) {
        const int j = (tid + k * kDecodeThreads) * 4, left = a.V - 32 * (g.w0 + j);   // of the row
        if (j >= g.n) continue;
        if (left < 128) {   // the row's last words: no bits beyond it
            m4[k].x &= left < 32 ? (1u << left) - 1u : 0xFFFFFFFFu;
            m4[k].y &= left < 64 ? left < 32 ? 0u : (1u << (left - 32)) - 1u : 0xFFFFFFFFu;
            m4[k].z &= left < 96 ? left < 64 ? 0u : (1u << (left - 64)) - 1u : 0xFFFFFFFFu;
            m4[k].w &= left < 96 ? 0u : (1u << (left - 96)) - 1u;
        }
        reinterpret_cast<uint4*>(g.changed)[j / 4] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (tid == 0) g.mask[-1] = 0u;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kHeld; ++k) g.mark(held[k], a.V, report);
    for (int i = tid + kHeld * kDecodeThreads; i < len; i += kDecodeThreads) g.mark(__ldg(hist + i), a.V, report);
#pragma unroll
    for (int k = 0; k < kBiasEach; ++k) g.mark(id[k], a.V, report);
    __syncthreads();
    // allowed and changed, allowed and not; numbers: of each round's words, by threads, by warps
    g.total = 0;
    for (int k = 0; k < rounds; ++k) {
        const int j = (tid + k * kDecodeThreads) * 4;
        uint4 c = make_uint4(0u, 0u, 0u, 0u), m = k == 0 ? m4[0] : m4[kQuads - 1];
        if (j < g.n) {
            c = reinterpret_cast<const uint4*>(g.changed)[j / 4];
            c = make_uint4(c.x & m.x, c.y & m.y, c.z & m.z, c.w & m.w);
            reinterpret_cast<uint4*>(g.changed)[j / 4] = c;
            reinterpret_cast<uint4*>(g.mask)[j / 4] = make_uint4(m.x & ~c.x, m.y & ~c.y, m.z & ~c.z, m.w & ~c.w);
        }
        const int n0 = __popc(c.x), n1 = n0 + __popc(c.y), n2 = n1 + __popc(c.z), count = n2 + __popc(c.w);
        int upto = count;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += y;
        }
        if (lane == 31) s_sum[k][warp] = upto;
        __syncthreads();
        int at = upto - count + g.total;
#pragma unroll
        for (int w = 0; w < kDecodeWarps; ++w) {
            if (w < warp) at += s_sum[k][w];
            g.total += s_sum[k][w];
        }
        if (j < g.n)
            reinterpret_cast<uint2*>(g.before)[j / 4] =
                make_uint2((uint32_t)at | ((uint32_t)(at + n0) << 16), (uint32_t)(at + n1) | ((uint32_t)(at + n2) << 16));
    }
    if (tid == 0) g.mask[g.n] = 0u;
    __syncthreads();
    // the places, a word a thread: neighbouring words, full where their tokens are frequent ones, are different threads'
    for (int j = tid; j < g.n; j += kDecodeThreads) {
        uint32_t w = g.changed[j];
        if (w)
            for (int i = g.before[j]; w; w &= w - 1) g.place[i++] = 32u * j + __ffs((int)w) - 1;
    }
    for (int k = tid; k < g.total; k += kDecodeThreads) g.value[k] = n_bias ? 0xFFFFFFFFu : 0u;
    __syncthreads();
    if (g.total == 0) return;
    // of equal ids the first: the lowest index at each place
    int mine[kBiasEach];
#pragma unroll
    for (int k = 0; k < kBiasEach; ++k) mine[k] = -1;
    if (n_bias) {
#pragma unroll
        for (int k = 0; k < kBiasEach; ++k) {
            mine[k] = g.number(id[k]);
            if (mine[k] >= 0) atomicMin(g.value + mine[k], (uint32_t)(tid + k * kDecodeThreads));
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kBiasEach; ++k)
            if (mine[k] >= 0 && g.value[mine[k]] != (uint32_t)(tid + k * kDecodeThreads)) mine[k] = -1;
        __syncthreads();
        for (int k = tid; k < g.total; k += kDecodeThreads) g.value[k] = 0u;
        __syncthreads();
    }
    // times beyond the prompt; the highest bit: in the prompt
    const int prompt = a.p.prompt_lengths_dev ? __ldg(a.p.prompt_lengths_dev + r) : 0;
    const auto count_one = [&](int i, int32_t t) {
        const int k = g.number(t);
        if (k < 0) return;
        if (i < prompt) atomicOr(g.value + k, 0x80000000u);
        else atomicAdd(g.value + k, 1u);
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k) count_one(tid + k * kDecodeThreads, held[k]);
    for (int i = tid + kHeld * kDecodeThreads; i < len; i += kDecodeThreads) count_one(i, __ldg(hist + i));
    __syncthreads();
    const float rep = a.p.repetition_dev ? __ldg(a.p.repetition_dev + r) : 1.0f;
    const float pres = a.p.presence_dev ? __ldg(a.p.presence_dev + r) : 0.0f;
    const float freq = a.p.frequency_dev ? __ldg(a.p.frequency_dev + r) : 0.0f;
    for (int k = tid; k < g.total; k += kDecodeThreads) {
        const uint32_t n = g.value[k], beyond = n & 0x7FFFFFFFu;
        float x = logit_at<BF16>(lrow, 32 * g.w0 + g.place[k]);
        if (n) x = x > 0.0f ? __fdiv_rn(x, rep) : __fmul_rn(x, rep);
        if (beyond) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, __uint2float_rn(beyond))), pres);
        g.value[k] = __float_as_uint(x);
    }
    __syncthreads();
    if (n_bias) {
#pragma unroll
        for (int k = 0; k < kBiasEach; ++k)
            if (mine[k] >= 0)
                g.value[mine[k]] = __float_as_uint(__uint_as_float(g.value[mine[k]]) +
                                                   __ldg(a.p.bias_values_dev + (int64_t)r * n_bias + tid + k * kDecodeThreads));
        __syncthreads();
    }
}

template <bool BF16, int FOLD>
__global__ void __launch_bounds__(kDecodeThreads, 2) penalized_kernel(const __grid_constant__ Rows a) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ DecodeShared sh;
    __shared__ uint4 s_keep[BF16 && FOLD != kFoldSample ? kDecodeKeep : 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Layout l = layout(a.segment, a.places);
    Segment g;
    g.mask = reinterpret_cast<uint32_t*>(smem + l.mask);
    g.changed = reinterpret_cast<uint32_t*>(smem + l.changed);
    g.before = reinterpret_cast<uint16_t*>(smem + l.before);
    g.value = reinterpret_cast<uint32_t*>(smem + l.value);
    g.place = reinterpret_cast<uint32_t*>(smem + l.place);
    uint16_t* list = reinterpret_cast<uint16_t*>(smem + l.list) + warp * kDecodeList;
    const int r = blockIdx.x / a.slices, slice = blockIdx.x - r * a.slices;
    if (BF16 && FOLD != kFoldSample) fill_keep(s_keep, tid);
    pdl_wait();
    pdl_trigger();
    const int w0 = slice * a.slice_words, w1 = min(a.W, w0 + a.slice_words);
    uint32_t* report = slice == 0 ? a.err : nullptr;
    int len = a.p.lengths_dev ? __ldg(a.p.lengths_dev + r) : a.p.history_len;
    if (len < 0 || len > a.p.history_len) {
        if (report && tid == 0) atomicOr(report, DOMINO_DEVERR_BAD_TOKEN);
        len = len < 0 ? 0 : a.p.history_len;
    }
    Decoder<BF16, FOLD> d;
    d.init(a.logits, a.stride, r, a.V, a.logprobs != nullptr, a.sample, s_keep, lane);
    float cm = -INFINITY, cs = 0.0f;   // of the changed tokens: largest (or score), its token, sum of exp against it
    int ci = INT_MAX;
    for (int j = w0; j < w1; j += a.segment) {
        g.w0 = j;
        g.n = min(a.segment, w1 - j);
        if (j > w0) __syncthreads();   // the segment before has been read
        make_segment<BF16>(g, a, r, len, d.lrow, j == w0 ? report : nullptr, tid);
        d.slice(g.mask, 32 * j, min(32 * g.n, a.V - 32 * j), list, warp);
        for (int k = tid; k < g.total; k += kDecodeThreads) {
            float x = __uint_as_float(g.value[k]);
            const int t = 32 * j + g.place[k];
            if constexpr (FOLD == kFoldSample) {
                int blk = -1;
                uint4 rnd;
                x = __fadd_rn(__fmul_rn(x, a.sample.inv_t), gumbel(a.sample, r, t, blk, rnd));
            }
            if (x != -INFINITY) acc_merge(cm, ci, cs, x, t, FOLD == kFoldLse ? 1.0f : 0.0f);
        }
    }
    d.finish();
    float m = d.m, s = d.s;
    int idx = d.idx;
    acc_merge(m, idx, s, cm, ci, cs);
    decode_combine(sh, m, idx, s, a.slices, lane, warp);
    const float lse = FOLD == kFoldLse ? log_sum_exp(m, s) : 0.0f;
    if (tid == 0 && slice == 0) {
        a.argmax[r] = m == -INFINITY ? -1 : idx;
        if (FOLD == kFoldLse && a.lse) a.lse[r] = lse;
    }
    if constexpr (FOLD == kFoldLse) {
        if (a.logprobs) {
            float* orow = a.logprobs + (int64_t)r * a.V;
            for (int j = w0; j < w1; j += a.segment) {
                if (w1 - w0 > a.segment) {   // more than one: made again
                    g.w0 = j;
                    g.n = min(a.segment, w1 - j);
                    __syncthreads();
                    make_segment<BF16>(g, a, r, len, d.lrow, nullptr, tid);
                }
                write_logprobs<BF16>(d.lrow, a.V, g.mask, 32 * j, min(32 * g.n, a.V - 32 * j), lse, orow, tid);
                __syncthreads();   // the changed tokens' over what stands there
                for (int k = tid; k < g.total; k += kDecodeThreads) {
                    const float x = __uint_as_float(g.value[k]);
                    orow[32 * j + g.place[k]] = x == -INFINITY ? x : x - lse;
                }
            }
        }
    }
    if (a.slices > 1) cluster_wait();
}

template <bool BF16, int FOLD>
cudaError_t launch_t(const Rows& a, int batch, cudaStream_t st) {
    constexpr int kDevices = 64;
    static std::atomic<bool> ready[kDevices];   // one array per kernel
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= kDevices || !ready[dev].load()) {
        e = cudaFuncSetAttribute(penalized_kernel<BF16, FOLD>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPenalizedSmem);
        if (e != cudaSuccess) return e;
        if (dev < kDevices) ready[dev].store(true);
    }
    return launch_cluster(penalized_kernel<BF16, FOLD>, dim3((unsigned)batch * (unsigned)a.slices), dim3(kDecodeThreads), a.slices,
                          (size_t)layout(a.segment, a.places).end, st, a);
}
template <bool BF16>
cudaError_t launch_fold(const Rows& a, int batch, bool sample, cudaStream_t st) {
    if (sample) return launch_t<BF16, kFoldSample>(a, batch, st);
    return a.lse || a.logprobs ? launch_t<BF16, kFoldLse>(a, batch, st) : launch_t<BF16, kFoldMax>(a, batch, st);
}

}  // namespace

cudaError_t launch_penalized(const PenalizedArgs& p, const LaunchEnv& env, cudaStream_t st) {
    Rows a{};
    a.logits = p.logits;
    a.stride = p.stride;
    a.mask = p.mask;
    a.p = p.p;
    a.V = p.n_tokens;
    a.W = (p.n_tokens + 31) / 32;
    a.argmax = p.argmax;
    a.lse = p.lse;
    a.logprobs = p.logprobs;
    a.sample = p.sample ? *p.sample : SampleArgs{0u, 0u, 0u, 0u, 1.0f};
    a.err = p.err;
    // CTAs per row as the decode without penalties takes them
    int s = 1;
    while (s < 8 && ((int64_t)p.batch * s * 2 <= env.num_sms ? a.W > 256 * s : (int64_t)p.batch * s <= env.num_sms && a.W > 2048 * s))
        s *= 2;
    a.slices = s;
    a.slice_words = ((a.W + s - 1) / s + 3) / 4 * 4;
    // fewer words at a time where a long history may change more tokens than fit
    const int64_t most = (int64_t)a.p.history_len + a.p.n_bias;
    for (a.segment = std::min(a.slice_words, kSegmentWords);; a.segment = a.segment * 3 / 16 * 4) {
        a.places = (int32_t)(std::min<int64_t>(most, 32 * (int64_t)a.segment) + 7) / 8 * 8;
        if (layout(a.segment, a.places).end <= kPenalizedSmem) break;
    }
    const int segments = (a.slice_words + a.segment - 1) / a.segment;
    a.segment = ((a.slice_words + segments - 1) / segments + 3) / 4 * 4;   // of about the same length
    return p.dtype == DOMINO_DTYPE_BF16 ? launch_fold<true>(a, p.batch, p.sample != nullptr, st)
                                        : launch_fold<false>(a, p.batch, p.sample != nullptr, st);
}

}  // namespace domino
