// tcgen05.cuh -- device helpers of the tensor-core products (loss.cu): memory
// barriers with bounded waits, TMA loads of operand tiles, the shared-memory
// and instruction descriptors of tcgen05.mma on bf16 operands, and loads of
// the accumulators from tensor memory.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace domino {
namespace {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// The address in the cluster of what lies at `addr` in CTA `rank`.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// Orders nothing but the arriving thread's reads of tensor memory: no other memory of the CTA is handed over by it (a
// release at the cluster's scope waits for the thread's stores: 2.7 of 15 cycles an instruction).
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar_in_cluster) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];\n" ::"r"(bar_in_cluster) : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ uint64_t timer_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;\n" : "=l"(t));
    return t;
}

// Waits for the phase `parity` of `bar` to end.  A wait ends after kWaitNs at
// the latest, or once another role of the CTA has given up (*failed): it then
// returns false with *failed set, and its caller leaves.  The clock is read once
// in kWaitTries tries: reading it takes longer than most waits.
constexpr uint64_t kWaitNs = 4000000000ull;
constexpr uint32_t kWaitTries = 256;
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* failed) {
    uint64_t end = 0;
    for (uint32_t i = 1; !bar_try(bar, parity); ++i) {
        if (i % kWaitTries) continue;
        if (*failed) return false;
        const uint64_t now = timer_ns();
        if (end == 0) end = now + kWaitNs;
        if (now > end) {
            *failed = 1u;
            return false;
        }
    }
    return true;
}

// One lane of a converged warp.  Loads, products and commits are issued inside of `if (elect_lane())`, by a warp that
// runs its loops whole: their addresses and descriptors then stay in uniform registers.  (A loop of one lane's own took
// 540 cycles to issue a k block's two loads and 650 its four products and commit.)
__device__ __forceinline__ bool elect_lane() {
    uint32_t p;
    asm volatile(
        "{\n.reg .pred q;\n"
        "elect.sync _|q, 0xffffffff;\n"
        "selp.u32 %0, 1, 0, q;\n}\n"
        : "=r"(p));
    return p != 0;
}
// bar_wait by a whole warp, which goes on or leaves as one.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* failed) {
    return __all_sync(0xffffffffu, bar_wait(bar, parity, failed));
}

// A box of the tensor that `map` describes, its corner at (x, y), into shared
// memory at `dst`; `bar` counts its bytes.  x is a multiple of 16 bytes.
// PAIR: `bar` may be the other CTA's of a pair (its address in the cluster).
template <bool PAIR>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
            "[%4];\n" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(map) : "memory");
}

// A tile in shared memory at `src` to the box of the tensor with its corner at (x, y), or added to what stands there;
// what lies outside of the tensor is left out.  x is a multiple of 16 bytes, both are inside of the tensor.
__device__ __forceinline__ void tma_store(const CUtensorMap* map, int32_t x, int32_t y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];\n" ::"l"(map), "r"(x), "r"(y),
                 "r"(src)
                 : "memory");
}
__device__ __forceinline__ void tma_add(const CUtensorMap* map, int32_t x, int32_t y, uint32_t src) {
    asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];\n" ::"l"(map),
                 "r"(x), "r"(y), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void tma_commit() { asm volatile("cp.async.bulk.commit_group;\n" ::: "memory"); }
// All but the last PENDING groups of this thread have read their shared memory.
template <int PENDING>
__device__ __forceinline__ void tma_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(PENDING) : "memory");
}
__device__ __forceinline__ void tma_wait_all() { asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory"); }
// What this thread wrote to shared memory is seen by the copies issued after a barrier with it.
__device__ __forceinline__ void tma_fence() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }

// Shared-memory descriptor of an operand tile in the 128-byte swizzle: start
// address, leading and stride byte offsets (16-byte units), descriptor version
// 1 (bits 46, 47), swizzle mode 2 (bits 61 to 63).
//   K-major (rows of 64 k, 128 bytes each): eight rows take 1024 bytes, the
//     stride offset; the leading offset is not used.
//   MN-major (rows of 64 m or n for each k): eight k take 1024 bytes, the
//     stride offset; the next 64 m or n lie a leading offset further.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t leading) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(leading >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}

// Instruction descriptor: bf16 operands, fp32 accumulator, M x N.
__host__ __device__ constexpr uint32_t mma_desc(int m, int n, bool a_mn, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// PAIR: a product of two CTAs, issued by the first: each holds half of A's rows
// and of B's, at the same addresses, and gets its rows of the accumulator.
template <bool PAIR>
__device__ __forceinline__ void mma_bf16(uint32_t acc, uint64_t a, uint64_t b, uint32_t desc, bool add) {
    if constexpr (PAIR)
        asm volatile(
            "{\n.reg .pred p;\n"
            "setp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(acc),
            "l"(a), "l"(b), "r"(desc), "r"(add ? 1u : 0u)
            : "memory");
    else
        asm volatile(
            "{\n.reg .pred p;\n"
            "setp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(acc),
            "l"(a), "l"(b), "r"(desc), "r"(add ? 1u : 0u)
            : "memory");
}
// `bar` (PAIR: of both CTAs) is arrived at once the products issued before have ended.
template <bool PAIR>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (PAIR)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(bar) : "memory");
}

// A warp of the CTA (PAIR: of both CTAs) calls these.
template <bool PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t out, uint32_t columns) {
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(out), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(out), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
    if constexpr (PAIR)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(addr), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(addr), "r"(columns) : "memory");
}
__device__ __forceinline__ void tcgen_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tcgen_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }

// 32 columns from `addr` on of the warp's 32 lanes: lane l gets row l's.
__device__ __forceinline__ void tmem_load32(float (&v)[32], uint32_t addr) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// The same of 16 columns, added to v.
__device__ __forceinline__ void tmem_add16(float* v, uint32_t addr) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] += __uint_as_float(r[i]);
}

}  // namespace
}  // namespace domino
