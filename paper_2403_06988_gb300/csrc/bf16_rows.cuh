// bf16_rows.cuh -- rows of bf16 at any alignment, eight values (16 bytes) a lane:
// reads of the 16-byte blocks that hold them, writes of whole blocks where they
// lie in the row.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace domino {
namespace {

constexpr int kN = 8;   // values of a lane

// Values off, off + 1, .. off + 7 of the sixteen in two consecutive blocks.
__device__ __forceinline__ uint4 eight_from(const uint4& a, const uint4& b, uint32_t off) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = off & 8 ? w[i + 4] : w[i];
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = off & 4 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = off & 2 ? w[i + 1] : w[i];
    const uint32_t shift = off & 1 ? 16 : 0;
    return make_uint4(__funnelshift_r(w[0], w[1], shift), __funnelshift_r(w[1], w[2], shift),
                      __funnelshift_r(w[2], w[3], shift), __funnelshift_r(w[3], w[4], shift));
}

// Up to eight values from p on, `left` to the row's end (at least one): the blocks
// that hold them, as they lie in memory, and the values (zeros beyond the end).
struct Eight {
    uint4 u, v;
    uint32_t off, n;
    __device__ __forceinline__ void zero() {
        u = v = make_uint4(0, 0, 0, 0);
        off = 0;
        n = kN;
    }
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int32_t left) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        const uint4* block = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
        off = (uint32_t)(at & 15) / 2;
        n = (uint32_t)(left < kN ? left : kN);
        u = *block;
        v = make_uint4(0, 0, 0, 0);
        if (off + n > kN) v = block[1];
    }
    __device__ __forceinline__ void get(float (&f)[kN]) const {
        const uint4 x = eight_from(u, v, off);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
#pragma unroll
        for (int i = 0; i < kN; ++i) f[i] = (uint32_t)i < n ? f[i] : 0.0f;
    }
};

// A warp's 256 consecutive values (eight a lane, `left` of lane 0's to the row's end) to a row of bf16 at any
// alignment: in the 16-byte blocks that lie in them, each lane's from its own values and the lane's before it, and one
// by one at the two ends.
__device__ __forceinline__ void store_any(__nv_bfloat16* to, const uint32_t (&w)[4], int32_t left, int lane) {
    // to, left: this lane's
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(to) & 15) / 2;
    uint4 before;
    before.x = __shfl_up_sync(0xffffffffu, w[0], 1);
    before.y = __shfl_up_sync(0xffffffffu, w[1], 1);
    before.z = __shfl_up_sync(0xffffffffu, w[2], 1);
    before.w = __shfl_up_sync(0xffffffffu, w[3], 1);
    const uint4 block = eight_from(before, make_uint4(w[0], w[1], w[2], w[3]), 8 - off);   // at `to` rounded down
    unsigned short* p = reinterpret_cast<unsigned short*>(to);
    const int32_t n = left < kN ? (left < 0 ? 0 : left) : kN;             // this lane's values
    const bool whole = (off == 0 || lane > 0) && left >= (int32_t)(kN - off);   // the block ends in the row
    if (whole) *reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(to) & ~(uintptr_t)15) = block;
    // beside the blocks: lane 0's first, what the next block would hold of the last lane's or of the row's last values
    const bool next_whole = lane < 31 && left - kN >= (int32_t)(kN - off) && off > 0;
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        const bool in_mine = e < (int)(kN - off);   // else in the next lane's block
        const bool one = in_mine ? !whole : !next_whole;
        if (e < n && one) p[e] = (unsigned short)(w[e / 2] >> (16 * (e & 1)));
    }
}

}  // namespace
}  // namespace domino
