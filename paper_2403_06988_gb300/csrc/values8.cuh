// values8.cuh -- eight values of a row a lane, bf16 or fp32 at any alignment, and
// e4m3 codes with a scale for each 128 values.
//
//   a = max |v| over the block, at least 2^-100;  scale = a / 448;  code = e4m3(v (448 / a))
//
// The scale is a times the rounded 1 / 448 (two roundings: a second division would be a tenth of a norm's instructions).
// 448 is the largest e4m3 value: the block's largest value takes it, and nothing
// overflows.  Sixteen lanes of eight values make a block of a row.
#pragma once
#include "bf16_rows.cuh"
#include "walk_common.cuh"

namespace domino {
namespace {

constexpr int kBlock8 = 128;              // values that share a scale, along a row
constexpr int kBlockLanes = kBlock8 / kN;
constexpr float kMost8 = 448.0f, kLeast8 = 0x1p-100f;

// Two values an instruction, each rounded once as one by one.
__device__ __forceinline__ unsigned long long pair_of(float a, float b) {
    unsigned long long x;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b));
    return x;
}
__device__ __forceinline__ void from_pair(float& a, float& b, unsigned long long x) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
}
__device__ __forceinline__ void add8(float (&f)[kN], const float (&g)[kN]) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
        unsigned long long r;
        asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_of(f[e], f[e + 1])), "l"(pair_of(g[e], g[e + 1])));
        from_pair(f[e], f[e + 1], r);
    }
}
__device__ __forceinline__ void mul8(float (&f)[kN], const float (&g)[kN]) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
        unsigned long long r;
        asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_of(f[e], f[e + 1])), "l"(pair_of(g[e], g[e + 1])));
        from_pair(f[e], f[e + 1], r);
    }
}
__device__ __forceinline__ void mul8(float (&f)[kN], float by) {
    const float g[kN] = {by, by, by, by, by, by, by, by};
    mul8(f, g);
}
// a b + c
__device__ __forceinline__ void fma8(float (&r)[kN], const float (&a)[kN], const float (&b)[kN], const float (&c)[kN]) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
        unsigned long long x;
        asm("fma.rn.f32x2 %0, %1, %2, %3;"
            : "=l"(x)
            : "l"(pair_of(a[e], a[e + 1])), "l"(pair_of(b[e], b[e + 1])), "l"(pair_of(c[e], c[e + 1])));
        from_pair(r[e], r[e + 1], x);
    }
}
__device__ __forceinline__ void fma8(float (&r)[kN], const float (&a)[kN], float b, const float (&c)[kN]) {
    const float g[kN] = {b, b, b, b, b, b, b, b};
    fma8(r, a, g, c);
}
// The products, added to the sums of the even and the odd ones.
__device__ __forceinline__ void dot8(float2& s, const float (&f)[kN], const float (&g)[kN]) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
        unsigned long long r;
        asm("fma.rn.f32x2 %0, %1, %2, %3;"
            : "=l"(r)
            : "l"(pair_of(f[e], f[e + 1])), "l"(pair_of(g[e], g[e + 1])), "l"(pair_of(s.x, s.y)));
        from_pair(s.x, s.y, r);
    }
}
// The squares, added to the sums of the even and the odd ones.
__device__ __forceinline__ void square8(float2& s, const float (&f)[kN]) {
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
        unsigned long long r;
        const unsigned long long x = pair_of(f[e], f[e + 1]);
        asm("fma.rn.f32x2 %0, %1, %1, %2;" : "=l"(r) : "l"(x), "l"(pair_of(s.x, s.y)));
        from_pair(s.x, s.y, r);
    }
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Values c, .. c + 7 of a row of dim; zeros beyond its end.  ALIGNED: the row begins on a 16-byte boundary.  load() reads
// and uses nothing of what it reads, so that a thread's loads are on their way together, and get() converts (128256 x 4096
// bf16 in codes: 259 us, converted as they come 689).  After keep() a get() converts again: what is kept meanwhile are the
// bits, not fp32 values.  Rows are read in the 16-byte blocks that hold their values.  Neither __ldg nor another assumption
// that the row is not written by this kernel: outputs may take inputs' places.
template <bool BF16, bool ALIGNED>
struct Vec8;
template <>
struct Vec8<true, true> {
    uint4 u;
    int32_t left;
    __device__ __forceinline__ void keep() { asm volatile("" : "+r"(u.x), "+r"(u.y), "+r"(u.z), "+r"(u.w)); }
    __device__ __forceinline__ void load(const void* row, int32_t c, int32_t dim) {
        left = dim - c;
        u = make_uint4(0u, 0u, 0u, 0u);
        if (left > 0) u = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(row) + c);
    }
    __device__ __forceinline__ void get(float (&f)[kN]) const {
        f[0] = bf16_lo(u.x), f[1] = bf16_hi(u.x), f[2] = bf16_lo(u.y), f[3] = bf16_hi(u.y);
        f[4] = bf16_lo(u.z), f[5] = bf16_hi(u.z), f[6] = bf16_lo(u.w), f[7] = bf16_hi(u.w);
        if (left > 0 && left < kN) {
#pragma unroll
            for (int e = 0; e < kN; ++e) f[e] = e < left ? f[e] : 0.0f;
        }
    }
};
template <>
struct Vec8<true, false> {
    Eight x;
    __device__ __forceinline__ void keep() {   // in one block from now on
        x.u = eight_from(x.u, x.v, x.off);
        x.v = make_uint4(0u, 0u, 0u, 0u);
        x.off = 0u;
        asm volatile("" : "+r"(x.u.x), "+r"(x.u.y), "+r"(x.u.z), "+r"(x.u.w));
    }
    __device__ __forceinline__ void load(const void* row, int32_t c, int32_t dim) {
        x.zero();
        if (dim > c) x.load(static_cast<const __nv_bfloat16*>(row) + c, dim - c);
    }
    __device__ __forceinline__ void get(float (&f)[kN]) const {
        const uint4 u = eight_from(x.u, x.v, x.off);
        f[0] = bf16_lo(u.x), f[1] = bf16_hi(u.x), f[2] = bf16_lo(u.y), f[3] = bf16_hi(u.y);
        f[4] = bf16_lo(u.z), f[5] = bf16_hi(u.z), f[6] = bf16_lo(u.w), f[7] = bf16_hi(u.w);
        if (x.n < kN) {   // the row's end
#pragma unroll
            for (int e = 0; e < kN; ++e) f[e] = (uint32_t)e < x.n ? f[e] : 0.0f;
        }
    }
};
template <>
struct Vec8<false, true> {
    float4 u, v;
    int32_t left;
    __device__ __forceinline__ void keep() {}
    __device__ __forceinline__ void load(const void* row, int32_t c, int32_t dim) {
        left = dim - c;
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(row) + c);
        u = v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (left > 0) u = p[0];
        if (left > 4) v = p[1];
    }
    __device__ __forceinline__ void get(float (&f)[kN]) const {
        f[0] = u.x, f[1] = u.y, f[2] = u.z, f[3] = u.w, f[4] = v.x, f[5] = v.y, f[6] = v.z, f[7] = v.w;
        if (left > 0 && left < kN) {
#pragma unroll
            for (int e = 0; e < kN; ++e) f[e] = e < left ? f[e] : 0.0f;
        }
    }
};
template <>
struct Vec8<false, false> {   // three blocks hold them (norm of 8000 x 333 10.8 us, read and written one by one 15.1)
    float4 a, b, c4;
    uint32_t off, n;
    __device__ __forceinline__ void keep() {   // in two blocks from now on
        float f[kN];
        get(f);
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
        c4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        off = 0u;
        n = kN;
    }
    __device__ __forceinline__ void load(const void* row, int32_t c, int32_t dim) {
        a = b = c4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        off = 0u;
        n = kN;
        if (c >= dim) return;
        const uintptr_t at = reinterpret_cast<uintptr_t>(static_cast<const float*>(row) + c);
        const float4* block = reinterpret_cast<const float4*>(at & ~(uintptr_t)15);
        off = (uint32_t)(at & 15) / 4;
        n = (uint32_t)min(dim - c, kN);
        a = block[0];
        if (off + n > 4) b = block[1];
        if (off + n > 8) c4 = block[2];
    }
    __device__ __forceinline__ void get(float (&f)[kN]) const {
        float w[12] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, c4.x, c4.y, c4.z, c4.w};
#pragma unroll
        for (int e = 0; e < kN + 1; ++e) w[e] = off & 2u ? w[e + 2] : w[e];
#pragma unroll
        for (int e = 0; e < kN; ++e) f[e] = off & 1u ? w[e + 1] : w[e];
        if (n < kN) {
#pragma unroll
            for (int e = 0; e < kN; ++e) f[e] = (uint32_t)e < n ? f[e] : 0.0f;
        }
    }
};

// Eight values of a weight.  What rows off the boundaries are multiplied with is on one all the same; where it is not, value
// by value.
template <bool BF16, bool ALIGNED>
struct VecOf : Vec8<BF16, true> {
    __device__ __forceinline__ void load(const void* p, int32_t c, int32_t dim) {
        const bool on = ALIGNED || (reinterpret_cast<uintptr_t>(p) & 15) == 0;
        Vec8<BF16, true>::load(p, c, on ? dim : 0);
        if (on) return;
        this->left = dim - c;
        if constexpr (BF16) {
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (e < this->left) w[e / 2] |= (uint32_t) static_cast<const unsigned short*>(p)[c + e] << (16 * (e & 1));
            this->u = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            float f[kN];
#pragma unroll
            for (int e = 0; e < kN; ++e) f[e] = e < this->left ? static_cast<const float*>(p)[c + e] : 0.0f;
            this->u = make_float4(f[0], f[1], f[2], f[3]);
            this->v = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
};
// A warp's 256 consecutive fp32 values (eight a lane, `left` of this lane's to the row's end) to a row at any alignment: in
// 16-byte blocks, each lane's first with the last values of the lane before it, and one by one at the two ends.
__device__ __forceinline__ void store_any4(float* p, const float (&f)[kN], int32_t left, int lane) {
    const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15) / 4;   // the same in every lane
    float w[kN + 3];   // from off values before the lane's first
    const float p5 = __shfl_up_sync(0xffffffffu, f[5], 1), p6 = __shfl_up_sync(0xffffffffu, f[6], 1), p7 = __shfl_up_sync(0xffffffffu, f[7], 1);
    const float all[kN + 3] = {p5, p6, p7, f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]};
    // w[k] = all[k + 3 - off]
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        const float x0 = all[k + 3], x1 = all[k + 2], x2 = all[k + 1], x3 = all[k];
        w[k] = off & 2 ? (off & 1 ? x3 : x2) : (off & 1 ? x1 : x0);
    }
    float4* block = reinterpret_cast<float4*>(p - off);
    const bool first = (off == 0 || lane > 0) && left >= 4 - off, second = left >= 8 - off;
    const bool next = off > 0 && lane < 31 && left - kN >= 4 - off;   // the next lane writes this one's last values
    if (first) block[0] = make_float4(w[0], w[1], w[2], w[3]);
    if (second) block[1] = make_float4(w[4], w[5], w[6], w[7]);
    if (!first || !second || (off > 0 && !next)) {
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const bool done = e < 4 - off ? first : e < 8 - off ? second : next;
            if (e < left && !done) p[e] = f[e];
        }
    }
}

// The same values to a row.  The whole warp calls it, its lanes with consecutive c's.  far: past the L2.
template <bool BF16, bool ALIGNED>
__device__ __forceinline__ void store8(void* row, int32_t c, int32_t dim, const float (&f)[kN], bool far, int lane) {
    const int32_t left = dim - c;
    if constexpr (BF16) {
        const uint32_t w[4] = {pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])};
        __nv_bfloat16* p = static_cast<__nv_bfloat16*>(row) + c;
        if constexpr (ALIGNED) {
            if (left >= kN) {
                if (far) __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
                else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
                for (int e = 0; e < kN; ++e)
                    if (e < left) reinterpret_cast<unsigned short*>(p)[e] = (unsigned short)(w[e / 2] >> (16 * (e & 1)));
            }
        } else {
            store_any(p, w, left, lane);
        }
    } else {
        float* p = static_cast<float*>(row) + c;
        if (ALIGNED && left >= kN) {
            const float4 u = make_float4(f[0], f[1], f[2], f[3]), v = make_float4(f[4], f[5], f[6], f[7]);
            if (far) {
                __stcs(reinterpret_cast<float4*>(p), u);
                __stcs(reinterpret_cast<float4*>(p) + 1, v);
            } else {
                reinterpret_cast<float4*>(p)[0] = u;
                reinterpret_cast<float4*>(p)[1] = v;
            }
        } else if constexpr (ALIGNED) {
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (e < left) p[e] = f[e];
        } else {
            store_any4(p, f, left, lane);
        }
    }
}

__device__ __forceinline__ float scale_of(float top) { return top * (1.0f / kMost8); }

__device__ __forceinline__ float largest(const float (&f)[kN]) {
    float a = 0.0f;
#pragma unroll
    for (int e = 0; e < kN; ++e) a = fmaxf(a, fabsf(f[e]));
    return a;
}
// The largest of a block's lanes.
__device__ __forceinline__ float block_largest(float a) {
#pragma unroll
    for (int off = kBlockLanes / 2; off > 0; off >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, off));
    return a;
}

__device__ __forceinline__ uint32_t two_codes(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// Eight codes at column c of a row of codes that begins on a 16-byte boundary, by = 448 / the block's largest; nothing at
// or beyond dim is written.
__device__ __forceinline__ void store_codes(uint8_t* row, int32_t c, int32_t dim, const float (&f)[kN], float by, bool far) {
    float v[kN] = {f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]};
    mul8(v, by);
    const uint32_t lo = two_codes(v[0], v[1]) | (two_codes(v[2], v[3]) << 16);
    const uint32_t hi = two_codes(v[4], v[5]) | (two_codes(v[6], v[7]) << 16);
    uint8_t* p = row + c;
    if (c + kN <= dim) {
        if (far) __stcs(reinterpret_cast<uint2*>(p), make_uint2(lo, hi));
        else *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e)
            if (c + e < dim) p[e] = (uint8_t)((e < 4 ? lo : hi) >> (8 * (e & 3)));
    }
}

}  // namespace
}  // namespace domino
