// Rounding of quotients to whole numbers of 8 bits, as the bounds of pages and the queries of their scores are stored.
#pragma once

#include "common.cuh"

namespace sv {

// The whole number nearest to x / scale (the quotient rounded to float32 first, halves to even), in [-127, 127]; 0 where
// scale is 0.
__device__ __forceinline__ int whole8(float x, float scale)
{
    return scale > 0.f ? min(max(__float2int_rn(__fdiv_rn(x, scale)), -127), 127) : 0;
}

// Eight of them as bytes, without dividing.  With inv = 1 / scale rounded to nearest, q = x inv rounded is within one unit in
// the last place of x / scale, and q + (x - q scale) inv, with the remainder exact in one fused operation, is x / scale
// rounded to nearest (Markstein's theorem on division by a correctly rounded reciprocal; nothing underflows where |q| > 1/4
// and scale > 1e-25).  Quotients of bf16 numbers are near or on halves too often (0.3 % of them) for an approximate
// quotient with a check: the divisions it fell back to were four fifths of the time of the kernel that scores pages.
// inv = 0 (whole8_inverse of a scale that is too small): real divisions.
__device__ __forceinline__ float whole8_inverse(float scale) { return scale > 1e-25f ? __frcp_rn(scale) : 0.f; }

__device__ __forceinline__ uint2 whole8x8(const float (&x)[8], float scale, float inv)
{
    constexpr float MAGIC = 12582912.f;                // 1.5 * 2^23: the sum rounds to whole numbers, its low bits hold them
    uint32_t t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float q = __fmul_rn(x[e], inv);
        t[e] = __float_as_uint(__fadd_rn(fmaf(fmaf(-q, scale, x[e]), inv, q), MAGIC));
    }
    if (inv == 0.f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = (uint32_t)whole8(x[e], scale);
    }
    uint2 w;
    w.x = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
    w.y = __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410);
    return w;
}

// the eight bf16 of 16 bytes
__device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = __uint_as_float(w[j] << 16);
        f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}

// 0xff for the negative bytes of w, 0 for the others
__device__ __forceinline__ uint32_t negative_bytes(uint32_t w)
{
    uint32_t m;
    asm("prmt.b32 %0, %1, 0, 0xba98;" : "=r"(m) : "r"(w));
    return m;
}

}  // namespace sv
