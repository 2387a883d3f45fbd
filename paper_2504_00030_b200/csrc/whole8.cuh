// Rounding of quotients to whole numbers of 8 bits, as the bounds of pages and the queries of their scores are stored.
#pragma once

#include "common.cuh"
#include "f32x2.cuh"

namespace sv {

// Of x / scale: the quotient rounded to float32, then to the nearest whole number (halves to even), in [-127, 127]; 0 where scale
// is 0 or no finite number.
//
// Eight of them as bytes, without dividing.  With inv = 1 / scale rounded to nearest, q = x inv rounded is within one unit in
// the last place of x / scale, and q + (x - q scale) inv, with the remainder exact in one fused operation, is x / scale
// rounded to nearest (Markstein's theorem on division by a correctly rounded reciprocal; nothing underflows where |q| > 1/4
// and scale > 1e-25; below, x and scale are taken 2^96 times as large, which is exact).  Quotients of bf16 numbers are near or
// on halves too often (0.3 % of them) for an approximate quotient with a check: the divisions it fell back to were four fifths
// of the time of the kernel that scores pages.
struct Whole8 {
    float scale, inv, up;
    __device__ __forceinline__ explicit Whole8(float s)
    {
        up = s <= 1e-25f ? 7.9228162514264338e28f : 1.f;       // 2^96
        scale = s * up;
        inv = scale > 0.f && scale <= 3.402823466e38f ? __frcp_rn(scale) : 0.f;
    }
};

__device__ __forceinline__ uint2 whole8x8(const float (&x)[8], const Whole8 &by)
{
    constexpr float MAGIC = 12582912.f;                // 1.5 * 2^23: the sum rounds to whole numbers, its low bits hold them
    const uint64_t inv = pair2(by.inv, by.inv), neg = pair2(-by.scale, -by.scale), magic = pair2(MAGIC, MAGIC);
    uint32_t t[8];
    uint64_t v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pair2(x[2 * e], x[2 * e + 1]);
    if (by.up != 1.f) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = mul2(v[e], pair2(by.up, by.up));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint64_t q = mul2(v[e], inv);
        float a, b;
        split2(add2(fma2(fma2(q, neg, v[e]), inv, q), magic), a, b);
        t[2 * e] = __float_as_uint(a);
        t[2 * e + 1] = __float_as_uint(b);
    }
    uint2 w;
    w.x = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
    w.y = __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410);
    return by.inv != 0.f ? w : make_uint2(0, 0);
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
