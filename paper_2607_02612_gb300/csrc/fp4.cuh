// Numbers of the cache in 4 bits: e2m1 codes (a sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6), eight to
// a word, and an e4m3 scale for 16 of them.  A product of the two has 6 significant bits and lies in 2^-10 .. 2688, so float16
// holds it exactly.
#pragma once

#include <cuda_fp16.h>

#include "ln.cuh"

namespace fz {

// Bytes 0 .. 3 of w, each two codes, as two float16 each (the lower four bits in the lower half).
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t (&r)[4]) {
    asm("{ .reg .b8 b0, b1, b2, b3;\n"
        "mov.b32 {b0, b1, b2, b3}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n"
        "cvt.rn.f16x2.e2m1x2 %3, b3; }"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
        : "r"(w));
}
// The two scales in the lower bytes of w as float16.
__device__ __forceinline__ uint32_t scales_to_half(uint32_t w) {
    uint32_t r;
    asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, lo; }" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float half_low(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)w)); }
__device__ __forceinline__ float half_high(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }

// The largest magnitude of three numbers; NaN if one is.
__device__ __forceinline__ float max_magnitude(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
    return r;
}
// S numbers of a group of 16, the even ones in e and the odd ones in o, the rest in the 16 / S lanes of `mask` around this one: their
// codes, four bits each, and the group's scale's byte.
//
// A code is the e2m1 number nearest to x / scale, ties to the even code, which is what the conversion makes of the quotient if
// the division's rounding neither leaves a tie nor makes one.  A scale has 4 significant bits and a tie lies at one of 3, so
// scale * tie is exact, and where x is not equal to it the quotient is further from the tie than its own rounding: correctly
// rounded it serves.  It comes of y = -x / scale but for a few roundings and one correction by the exact remainder x + y scale
// (of the negative quotient, so that -0 stays -0: the codes' signs are turned at the end).
template <int S> __device__ __forceinline__ unsigned long long quantise(const float2 (&e)[S / 4], const float2 (&o)[S / 4], unsigned mask, uint32_t &scale) {
    float top = max_magnitude(e[0].x, e[0].y, o[0].x);
#pragma unroll
    for (int i = 1; i < S / 4; ++i) {
        top = max_magnitude(top, o[i - 1].y, e[i].x);
        top = max_magnitude(top, e[i].y, o[i].x);
    }
    top = max_magnitude(top, o[S / 4 - 1].y, o[S / 4 - 1].y);
#pragma unroll
    for (int d = 1; d < 16 / S; d <<= 1) {
        const float other = __shfl_xor_sync(mask, top, d);
        top = max_magnitude(top, other, other);
    }
    const float want = top * (1.0f / 6.0f);
    uint16_t s;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(s) : "f"(0.0f), "f"(want));
    const float z = half_low(scales_to_half(s));
    const bool fine = top < INFINITY, some = fine && s != 0;
    scale = fine ? (uint32_t)s : 0x7Fu;
    const float inv = some ? -__frcp_rn(z) : 0.0f;
    const float2 zz = make_float2(z, z), ii = make_float2(inv, inv);
    uint32_t codes[S > 8 ? 2 : 1] = {0u};
#pragma unroll
    for (int i = 0; i < S / 4; ++i) {
        float2 ye = mul2(e[i], ii), yo = mul2(o[i], ii);
        ye = fma2(fma2(ye, zz, e[i]), ii, ye);
        yo = fma2(fma2(yo, zz, o[i]), ii, yo);
        uint16_t w;
        asm("{ .reg .b8 b0, b1;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
            "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
            "mov.b16 %0, {b0, b1}; }"
            : "=h"(w)
            : "f"(ye.x), "f"(yo.x), "f"(ye.y), "f"(yo.y));
        codes[i / 2] |= (uint32_t)w << (i % 2 * 16);
    }
    const uint32_t flip = some ? 0xFFFFFFFFu : 0u;
    const uint32_t low = (codes[0] ^ 0x88888888u) & flip;
    if constexpr (S > 8) return low | (unsigned long long)((codes[1] ^ 0x88888888u) & flip) << 32;
    else return low;
}

}  // namespace fz
