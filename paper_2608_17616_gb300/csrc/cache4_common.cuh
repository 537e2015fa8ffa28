// Rows in 4 bits (mone_cache4): groups of 16 values, 2^exp x scale x code, the scale e4m3, the code e2m1.  A product of the two has at
// most 4 + 2 bits and lies in 2^-10 .. 2688 (or is 0), so it is exact in bf16 and in fp16.
#pragma once

#include <cuda_fp16.h>

#include "cache_common.cuh"

namespace mone {

// Eight codes of a word as four pairs of halves: element 2 i, low, and 2 i + 1
__device__ __forceinline__ void code_halves(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}
// Two scales, the low byte's low
__device__ __forceinline__ uint32_t scale_halves(uint32_t two) {
    uint32_t h;
    asm("{\n\t.reg .b16 s;\n\tcvt.u16.u32 s, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, s;\n\t}" : "=r"(h) : "r"(two));
    return h;
}
__device__ __forceinline__ float scale_float(uint32_t one) { return __low2float(__halves2half2(__ushort_as_half((unsigned short)scale_halves(one & 0xff)), __half())); }
__device__ __forceinline__ float2 halves_float2(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

// a / b rounded to odd: the next quotient toward zero, its last bit set if it is not exact, so that no rounding after it, to far fewer bits,
// goes another way than a / b itself would (a >= 0, b > 0, inv the rounded 1 / b; a below 2^100 and normal where it matters).  (The
// remainder of a quotient rounded to the nearest is exact in a fused multiply-add.)
__device__ __forceinline__ float quotient_odd(float a, float b, float inv) {
    float q = a * inv;
    q = fmaf(fmaf(-q, b, a), inv, q);
    const float rem = fmaf(-q, b, a);
    const int down = __float_as_int(q) - (rem < 0.f);
    return __int_as_float(rem == 0.f ? down : down | 1);
}

// The scale of a group whose largest |x| / 2^exp is `most`
__device__ __forceinline__ uint32_t encode_scale(float most) {
    uint32_t s;
    const float q = quotient_odd(fminf(most, 2688.f), 6.f, 1.f / 6.f);
    asm("{\n\t.reg .b16 s;\n\tcvt.rn.satfinite.e4m3x2.f32 s, %1, %1;\n\tcvt.u32.u16 %0, s;\n\t}" : "=r"(s) : "f"(q));
    return s & 0xff;
}
// Two codes, of x0 low
__device__ __forceinline__ uint32_t code_two(float x0, float x1) {
    uint32_t c;
    asm("{\n\t.reg .b8 c;\n\tcvt.rn.satfinite.e2m1x2.f32 c, %2, %1;\n\tcvt.u32.u8 %0, c;\n\t}" : "=r"(c) : "f"(x0), "f"(x1));
    return c;
}
// of x0 (low) and x1 under scale `s` > 0, inv the rounded 1 / s
__device__ __forceinline__ uint32_t encode_two(float x0, float x1, float s, float inv) {
    return code_two(copysignf(quotient_odd(fminf(fabsf(x0), 8.f * s), s, inv), x0), copysignf(quotient_odd(fminf(fabsf(x1), 8.f * s), s, inv), x1));
}

__device__ __forceinline__ uint32_t mul_halves(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

}  // namespace mone
