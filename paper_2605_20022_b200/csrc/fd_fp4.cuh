// The 4-bit KV cache: layout of its pages, and the conversions from and to its values.
//
// 16 consecutive elements of a head's row share an e4m3 scale and are held as e2m1 codes.  A value's significand then has
// at most 2 + 4 bits, so code * scale is exact in bf16 and, as the exponents of the two stay within [2^-10, 2688], in
// fp16 as well: reading the cache rounds nothing.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace fd {

constexpr int kFp4Group = 16;  // elements per scale

// Bytes of one page (16 tokens) of K or V of one kv-head: codes [16][d / 2], then scales [16][d / 16].
__host__ __device__ constexpr int fp4_page_bytes(int d) { return 16 * (d / 2 + d / 16); }
__host__ __device__ constexpr int fp4_scale_offset(int d) { return 16 * (d / 2); }
// Where page `page`'s K (which = 0) or V (which = 1) of kv-head h starts.
__host__ __device__ constexpr long long fp4_page_offset(long long page, int Hkv, int h, int which, int d) {
    return ((page * Hkv + h) * 2 + which) * fp4_page_bytes(d);
}

// Four bytes of codes -> eight fp16 values, in order.
__device__ __forceinline__ void e2m1x8_to_half(uint32_t codes, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
}
// Two scale bytes -> two fp16 values.
__device__ __forceinline__ uint32_t e4m3x2_to_half(uint16_t scales) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(scales));
    return h;
}
__device__ __forceinline__ __half2 as_half2(uint32_t u) { return *reinterpret_cast<const __half2*>(&u); }
__device__ __forceinline__ uint32_t as_u32(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
__device__ __forceinline__ float e4m3_to_float(uint8_t scale) { return __low2float(as_half2(e4m3x2_to_half(scale))); }

// Scale byte of a group whose largest magnitude is amax: nearest e4m3 number to amax / 6 (true division: with a
// product by 1 / 6 the ties of bf16 inputs would fall either way), at most 448.
__device__ __forceinline__ uint8_t e4m3_scale(float amax) {
    const float s = fminf(__fdiv_rn(amax, 6.0f), 448.0f);
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(s));
    return (uint8_t)(r & 0xff);
}

// Thresholds of a group with scale s: t[k] separates codes k and k + 1.  Each is a product of at most 3 + 4 bits, hence
// exact, so the comparison below is the definition (nearest multiple of s, of two the even code), not an approximation of
// it; x / s would round, and x * (1 / s) would put exact ties -- common among bf16 inputs -- on either side.
struct Fp4Thresholds {
    float t[7];
    __device__ __forceinline__ explicit Fp4Thresholds(float s) {
        const float k[7] = {0.25f, 0.75f, 1.25f, 1.75f, 2.5f, 3.5f, 5.0f};
#pragma unroll
        for (int i = 0; i < 7; ++i) t[i] = s > 0.f ? k[i] * s : INFINITY;  // zero scale: every code is 0 (an infinity cannot meet it)
    }
};
// Code of x: a binary search; an even code takes its lower threshold in (>=), an odd one does not (>).
__device__ __forceinline__ uint32_t e2m1_code(float x, const Fp4Thresholds& th) {
    const float a = fabsf(x);  // a NaN fails every comparison: code 0
    const bool c2 = a >= th.t[3];
    const bool c1 = a >= (c2 ? th.t[5] : th.t[1]);
    const bool c0 = a > (c2 ? (c1 ? th.t[6] : th.t[4]) : (c1 ? th.t[2] : th.t[0]));
    return (c2 ? 4u : 0u) | (c1 ? 2u : 0u) | (c0 ? 1u : 0u) | (x < 0.f ? 8u : 0u);
}
// Eight elements -> four bytes of codes.
__device__ __forceinline__ uint32_t e2m1_code8(const float* x, const Fp4Thresholds& th) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= e2m1_code(x[i], th) << (4 * i);
    return w;
}

}  // namespace fd
