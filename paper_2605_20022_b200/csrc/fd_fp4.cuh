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

// max that keeps a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// x / by, correctly rounded: a product with the rounded reciprocal, and one step with the exact remainder (Markstein, "Computation
// of elementary functions on the IBM RISC System/6000 processor", 1990).  Three instructions against the ten of a
// division.  x finite and neither so large nor so small that the remainder leaves the range.
__device__ __forceinline__ float quotient(float x, float by, float inv) {
    const float q = fmaf(x, inv, 0.f);  // (the sum with +0 turns a -0 into +0)
    return fmaf(fmaf(-q, by, x), inv, q);
}

// Quantisation of groups of x / by (by: the scale of K or of V).  Every step of the definition is a correctly rounded quotient:
// y = x / by, the scale the nearest e4m3 number to max |y| / 6 (a product with 1 / 6 would put the ties of bf16 inputs on
// either side), at most 448, and the code the e2m1 conversion of y / s.  The last is the nearest code, of two the even one,
// exactly, for a y / s that is not a tie does not round onto one: a tie t is 1, 1.25, 1.5 or 1.75 times a power of two and
// t s has at most 7 bits, so y differs from t s by at least one unit in its last place and y / s from t by more than 2^-24
// of it, while t's neighbours are at least 2^-24 of it (above) or 2^-25 (below, t = 1) from the middle.
//
// odd(amax) says whether a group must go the long way: something in it is not finite, or so large (or by so far from 1)
// that the remainders leave their range.  Far below 2^-90 they may underflow, where every quotient is held as 0 anyway.
struct Fp4Scale {
    float s, inv;
    uint8_t byte;
    __device__ __forceinline__ void round(float sixth) {
        uint16_t r;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(fminf(sixth, 448.0f)));
        byte = (uint8_t)(r & 0xff);
        s = e4m3_to_float(byte);
        float r0;  // 1 / s, correctly rounded: eight significands, none of whose reciprocals is near a midpoint
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(s));
        inv = s > 0.f ? fmaf(fmaf(-s, r0, 1.0f), r0, r0) : 1e-30f;  // (zero scale: every quotient comes out as a zero of x's sign)
    }
};

struct Fp4Quantiser {
    float by, inv;
    bool quick;
    __device__ __forceinline__ explicit Fp4Quantiser(float b) {
        by = b;
        inv = __fdiv_rn(1.0f, b);
        quick = b > 1e-9f && b < 1e9f;
    }
    __device__ __forceinline__ bool odd(float amax_nan) const { return !quick || !(amax_nan < 1.2379400e27f); }
    // of a group whose largest magnitude is amax (division is monotone: the largest quotient is the largest x's)
    __device__ __forceinline__ Fp4Scale scale(float amax) const {
        Fp4Scale g;
        g.round(quotient(quotient(amax, by, inv), 6.0f, 1.0f / 6.0f));
        return g;
    }
    template <int N>
    __device__ __forceinline__ uint32_t codes(const float* x, const Fp4Scale& g) const {
        float q[N];
#pragma unroll
        for (int k = 0; k < N; ++k) q[k] = quotient(quotient(x[k], by, inv), g.s, g.inv);
        return convert<N>(q);
    }
    // The long way: a NaN counts as 0, an infinity takes the largest code.
    __device__ __forceinline__ Fp4Scale scale_long(float amax_without_nan) const {
        Fp4Scale g;
        g.round(__fdiv_rn(__fdiv_rn(amax_without_nan, by), 6.0f));
        return g;
    }
    template <int N>
    __device__ __forceinline__ uint32_t codes_long(const float* x, const Fp4Scale& g) const {
        float q[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float y = __fdiv_rn(x[k], by);
            q[k] = y != y ? 0.f : y == 0.f ? 0.f : g.s > 0.f ? __fdiv_rn(y, g.s) : copysignf(0.f, y);
        }
        return convert<N>(q);
    }
    // N elements (4 or 8) -> their codes, the first in the low bits.
    template <int N>
    __device__ __forceinline__ static uint32_t convert(const float (&q)[N]) {
        uint32_t w;
        if (N == 4) {
            uint16_t h;
            asm("{\n\t.reg .b8 b0, b1;\n\t"
                "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
                "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
                "mov.b16 %0, {b0, b1};\n\t}"
                : "=h"(h)
                : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]));
            w = h;
        } else {
            asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
                "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
                "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
                "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
                "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
                "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
                : "=r"(w)
                : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[N > 4 ? 4 : 0]), "f"(q[N > 4 ? 5 : 0]), "f"(q[N > 4 ? 6 : 0]), "f"(q[N > 4 ? 7 : 0]));
        }
        return w;
    }
};

}  // namespace fd
