// The 8-bit KV cache: layout of its pages, and the conversions from and to its values.
//
// The 16 tokens of a page share, for each kv-head and for K and V apart, one scale; every element is an e4m3 code.  The scale is
// a power of two from 2^-15 to 2^7, the smallest for which the largest magnitude of the block's tokens is at most 448 (e4m3's
// largest) times it.  A power of two loses nothing against amax / 448: e4m3 is a floating format, its steps follow the
// element, not the scale.  What it gains: products with it are exact, so when a louder token joins a block the codes
// that are there move to the new scale without a second rounding (but for those that fall among e4m3's subnormals), and code *
// scale -- four significant bits, multiples of 2^-24, at most 448 * 2^7 = 57344 -- is exact in fp16 as it is in bf16.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "fd_fp4.cuh"  // as_half2, as_u32, e4m3x2_to_half

namespace fd {

constexpr int kFp8Tail = 16;  // bytes behind a block's codes: the scale in 32 bits, then zeros (blocks stay 16-byte multiples)
constexpr int kFp8MinExp = -15, kFp8MaxExp = 7;

// Bytes of one block (a page's 16 tokens of K or V of one kv-head): codes [16][d], then the tail.
__host__ __device__ constexpr int fp8_block_bytes(int d) { return 16 * d + kFp8Tail; }
// Where page `page`'s K (which = 0) or V (which = 1) of kv-head h starts.
__host__ __device__ constexpr long long fp8_block_offset(long long page, int Hkv, int h, int which, int d) {
    return ((page * Hkv + h) * 2 + which) * fp8_block_bytes(d);
}

// The exponent of the scale of a block whose largest magnitude is amax: 448 is 1.75 * 2^8, so adding all mantissa bits above
// 0.75 carries into the exponent exactly where amax passes 448 times the power of two below it.
__device__ __forceinline__ int fp8_scale_exp(float amax) {
    const int e = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 135;
    return min(max(e, kFp8MinExp), kFp8MaxExp);
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // e in [-126, 127]

// Two fp32 values -> two codes, the first in the low byte: nearest, ties to even; beyond 448, infinities too, 448; a NaN stays one.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// Four codes -> four fp16 values in two words.
__device__ __forceinline__ void e4m3x4_to_half(uint32_t codes, uint32_t& a, uint32_t& b) {
    a = e4m3x2_to_half((uint16_t)(codes & 0xffffu));
    b = e4m3x2_to_half((uint16_t)(codes >> 16));
}

}  // namespace fd
