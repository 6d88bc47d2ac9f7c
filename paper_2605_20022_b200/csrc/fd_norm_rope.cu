// Norm of every query and key head, rotation by the position, and the append, in one pass over the projection's output.
//
// D / 8 lanes share a head, 8 consecutive elements (16 bytes) each: the sum of squares is a shuffle tree over those
// lanes, and the element a rotation pairs with element i lies rot_dim / 16 lanes away (or in the same lane, when adjacent
// elements are paired).  A CTA takes one row; the groups of lanes stride over its heads, so the cosines and sines of the
// row's position are read once per lane and stay in registers.  In 4 bits a scale group is two lanes.
#include <algorithm>

#include "fd_fp4.cuh"
#include "fd_internal.cuh"

namespace fd {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void to_float8(const uint4& raw, float (&x)[8]) {
    const __nv_bfloat162* e = reinterpret_cast<const __nv_bfloat162*>(&raw);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = __bfloat1622float2(e[k]);
        x[2 * k] = f.x;
        x[2 * k + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 to_bf16x8(const float (&x)[8]) {
    uint4 raw;
    __nv_bfloat162* e = reinterpret_cast<__nv_bfloat162*>(&raw);
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
    return raw;
}

}  // namespace

template <int D, bool FP4>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(NormRopeParams p) {
    constexpr int LPH = D / 8;                 // lanes per head
    constexpr int kGroups = kThreads / LPH;    // heads in flight per CTA
    const int sub = threadIdx.x % LPH, grp = threadIdx.x / LPH, e0 = sub * 8;
    const unsigned mask = LPH == 32 ? 0xffffffffu : (((1u << LPH) - 1u) << ((threadIdx.x & 31) / LPH * LPH));
    const int heads = p.Hq + 2 * p.Hkv, R = p.rot_dim;
    float wq[8], wk[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) wq[k] = wk[k] = 1.f;
    if (p.q_weight) to_float8(*reinterpret_cast<const uint4*>(p.q_weight + e0), wq);
    if (p.k_weight) to_float8(*reinterpret_cast<const uint4*>(p.k_weight + e0), wk);
    for (int t = blockIdx.x; t < p.total_rows; t += gridDim.x) {
        const int slot = p.slot_map[t], pos = R ? p.positions[t] : 0;
        if (slot < 0) continue;  // padding
        if (R && (unsigned)pos >= (unsigned)p.max_positions) {
            if (threadIdx.x == 0) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
            continue;
        }
        const int page = slot >> 4, tok = slot & 15;
        const bool store_kv = page < p.num_pages;  // never form an address from a bad slot
        if (!store_kv && threadIdx.x == 0) atomicOr(p.status, FD_DEV_BAD_PAGE);
        // cosine and signed sine of each of the lane's elements: y_e = x_e c + x_partner s
        float c[8], s[8];
        const bool turn = e0 < R;
        if (turn) {
            const float* row = p.cos_sin + (long long)pos * R;
            if (p.adjacent) {
                const float4 cc = *reinterpret_cast<const float4*>(row + e0 / 2), ss = *reinterpret_cast<const float4*>(row + R / 2 + e0 / 2);
                const float c4[4] = {cc.x, cc.y, cc.z, cc.w}, s4[4] = {ss.x, ss.y, ss.z, ss.w};
#pragma unroll
                for (int k = 0; k < 8; ++k) { c[k] = c4[k >> 1]; s[k] = (k & 1) ? s4[k >> 1] : -s4[k >> 1]; }
            } else {
                const bool hi = e0 >= R / 2;
                const float4* cr = reinterpret_cast<const float4*>(row + (hi ? e0 - R / 2 : e0));
                const float4* sr = reinterpret_cast<const float4*>(row + (hi ? e0 : e0 + R / 2));
                const float4 c0 = cr[0], c1 = cr[1], s0 = sr[0], s1 = sr[1];
                const float c8[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, s8[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
                for (int k = 0; k < 8; ++k) { c[k] = c8[k]; s[k] = hi ? s8[k] : -s8[k]; }
            }
        }
        const int partner = p.adjacent || !turn ? sub : (e0 < R / 2 ? sub + R / 16 : sub - R / 16);
        for (int h = grp; h < heads; h += kGroups) {
            const uint4 raw = *reinterpret_cast<const uint4*>(p.qkv + (long long)t * p.row_stride + (long long)h * D + e0);
            float x[8];
            to_float8(raw, x);
            const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
            if (!is_v) {
                if (is_q ? p.q_weight != nullptr : p.k_weight != nullptr) {
                    float ss = 0.f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) ss = fmaf(x[k], x[k], ss);
#pragma unroll
                    for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(mask, ss, o);
                    const float r = __fdiv_rn(1.0f, __fsqrt_rn(ss * (1.0f / D) + p.eps));
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = x[k] * r * (is_q ? wq[k] : wk[k]);
                }
                if (R) {
                    float y[8];
                    if (p.adjacent) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = x[k ^ 1];
                    } else {
                        const int src = (threadIdx.x & 31) - sub + partner;
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = __shfl_sync(mask, x[k], src);
                    }
                    if (turn) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[k] = fmaf(x[k], c[k], y[k] * s[k]);
                    }
                }
            }
            if (is_q) {
                *reinterpret_cast<uint4*>(p.q_out + ((long long)t * p.Hq + h) * D + e0) = to_bf16x8(x);
                continue;
            }
            if (!store_kv) continue;  // (uniform over the CTA)
            const int which = is_v ? 1 : 0, kvh = h - p.Hq - (is_v ? p.Hkv : 0);
            if (!FP4) {
                *reinterpret_cast<uint4*>(p.kv + ((((long long)page * 2 + which) * p.Hkv + kvh) * 16 + tok) * D + e0) = is_v ? raw : to_bf16x8(x);
            } else {
                const float by = which ? p.v_scale : p.k_scale;
                float amax = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    x[k] = __fdiv_rn(x[k], by);
                    amax = fmaxf(amax, fabsf(x[k]));
                }
                amax = fmaxf(amax, __shfl_xor_sync(mask, amax, 1));
                const uint8_t sb = e4m3_scale(amax);
                const Fp4Thresholds th(e4m3_to_float(sb));
                unsigned char* base = p.kv4 + fp4_page_offset(page, p.Hkv, kvh, which, D);
                *reinterpret_cast<uint32_t*>(base + tok * (D / 2) + e0 / 2) = e2m1_code8(x, th);
                if ((sub & 1) == 0) base[fp4_scale_offset(D) + tok * (D / 16) + e0 / 16] = sb;
            }
        }
    }
}

void launch_norm_rope(const NormRopeParams& p, cudaStream_t s) {
    const int grid = std::min(p.total_rows, 8 * p.n_sms);
    const bool fp4 = p.kv4 != nullptr;
    if (p.d == 64) {
        if (fp4) norm_rope_kernel<64, true><<<grid, kThreads, 0, s>>>(p);
        else norm_rope_kernel<64, false><<<grid, kThreads, 0, s>>>(p);
    } else {
        if (fp4) norm_rope_kernel<128, true><<<grid, kThreads, 0, s>>>(p);
        else norm_rope_kernel<128, false><<<grid, kThreads, 0, s>>>(p);
    }
}

}  // namespace fd
