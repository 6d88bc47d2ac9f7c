// Norm of every query and key head, rotation by the position, and the append, in one pass over the projection's output.
//
// D / 8 lanes share a head, 8 elements each; a warp takes a part of one row's heads, so the row's slot, position, cosines and
// sines are read once and stay in registers, the heads' loads are independent of one another, and no warp waits for another.
// A row is cut into as many parts as it takes to occupy the GPU (one row's 48 heads are 24 warps' work; a batch of prompts is a
// warp a row).  Two layouts of a lane's elements:
//   kHalves   the whole head is rotated and halves are paired: elements 4 l .. 4 l + 3 and the same of the upper half, so that a
//             pair lies in one lane;
//   kGeneral  8 consecutive elements: the partner lies in the same lane (adjacent pairs) or rot_dim / 16 lanes away.
// In 4 bits a scale group is four lanes (kHalves) or two.  12 KB in, 8 KB and the cache out per row of 32 + 8 + 8 heads of 128:
// 9785 rows take 69 us into 4-bit pages and 66 into bf16 pages (33 and 37 us of bytes), calls replayed from a graph; adjacent
// pairs 66 and 57, half of the head rotated 69 and 61.  The warps wait for their loads: a quarter of them is resident, as registers
// hold the loads in flight, and half of the issue slots are used.  A CTA a row, and the read back of the cache behind it, took
// 128 us, a warp a row 91.  One sequence's 32 rows: 2.9 us.
#include <algorithm>
#include <type_traits>

#include "fd_fp4.cuh"
#include "fd_internal.cuh"

namespace fd {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
enum { kHalves = 0, kGeneral = 1 };

// A lane's eight elements from or to the head that starts at `head`: two runs of four, or one of eight.
template <int D, int LAYOUT>
__device__ __forceinline__ uint4 load8(const __nv_bfloat16* head, int sub) {
    if (LAYOUT == kGeneral) return *reinterpret_cast<const uint4*>(head + sub * 8);
    const uint2 lo = *reinterpret_cast<const uint2*>(head + sub * 4), hi = *reinterpret_cast<const uint2*>(head + D / 2 + sub * 4);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
}
template <int D, int LAYOUT>
__device__ __forceinline__ void store8(__nv_bfloat16* head, int sub, const uint4& v) {
    if (LAYOUT == kGeneral) {
        *reinterpret_cast<uint4*>(head + sub * 8) = v;
    } else {
        *reinterpret_cast<uint2*>(head + sub * 4) = make_uint2(v.x, v.y);
        *reinterpret_cast<uint2*>(head + D / 2 + sub * 4) = make_uint2(v.z, v.w);
    }
}
__device__ __forceinline__ void unpack8(const uint4& raw, float2 (&x)[4]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = make_float2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack8(const float2 (&x)[4]) {
    uint4 raw;
    __nv_bfloat162* e = reinterpret_cast<__nv_bfloat162*>(&raw);
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = __floats2bfloat162_rn(x[k].x, x[k].y);
    return raw;
}

// What of a row stays in registers while its heads are worked through.
template <int LAYOUT>
struct Turn {
    float2 c[LAYOUT == kHalves ? 2 : 4], s[LAYOUT == kHalves ? 2 : 4];  // of the lane's pairs, or (signed) of each of its elements
    int partner;   // kGeneral: the lane that holds the partners
    bool any, adjacent, mine;
};

// Norm (weight w; scaled: there is one) and rotation of a head's elements.
template <int D, int LAYOUT>
__device__ __forceinline__ void norm_and_turn(float2 (&x)[4], const float2 (&w)[4], bool scaled, float eps, const Turn<LAYOUT>& t) {
    constexpr int LPH = D / 8;
    if (scaled) {
        float2 sq = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 4; ++k) sq = __ffma2_rn(x[k], x[k], sq);
        float ss = sq.x + sq.y;
#pragma unroll
        for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float v = ss * (1.0f / D) + eps, r0 = rsqrtf(v);
        const float r = fmaf(0.5f * r0, fmaf(-v * r0, r0, 1.0f), r0);  // one Newton step: to the last place or next to it
        const float rr = v < 1e30f && v > 1e-30f ? r : r0;            // (out there the step's products leave the range)
        const float2 r2 = make_float2(rr, rr);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = __fmul2_rn(__fmul2_rn(x[k], r2), w[k]);
    }
    if (LAYOUT == kHalves) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float2 a = x[k], b = x[k + 2], bs = __fmul2_rn(b, t.s[k]);
            x[k] = __ffma2_rn(a, t.c[k], make_float2(-bs.x, -bs.y));
            x[k + 2] = __ffma2_rn(b, t.c[k], __fmul2_rn(a, t.s[k]));
        }
    } else if (t.any) {
        float2 y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            y[k] = t.adjacent ? make_float2(x[k].y, x[k].x)
                              : make_float2(__shfl_sync(0xffffffffu, x[k].x, t.partner), __shfl_sync(0xffffffffu, x[k].y, t.partner));
        if (t.mine) {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __ffma2_rn(x[k], t.c[LAYOUT == kHalves ? 0 : k], __fmul2_rn(y[k], t.s[LAYOUT == kHalves ? 0 : k]));
        }
    }
}

// A head of k or v into the 4-bit cache: `base` is its page, store: this lane's head exists.  The whole warp (it shuffles).
template <int D, int LAYOUT>
__device__ __forceinline__ void store_fp4(const float2 (&x2)[4], const Fp4Quantiser& by, unsigned char* base, int tok, int sub, bool store) {
    const float x[8] = {x2[0].x, x2[0].y, x2[1].x, x2[1].y, x2[2].x, x2[2].y, x2[3].x, x2[3].y};
    constexpr int N = LAYOUT == kHalves ? 4 : 8, G = 8 / N;  // elements of a group in this lane, and groups
    auto widest = [&](const float* y, auto mx) {             // over the group's lanes
        float a = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) a = mx(a, fabsf(y[k]));
        a = mx(a, __shfl_xor_sync(0xffffffffu, a, 1));
        return N == 8 ? a : mx(a, __shfl_xor_sync(0xffffffffu, a, 2));
    };
    float amax[G];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < G; ++i) {
        amax[i] = widest(x + N * i, [](float a, float b) { return max_nan(a, b); });
        odd = odd || by.odd(amax[i]);
    }
    Fp4Scale g[G];
    uint32_t w[G];
    if (!__any_sync(0xffffffffu, odd)) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            g[i] = by.scale(amax[i]);
            w[i] = by.codes<N>(x + N * i, g[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            g[i] = by.scale_long(widest(x + N * i, [](float a, float b) { return fmaxf(a == a ? a : 0.f, b == b ? b : 0.f); }));  // (drops a NaN)
            w[i] = by.codes_long<N>(x + N * i, g[i]);
        }
    }
    if (!store) return;
    unsigned char *codes = base + tok * (D / 2), *scales = base + fp4_scale_offset(D) + tok * (D / 16);
#pragma unroll
    for (int i = 0; i < G; ++i) {
        if (N == 4) *reinterpret_cast<uint16_t*>(codes + i * (D / 4) + sub * 2) = (uint16_t)w[i];
        else *reinterpret_cast<uint32_t*>(codes + sub * 4) = w[i];
        if ((sub & (16 / N - 1)) == 0) scales[i * (D / 32) + sub / (16 / N)] = g[i].byte;
    }
}

}  // namespace

// The heads i0, i0 + di, ... (in steps of 32 / LPH heads) of one kind -- KIND 0: q, 1: k, 2: v -- of a row; `src` is this lane's
// place in the kind's first head, `dst` where its first head goes.  The loads of the next steps are in flight while one is worked on.
template <int D, bool FP4, int LAYOUT, int KIND>
__device__ __forceinline__ void do_heads(const __nv_bfloat16* src, int count, int i0, int di, const float2 (&w)[4], bool scaled, float eps,
                                         const Turn<LAYOUT>& turn, __nv_bfloat16* dst, long long dst_step, const Fp4Quantiser& by,
                                         unsigned char* dst4, int tok, int sub, int hl) {
    constexpr int HPW = 256 / D, L = KIND == 2 ? kGeneral : LAYOUT;  // v is not rotated: consecutive elements whatever the layout
    constexpr int U = KIND == 0 ? 4 : 2;  // loads in flight
    const int step = di * HPW;
    int h = i0 * HPW + hl;
    const __nv_bfloat16* from = src + (long long)h * D;
    uint4 next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        next[u] = make_uint4(0, 0, 0, 0);
        if (h + u * step < count) next[u] = load8<D, L>(from + u * step * D, sub);
    }
    for (; h - hl < count; h += U * step) {  // uniform over the warp (it shuffles)
        from += U * step * D;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int hu = h + u * step;
            if (u > 0 && hu - hl >= count) break;  // uniform
            const uint4 now = next[u];
            if (hu + U * step < count) next[u] = load8<D, L>(from + u * step * D, sub);
            float2 x[4];
            unpack8(now, x);
            if (KIND < 2) norm_and_turn<D, LAYOUT>(x, w, scaled, eps, turn);
            if (FP4 && KIND > 0) store_fp4<D, L>(x, by, dst4 + (long long)min(hu, count - 1) * (2 * fp4_page_bytes(D)), tok, sub, hu < count);
            else if (hu < count) store8<D, L>(dst + hu * dst_step, sub, KIND == 2 ? now : pack8(x));
        }
    }
}

// FMT: where k and v go (FD_KV_BF16, FD_KV_FP4, FD_KV_ROWS).
template <int D, int FMT, int LAYOUT>
__global__ void __launch_bounds__(kThreads, 5) norm_rope_kernel(NormRopeParams p, int parts) {
    constexpr bool FP4 = FMT == FD_KV_FP4, ROWS = FMT == FD_KV_ROWS;
    constexpr int LPH = D / 8;         // lanes per head
    constexpr int HPW = 32 / LPH;      // heads a warp works on at a time
    const int lane = threadIdx.x & 31, sub = lane % LPH, hl = lane / LPH, R = p.rot_dim;
    const int nq = (p.Hq + HPW - 1) / HPW, nk = (p.Hkv + HPW - 1) / HPW;
    float2 wq[4], wk[4];
    if (p.q_weight) unpack8(load8<D, LAYOUT>(p.q_weight, sub), wq);
    if (p.k_weight) unpack8(load8<D, LAYOUT>(p.k_weight, sub), wk);
    const Fp4Quantiser by_k(FP4 ? p.k_scale : 1.f), by_v(FP4 ? p.v_scale : 1.f);
    const long long tasks = (long long)p.total_rows * parts;
    for (long long task = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); task < tasks; task += (long long)gridDim.x * kWarps) {
        const int t = (int)(task / parts), part = (int)(task - (long long)t * parts);
        const int slot = p.slot_map[t], pos = R ? p.positions[t] : 0;
        const __nv_bfloat16* src = p.qkv + (long long)t * p.row_stride;
        if (slot < 0) continue;  // padding (uniform over the warp, as all that depends on the row)
        if (R && (unsigned)pos >= (unsigned)p.max_positions) {
            if (lane == 0) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
            continue;
        }
        const int page = slot >> 4, tok = slot & 15;
        const bool store_kv = page < p.num_pages;  // never form an address from a bad slot
        if (!store_kv && lane == 0) atomicOr(p.status, FD_DEV_BAD_PAGE);
        Turn<LAYOUT> turn;
        turn.any = R > 0;
        turn.adjacent = p.adjacent;
        turn.mine = sub * 8 < R;
        turn.partner = lane;
        if (LAYOUT == kHalves) {
            const float* row = p.cos_sin + (long long)pos * D + sub * 4;
            const float4 cc = *reinterpret_cast<const float4*>(row), ss = *reinterpret_cast<const float4*>(row + D / 2);
            turn.c[0] = make_float2(cc.x, cc.y); turn.c[1] = make_float2(cc.z, cc.w);
            turn.s[0] = make_float2(ss.x, ss.y); turn.s[1] = make_float2(ss.z, ss.w);
        } else if (turn.mine) {
            constexpr int kLast = LAYOUT == kHalves ? 1 : 3;
            const int e0 = sub * 8;
            const float* row = p.cos_sin + (long long)pos * R;
            if (p.adjacent) {
                const float4 cc = *reinterpret_cast<const float4*>(row + e0 / 2), ss = *reinterpret_cast<const float4*>(row + R / 2 + e0 / 2);
                const float c4[4] = {cc.x, cc.y, cc.z, cc.w}, s4[4] = {ss.x, ss.y, ss.z, ss.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    turn.c[k < kLast ? k : kLast] = make_float2(c4[k], c4[k]);
                    turn.s[k < kLast ? k : kLast] = make_float2(-s4[k], s4[k]);
                }
            } else {
                const bool hi = e0 >= R / 2;
                const float* cr = row + (hi ? e0 - R / 2 : e0);
                const float* sr = cr + R / 2;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 cc = *reinterpret_cast<const float2*>(cr + 2 * k), ss = *reinterpret_cast<const float2*>(sr + 2 * k);
                    turn.c[k < kLast ? k : kLast] = cc;
                    turn.s[k < kLast ? k : kLast] = hi ? ss : make_float2(-ss.x, -ss.y);
                }
                turn.partner = hi ? lane - R / 16 : lane + R / 16;
            }
        }
        // a row's steps, q's first, go round the parts: where k's and v's begin for this one
        const int ik = ((part - nq) % parts + parts) % parts, iv = ((part - nq - nk) % parts + parts) % parts;
        do_heads<D, FP4, LAYOUT, 0>(src, p.Hq, part, parts, wq, p.q_weight != nullptr, p.eps, turn, p.q_out + (long long)t * p.Hq * D, D, by_k, nullptr, tok,
                                    sub, hl);
        if (!store_kv) continue;
        // (steps that the compiler knows; out of the parameters they cost 5 % on two prompts into bf16 pages, 9.7 us for 9.3)
        constexpr int head_step = ROWS ? D : 16 * D;
        __nv_bfloat16* k_dst = FP4 ? nullptr : p.kv + (ROWS ? (long long)slot * p.Hkv : (long long)page * 2 * p.Hkv * 16 + tok) * D;
        unsigned char* k_dst4 = FP4 ? p.kv4 + fp4_page_offset(page, p.Hkv, 0, 0, D) : nullptr;
        do_heads<D, FP4, LAYOUT, 1>(src + (long long)p.Hq * D, p.Hkv, ik, parts, wk, p.k_weight != nullptr, p.eps, turn, k_dst, head_step, by_k, k_dst4, tok, sub, hl);
        do_heads<D, FP4, LAYOUT, 2>(src + (long long)(p.Hq + p.Hkv) * D, p.Hkv, iv, parts, wk, false, p.eps, turn,
                                    FP4 ? nullptr : k_dst + (long long)p.Hkv * (ROWS ? p.num_pages * 16LL : 16) * D, head_step, by_v, FP4 ? k_dst4 + fp4_page_bytes(D) : nullptr, tok, sub, hl);
    }
}

template <int D, int FMT>
static void launch_layout(const NormRopeParams& p, cudaStream_t s) {
    constexpr int HPW = 32 / (D / 8);
    const int steps = (p.Hq + HPW - 1) / HPW + 2 * ((p.Hkv + HPW - 1) / HPW);
    // as many parts to a row as keep about sixteen warps on every SM busy, of at least one step each
    const int parts = (int)std::max(1LL, std::min<long long>(steps, 16LL * p.n_sms / p.total_rows));
    const long long ctas = ((long long)p.total_rows * parts + kWarps - 1) / kWarps;
    const int grid = (int)std::min<long long>(ctas, 16LL * p.n_sms);
    if (!p.adjacent && p.rot_dim == D) norm_rope_kernel<D, FMT, kHalves><<<grid, kThreads, 0, s>>>(p, parts);
    else norm_rope_kernel<D, FMT, kGeneral><<<grid, kThreads, 0, s>>>(p, parts);
}

void launch_norm_rope(const NormRopeParams& p, cudaStream_t s) {
    auto of = [&](auto d) {
        constexpr int D = decltype(d)::value;
        p.fmt == FD_KV_FP4 ? launch_layout<D, FD_KV_FP4>(p, s) : p.fmt == FD_KV_ROWS ? launch_layout<D, FD_KV_ROWS>(p, s) : launch_layout<D, FD_KV_BF16>(p, s);
    };
    if (p.d == 64) of(std::integral_constant<int, 64>{});
    else of(std::integral_constant<int, 128>{});
}

}  // namespace fd
