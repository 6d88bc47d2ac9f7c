// The work list of a prompt attention call, and the CUDA-core form of the attention: the path of a context that asks for
// FD_ATTN_SIMT, and what the tensor-core form is compared with.
#include <algorithm>

#include "fd_prompt.cuh"

namespace fd {

constexpr int kPlanThreads = 1024, kPlanMaxBatch = 4096;

__global__ void __launch_bounds__(kPlanThreads) prompt_plan_kernel(PromptParams p, int n_pow2) {
    __shared__ unsigned long long key[kPlanMaxBatch];
    __shared__ long long wsum[kPlanThreads / 32][2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.batch, per = 2 * p.tile_tokens;
    bool bad = false;
    // prefix sums of two numbers a sequence, 1024 sequences at a time
    auto scan2 = [&](long long a, long long c, long long* carry, long long& sa, long long& sc) {
        sa = a; sc = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long ua = __shfl_up_sync(0xffffffffu, sa, o), uc = __shfl_up_sync(0xffffffffu, sc, o);
            if (lane >= o) { sa += ua; sc += uc; }
        }
        __syncthreads();
        if (lane == 31) { wsum[warp][0] = sa; wsum[warp][1] = sc; }
        __syncthreads();
        long long ba = carry[0], bc = carry[1];
        for (int k = 0; k < kPlanThreads / 32; ++k) {
            if (k < warp) { ba += wsum[k][0]; bc += wsum[k][1]; }
            carry[0] += wsum[k][0];
            carry[1] += wsum[k][1];
        }
        sa += ba; sc += bc;  // inclusive
    };
    long long carry[2] = {0, 0};
    if (tid == 0) { p.plan.cu_q[0] = 0; p.plan.cu_kv[0] = 0; p.plan.pre[0] = 0; }
    for (int base = 0; base < n_pow2; base += kPlanThreads) {
        const int b = base + tid;
        long long Lq = 0, Lk = 0;
        if (b < B) {
            Lq = p.q_lens[b];
            Lk = p.kv_lens ? p.kv_lens[b] : Lq;
            if (Lq < 0 || Lk < 0) { bad = true; Lq = Lk = 0; }
        }
        // longest first, of equal ones the first sequence first; padding sorts behind everything
        if (b < n_pow2) key[b] = b < B ? ((unsigned long long)((Lq + per - 1) / per + 1) << 32) | (0xffffffffu - b) : 0ull;
        long long sq, sk;
        scan2(Lq, Lk, carry, sq, sk);
        if (b < B) {
            p.plan.cu_q[b + 1] = (int)min(sq, 0x7fffffffLL);
            p.plan.cu_kv[b + 1] = (int)min(sk, 0x7fffffffLL);
        }
    }
    bad = __syncthreads_or(bad) != 0 || carry[0] != p.total_q || carry[1] != p.total_kv;
    for (int k = 2; k <= n_pow2; k <<= 1)  // bitonic sort, falling
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int i = tid; i < n_pow2; i += kPlanThreads) {
                const int o = i ^ j;
                if (o > i) {
                    const unsigned long long x = key[i], y = key[o];
                    if ((x < y) == ((i & k) == 0)) { key[i] = y; key[o] = x; }
                }
            }
            __syncthreads();
        }
    long long carry2[2] = {0, 0};
    for (int base = 0; base < B; base += kPlanThreads) {
        const int i = base + tid;
        const long long n = i < B ? (long long)(key[i] >> 32) - 1 : 0;
        long long sn, unused;
        scan2(n, 0, carry2, sn, unused);
        if (i < B) {
            p.plan.perm[i] = (int)(0xffffffffu - (unsigned)(key[i] & 0xffffffffu));
            p.plan.blocks[i] = (int)n;
            p.plan.pre[i + 1] = (int)min(sn, 0x7fffffffLL);
        }
    }
    if (tid == 0) {
        *p.plan.fatal = bad;
        if (bad) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
    }
}

cudaError_t launch_prompt_plan(const PromptParams& p, cudaStream_t s) {
    int n = 1;
    while (n < p.batch) n <<= 1;
    return launch(prompt_plan_kernel, 1, kPlanThreads, 0, s, p, n);
}

// One thread a query row; K and V pass through shared memory 16 keys at a time; the online softmax in the log2 domain.
template <int D>
__global__ void __launch_bounds__(kMaxRows) prompt_simt_kernel(PromptParams p) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    float* qT = reinterpret_cast<float*>(smem_raw);                                     // [D][128], pre-scaled
    __nv_bfloat16* ks = reinterpret_cast<__nv_bfloat16*>(smem_raw + D * kMaxRows * 4);  // [16][D]
    __nv_bfloat16* vs = ks + 16 * D;
    const int r = threadIdx.x, G = p.G;
    if (*p.plan.fatal) {  // a defined output, zeros
        const long long n16 = (long long)p.total_q * p.Hq * D / 8;
        for (long long i = (long long)blockIdx.x * kMaxRows + r; i < n16; i += (long long)gridDim.x * kMaxRows)
            reinterpret_cast<uint4*>(p.out)[i] = make_uint4(0, 0, 0, 0);
        return;
    }
    const long long total = (long long)p.plan.pre[p.batch] * p.Hkv;
    for (int turn = 0; (long long)turn * gridDim.x < total; ++turn) {
        const long long t = prompt_turn(turn, blockIdx.x, gridDim.x);
        if (t >= total) continue;
        const PromptItem it = prompt_item(p.plan, p.batch, p.Hkv, t);
        for (int half = 0; half < 2; ++half) {
            const int t0 = (it.place * 2 + half) * p.tile_tokens, rows = min(p.tile_tokens, it.Lq - t0) * G;
            if (rows <= 0) break;
            const int tok = t0 + r / G, head = it.kvh * G + r % G;
            const int limit = r < rows ? it.Lk - it.Lq + tok + 1 : 0;             // keys the row sees
            const int last = min(it.Lk, it.Lk - it.Lq + t0 + (rows - 1) / G + 1);  // ... and any row of the tile
            __syncthreads();  // the tile before is done with qT
            const __nv_bfloat16* qr = p.q + (it.row0 + (long long)tok) * p.q_stride + (long long)head * D;
            for (int c = 0; c < D; ++c) qT[c * kMaxRows + r] = r < rows ? __bfloat162float(qr[c]) * p.scale_log2e : 0.f;
            float m = -INFINITY, l = 0.f, acc[D];
#pragma unroll
            for (int c = 0; c < D; ++c) acc[c] = 0.f;
            for (int j0 = 0; j0 < last; j0 += 16) {
                __syncthreads();
                for (int e = r; e < 16 * D / 8; e += kMaxRows) {
                    const int j = j0 + e / (D / 8), c = (e % (D / 8)) * 8;
                    const long long at = (it.kv0 + (long long)j) * p.kv_stride + (long long)it.kvh * D + c;
                    const uint4 zero = make_uint4(0, 0, 0, 0);
                    reinterpret_cast<uint4*>(ks)[e] = j < last ? *reinterpret_cast<const uint4*>(p.k + at) : zero;
                    reinterpret_cast<uint4*>(vs)[e] = j < last ? *reinterpret_cast<const uint4*>(p.v + at) : zero;
                }
                __syncthreads();
                const int seen = min(16, limit - j0);
                if (seen <= 0) continue;
                float s[16], pm = -INFINITY;
#pragma unroll
                for (int k = 0; k < 16; ++k) s[k] = 0.f;
                for (int c = 0; c < D; c += 2) {
                    const float q0 = qT[c * kMaxRows + r], q1 = qT[(c + 1) * kMaxRows + r];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float2 kk = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(ks + k * D + c));
                        s[k] = fmaf(q0, kk.x, fmaf(q1, kk.y, s[k]));
                    }
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    s[k] = k < seen ? s[k] : -INFINITY;
                    pm = fmaxf(pm, s[k]);
                }
                const float m_new = fmaxf(m, pm), alpha = m == -INFINITY ? 0.f : exp2f(m - m_new);
                l *= alpha;
#pragma unroll
                for (int c = 0; c < D; ++c) acc[c] *= alpha;
                m = m_new;
#pragma unroll 1
                for (int k = 0; k < seen; ++k) {
                    float pj = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) pj = i == k ? s[i] : pj;
                    pj = exp2f(pj - m);
                    l += pj;
#pragma unroll
                    for (int c = 0; c < D; c += 2) {
                        const float2 vv = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(vs + k * D + c));
                        acc[c] = fmaf(pj, vv.x, acc[c]);
                        acc[c + 1] = fmaf(pj, vv.y, acc[c + 1]);
                    }
                }
            }
            if (r < rows) {
                __nv_bfloat16* dst = p.out + ((it.row0 + (long long)tok) * p.Hq + head) * D;
                store_cols_bf16<D>(dst, acc, limit > 0 ? 1.f / l : 0.f);  // (a row that sees no key: zeros)
            }
        }
    }
}

cudaError_t prompt_simt_prepare(int d) {
    if (d != 128) return cudaSuccess;
    return cudaFuncSetAttribute(prompt_simt_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * kMaxRows * 4 + 2 * 16 * 128 * 2);
}

void launch_prompt_simt(const PromptParams& p, cudaStream_t s) {
    const int smem = p.d * kMaxRows * 4 + 2 * 16 * p.d * 2;
    if (p.d == 64) prompt_simt_kernel<64><<<p.n_ctas, kMaxRows, smem, s>>>(p);
    else prompt_simt_kernel<128><<<p.n_ctas, kMaxRows, smem, s>>>(p);
}

}  // namespace fd
