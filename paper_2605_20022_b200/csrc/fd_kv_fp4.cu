// K and V of the query block into the 4-bit cache and out of it.
//
// A thread owns one scale group: 16 elements, 32 bytes of bf16 on one side, 8 bytes of codes and a scale byte on the other.
// Neighbouring threads own neighbouring groups of a row, so both sides are contiguous across a warp.
#include <algorithm>

#include "fd_fp4.cuh"
#include "fd_internal.cuh"

namespace fd {

namespace {

constexpr int kThreads = 256;

constexpr int kWarps = kThreads / 32;
constexpr int kMaxBatch = 4096;  // what fd_create allows

// Exclusive scan of the query lengths into cu[0 .. B] (negative lengths count as 0, sums beyond 32 bits saturate).
__device__ __forceinline__ void scan_lengths(const int32_t* q_lens, int B, int* cu, long long* wsum) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long carry = 0;
    if (tid == 0) cu[0] = 0;
    for (int base = 0; base < B; base += kThreads) {
        long long v = base + tid < B ? max(q_lens[base + tid], 0) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        __syncthreads();  // wsum may still be read from the previous round
        if (lane == 31) wsum[warp] = v;
        __syncthreads();
        long long before = carry;
        for (int k = 0; k < kWarps; ++k) {
            if (k < warp) before += wsum[k];
            carry += wsum[k];
        }
        if (base + tid < B) cu[base + tid + 1] = (int)min(before + v, 0x7fffffffLL);
    }
    __syncthreads();
}

// The sequence that owns query row `row`: the last b with cu[b] <= row (a whole warp; 32 probes a round, at most three rounds).
__device__ __forceinline__ int owner_of_row(const int* cu, int B, long long row) {
    int lo = 0, n = B;  // the answer lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + (int)(threadIdx.x & 31) * step;
        const unsigned below = __ballot_sync(0xffffffffu, at < lo + n && cu[min(at, B)] <= row);
        const int k = 31 - __clz(below | 1u);
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

__device__ __forceinline__ void load_group(const __nv_bfloat16* src, float by, float (&x)[kFp4Group]) {
    __align__(16) __nv_bfloat16 e[kFp4Group];
    reinterpret_cast<uint4*>(e)[0] = reinterpret_cast<const uint4*>(src)[0];
    reinterpret_cast<uint4*>(e)[1] = reinterpret_cast<const uint4*>(src)[1];
#pragma unroll
    for (int k = 0; k < kFp4Group; ++k) x[k] = __fdiv_rn(__bfloat162float(e[k]), by);
}

}  // namespace

template <bool READ>
__global__ void __launch_bounds__(kThreads) kv_rows_fp4_kernel(Fp4RowsParams p) {
    __shared__ int cu[kMaxBatch + 1];
    __shared__ long long wsum[kWarps];
    const int tid = threadIdx.x, lane = tid & 31;
    scan_lengths(p.q_lens, p.batch, cu, wsum);
    const int groups = p.d / kFp4Group, per_row = p.Hkv * groups;  // of K, and again of V
    const long long rows = min(cu[p.batch], p.total_rows);
    bool bad_page = false;
    if (blockIdx.x == 0)  // a sequence that is skipped: the status alone (its rows are met below, by whoever owns them)
        for (int b = tid; b < p.batch; b += kThreads) {
            const long long n = p.prefix_lens[b], Lq = p.q_lens[b];
            if (Lq > 0 && (n < 0 || cu[b] + Lq > p.total_rows || n + Lq > (long long)p.max_pages * 16)) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
        }
    for (long long row = (long long)blockIdx.x * kWarps + (tid >> 5); row < rows; row += (long long)gridDim.x * kWarps) {  // a warp a row
        const int b = owner_of_row(cu, p.batch, row);
        const int n = p.prefix_lens[b], Lq = p.q_lens[b];
        const bool skip = n < 0 || (long long)cu[b] + Lq > p.total_rows || (long long)n + Lq > (long long)p.max_pages * 16;
        if (skip && !READ) continue;
        const int j = skip ? 0 : n + (int)(row - cu[b]);
        const int page = skip ? -1 : p.page_table[(long long)b * p.max_pages + (j >> 4)];
        const bool ok = (unsigned)page < (unsigned)p.num_pages;  // never form an address from a bad id
        bad_page = bad_page || (!ok && !skip);
        for (int e = lane; e < 2 * per_row; e += 32) {
            const int which = e / per_row, h = e % per_row / groups, g = e % groups;
            __nv_bfloat16* rowp = (which ? p.v : p.k) + (row * p.Hkv + h) * p.d + g * kFp4Group;
            const float by = which ? p.v_scale : p.k_scale;
            if (!ok) {
                if (READ) {
                    reinterpret_cast<uint4*>(rowp)[0] = make_uint4(0, 0, 0, 0);
                    reinterpret_cast<uint4*>(rowp)[1] = make_uint4(0, 0, 0, 0);
                }
                continue;
            }
            unsigned char* base = p.kv4 + fp4_page_offset(page, p.Hkv, h, which, p.d);
            uint2* codes = reinterpret_cast<uint2*>(base + (j & 15) * (p.d / 2) + g * 8);
            unsigned char* scale = base + fp4_scale_offset(p.d) + (j & 15) * groups + g;
            if (READ) {
                const uint2 c = *codes;
                const float s = e4m3_to_float(*scale);
                uint32_t h4[2][4];
                e2m1x8_to_half(c.x, h4[0]);
                e2m1x8_to_half(c.y, h4[1]);
                __align__(16) __nv_bfloat162 v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 f = __half22float2(as_half2(h4[k >> 2][k & 3]));  // f * s is exact: one rounding, by the product with `by`
                    v[k] = __floats2bfloat162_rn(f.x * s * by, f.y * s * by);
                }
                reinterpret_cast<uint4*>(rowp)[0] = reinterpret_cast<const uint4*>(v)[0];
                reinterpret_cast<uint4*>(rowp)[1] = reinterpret_cast<const uint4*>(v)[1];
            } else {
                float x[kFp4Group], amax = 0.f;
                load_group(rowp, by, x);
#pragma unroll
                for (int k = 0; k < kFp4Group; ++k) amax = fmaxf(amax, fabsf(x[k]));  // (fmaxf drops a NaN)
                const uint8_t sb = e4m3_scale(amax);
                const Fp4Thresholds th(e4m3_to_float(sb));
                *codes = make_uint2(e2m1_code8(x, th), e2m1_code8(x + 8, th));
                *scale = sb;
            }
        }
    }
    if (bad_page) atomicOr(p.status, FD_DEV_BAD_PAGE);
}

static int rows_grid(const Fp4RowsParams& p) { return std::max(1, std::min((p.total_rows + kWarps - 1) / kWarps, 8 * p.n_sms)); }

void launch_kv_append_fp4(const Fp4RowsParams& p, cudaStream_t s) { kv_rows_fp4_kernel<false><<<rows_grid(p), kThreads, 0, s>>>(p); }

void launch_kv_read_fp4(const Fp4RowsParams& p, cudaStream_t s) { kv_rows_fp4_kernel<true><<<rows_grid(p), kThreads, 0, s>>>(p); }

}  // namespace fd
