// K and V of the query block into the 4-bit cache and out of it.
//
// A thread owns one scale group: 16 elements, 32 bytes of bf16 on one side, 8 bytes of codes and a scale byte on the other.
// Neighbouring threads own neighbouring groups of a row, so both sides are contiguous across a warp.  A CTA takes a run of
// rows: first a thread per row finds the row's sequence and page (a search and a dependent load), then all threads stream
// the run's groups with nothing but loads and stores between them.
// 24 prompts of 8 heads of 64 (20 k rows, 41 MB in) take 21 us to append and 17 us to read back, calls replayed from a graph (7.7 us
// of bytes each).  The warps wait for their loads: half of the issue slots are used in the append, two fifths in the read.  One
// behind the other through the Python entry points the two take 42 us; with the look-up made for every group they took 53.
// A few rows (64 sequences, 1-16 each) are launch latency and the look-up: 5.8 and 4.2 us.
#include <algorithm>

#include "fd_fp4.cuh"
#include "fd_internal.cuh"

namespace fd {

namespace {

constexpr int kThreads = 256;

constexpr int kWarps = kThreads / 32;
constexpr int kMaxBatch = 4096;  // what fd_create allows
constexpr int kRun = 64;         // most rows of a run

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

}  // namespace

template <bool READ>
__global__ void __launch_bounds__(kThreads, READ ? 4 : 3) kv_rows_fp4_kernel(Fp4RowsParams p, int run, unsigned per_row_inv) {
    __shared__ int cu[kMaxBatch + 1];
    __shared__ long long wsum[kWarps];
    __shared__ long long s_page[kRun];  // where the row's page starts in the cache; -1: no page to read or write
    __shared__ int s_tok[kRun];         // its token there
    const int tid = threadIdx.x;
    scan_lengths(p.q_lens, p.batch, cu, wsum);
    const int g_shift = p.d == 64 ? 2 : 3, per_row = p.Hkv << g_shift;  // groups of K, and again of V
    const int page_bytes = fp4_page_bytes(p.d);
    const long long rows = min(cu[p.batch], p.total_rows);
    if (blockIdx.x == 0)  // a sequence that is skipped: the status alone (its rows are met below, by whoever owns them)
        for (int b = tid; b < p.batch; b += kThreads) {
            const long long n = p.prefix_lens[b], Lq = p.q_lens[b];
            if (Lq > 0 && (n < 0 || cu[b] + Lq > p.total_rows || n + Lq > (long long)p.max_pages * 16)) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
        }
    const Fp4Quantiser by_k(p.k_scale), by_v(p.v_scale);
    for (long long r0 = (long long)blockIdx.x * run; r0 < rows; r0 += (long long)gridDim.x * run) {
        const int n_rows = (int)min((long long)run, rows - r0);
        __syncthreads();  // the run before has been worked through
        if (tid < n_rows) {
            const long long row = r0 + tid;
            int lo = 0, hi = p.batch;  // the sequence that owns the row: the last one that starts at or before it
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (cu[mid] <= row) lo = mid; else hi = mid;
            }
            const int n = p.prefix_lens[lo], Lq = p.q_lens[lo];
            long long at = -1;
            int tok = 0;
            if (n >= 0 && (long long)cu[lo] + Lq <= p.total_rows && (long long)n + Lq <= (long long)p.max_pages * 16) {
                const int j = n + (int)(row - cu[lo]);
                const int page = p.page_table[(long long)lo * p.max_pages + (j >> 4)];
                tok = j & 15;
                if ((unsigned)page < (unsigned)p.num_pages) at = fp4_page_offset(page, p.Hkv, 0, 0, p.d);  // never form an address from a bad id
                else atomicOr(p.status, FD_DEV_BAD_PAGE);
            }
            s_page[tid] = at;
            s_tok[tid] = tok;
        }
        __syncthreads();
        const int items = n_rows * 2 * per_row;
        auto locate = [&](int e, bool& ok, int& which, __nv_bfloat16*& rowp, unsigned char*& codes, unsigned char*& scale) {
            const int i = (int)__umulhi((unsigned)e, per_row_inv), rem = e - i * 2 * per_row;  // row of the run, group of the row
            which = rem >= per_row;
            const int hg = rem - which * per_row, h = hg >> g_shift, g = hg & ((1 << g_shift) - 1);
            const long long at = s_page[i];
            const int tok = s_tok[i];
            ok = at >= 0;
            rowp = (which ? p.v : p.k) + ((r0 + i) * per_row + hg) * kFp4Group;
            unsigned char* base = p.kv4 + at + (h * 2 + which) * page_bytes;
            codes = base + tok * (p.d / 2) + g * 8;
            scale = base + fp4_scale_offset(p.d) + (tok << g_shift) + g;
        };
        constexpr int U = READ ? 4 : 2;  // items in flight per thread
        for (int e0 = tid; e0 < items; e0 += U * kThreads) {
            bool ok[U];
            int which[U];
            __nv_bfloat16* rowp[U];
            unsigned char *codes[U], *scale[U];
            uint4 raw[U][READ ? 1 : 2];
            unsigned char sb[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = min(e0 + u * kThreads, items - 1);  // (past the end: the last item again)
                locate(e, ok[u], which[u], rowp[u], codes[u], scale[u]);
                if (READ) {
                    raw[u][0] = make_uint4(0, 0, 0, 0);
                    sb[u] = 0;
                    if (ok[u]) {
                        const uint2 c = *reinterpret_cast<const uint2*>(codes[u]);
                        raw[u][0].x = c.x; raw[u][0].y = c.y;
                        sb[u] = *scale[u];
                    }
                } else if (ok[u]) {
                    raw[u][0] = reinterpret_cast<const uint4*>(rowp[u])[0];
                    raw[u][READ ? 0 : 1] = reinterpret_cast<const uint4*>(rowp[u])[1];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (e0 + u * kThreads >= items) break;
                if (READ) {  // (no page: codes and scale of zero)
                    const float m = which[u] ? by_v.by : by_k.by;
                    const __half2 f = __half2half2(__low2half(as_half2(e4m3x2_to_half(sb[u]))));
                    uint32_t h4[2][4];
                    e2m1x8_to_half(raw[u][0].x, h4[0]);
                    e2m1x8_to_half(raw[u][0].y, h4[1]);
                    __align__(16) __nv_bfloat162 v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float2 c = __half22float2(__hmul2(as_half2(h4[k >> 2][k & 3]), f));  // code * scale is exact in fp16
                        v[k] = __floats2bfloat162_rn(c.x * m, c.y * m);
                    }
                    reinterpret_cast<uint4*>(rowp[u])[0] = reinterpret_cast<const uint4*>(v)[0];
                    reinterpret_cast<uint4*>(rowp[u])[1] = reinterpret_cast<const uint4*>(v)[1];
                } else if (ok[u]) {
                    float x[kFp4Group], amax = 0.f;
                    const __nv_bfloat162* e2 = reinterpret_cast<const __nv_bfloat162*>(raw[u]);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float2 f = __bfloat1622float2(e2[k]);
                        x[2 * k] = f.x;
                        x[2 * k + 1] = f.y;
                    }
                    Fp4Quantiser by = by_k;
                    if (which[u]) by = by_v;
#pragma unroll
                    for (int k = 0; k < kFp4Group; ++k) amax = max_nan(amax, fabsf(x[k]));
                    Fp4Scale g;
                    uint2 w;
                    if (!by.odd(amax)) {
                        g = by.scale(amax);
                        w = make_uint2(by.codes<8>(x, g), by.codes<8>(x + 8, g));
                    } else {
                        amax = 0.f;
#pragma unroll
                        for (int k = 0; k < kFp4Group; ++k) amax = fmaxf(amax, fabsf(x[k]));  // (drops a NaN)
                        g = by.scale_long(amax);
                        w = make_uint2(by.codes_long<8>(x, g), by.codes_long<8>(x + 8, g));
                    }
                    *reinterpret_cast<uint2*>(codes[u]) = w;
                    *scale[u] = g.byte;
                }
            }
        }
    }
}

// A run is short enough for every SM to have some, and long enough for its look-ups to be few.
template <bool READ>
static void launch_rows(const Fp4RowsParams& p, cudaStream_t s) {
    // The kernel takes floor(e / per_row), e < run * per_row, as the high half of a product with the reciprocal rounded up.  Before
    // it is cut off that is too large by at most e / 2^32, and e / per_row is at least 1 / per_row below the next whole number: exact
    // while run * per_row^2 < 2^32.  Longer rows (from 512 kv-heads of 128 on) get shorter runs; where a run is one row the quotient
    // is 0, and so is the product with a reciprocal of 0.
    const long long per_row = 2LL * p.Hkv * (p.d / kFp4Group), exact = 0xffffffffLL / (per_row * per_row);
    const long long resident = 4LL * p.n_sms, wanted = std::min<long long>(kRun, (p.total_rows + resident - 1) / resident);
    const int run = (int)std::max(1LL, std::min(wanted, exact));
    const int grid = (int)std::max(1LL, std::min((p.total_rows + run - 1LL) / run, resident));
    kv_rows_fp4_kernel<READ><<<grid, kThreads, 0, s>>>(p, run, run == 1 ? 0u : (unsigned)(0xffffffffLL / per_row + 1));
}

void launch_kv_append_fp4(const Fp4RowsParams& p, cudaStream_t s) { launch_rows<false>(p, s); }

void launch_kv_read_fp4(const Fp4RowsParams& p, cudaStream_t s) { launch_rows<true>(p, s); }

}  // namespace fd
