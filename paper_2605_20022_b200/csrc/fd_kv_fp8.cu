// K and V of the query block into the 8-bit cache and out of it.
//
// Append: a warp owns a block -- the 16 tokens of a page, one kv-head, K or V -- because the block's scale needs all of its
// tokens: the new ones from the call's rows and, where the block is begun already, the codes it holds.  Everything is read
// into registers (32 lanes x 8 elements at a time, contiguous on both sides), the largest magnitude goes round the warp, and
// codes and scale go out; codes that were there are written again only if the scale has changed.  No two warps share a block, so
// nothing is ordered by timing.  Read: 16 codes a thread.
// Both: a CTA takes a run of pages (rows) whose sequences and page ids it looks up first, a thread each.
// 24 prompts of 8 heads of 64 (20 k rows) take 13.5 us to append and 14.7 to read back, replayed from a graph (9.6 us of bytes each):
// two thirds of the time is bytes, the rest launch, scan and look-ups.  (Dropped: five or six CTAs an SM for the append 15.6 and 17.0 us; four
// loads in flight a thread for the read 16.2.)  A few rows (64 sequences, 1-16 each): 7.0 and 4.4, a chain of lengths, scan, page
// table, block.
#include <algorithm>

#include "fd_fp8.cuh"
#include "fd_internal.cuh"

namespace fd {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxBatch = 4096;  // what fd_create allows
constexpr int kRun = 64;         // most pages, or rows, of a run

// Does the call leave sequence b out?  (row0: its first row, saturated)
__device__ __forceinline__ bool skipped(const Fp8RowsParams& p, long long n, long long Lq, long long row0) {
    return n < 0 || Lq < 0 || row0 + Lq > p.total_rows || n + Lq > (long long)p.max_pages * 16;
}

// Exclusive scans over the sequences into rows[0 .. B] (negative lengths count as 0) and, for PAGES, into pages[0 .. B] (pages
// that the rows of a sequence reach into; none for a sequence left out).  Sums beyond 32 bits saturate.
template <bool PAGES>
__device__ __forceinline__ void scan_sequences(const Fp8RowsParams& p, int* rows, int* pages, long long (*wsum)[2]) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    long long carry_r = 0, carry_p = 0;
    if (tid == 0) {
        rows[0] = 0;
        if (PAGES) pages[0] = 0;
    }
    for (int base = 0; base < p.batch; base += kThreads) {
        const int b = base + tid;
        const long long Lq = b < p.batch ? p.q_lens[b] : 0, n = PAGES && b < p.batch ? p.prefix_lens[b] : 0;
        long long r = max(Lq, 0LL);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, r, o);
            if (lane >= o) r += u;
        }
        __syncthreads();  // wsum may still be read from the previous round
        if (lane == 31) wsum[warp][0] = r;
        __syncthreads();
        long long before = carry_r;
        for (int k = 0; k < kWarps; ++k) {
            if (k < warp) before += wsum[k][0];
            carry_r += wsum[k][0];
        }
        if (b < p.batch) rows[b + 1] = (int)min(before + r, 0x7fffffffLL);
        if (PAGES) {
            long long w = 0;
            if (Lq > 0 && !skipped(p, n, Lq, before + r - Lq)) w = (n + Lq + 15) / 16 - n / 16;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long u = __shfl_up_sync(0xffffffffu, w, o);
                if (lane >= o) w += u;
            }
            if (lane == 31) wsum[warp][1] = w;
            __syncthreads();
            long long pb = carry_p;
            for (int k = 0; k < kWarps; ++k) {
                if (k < warp) pb += wsum[k][1];
                carry_p += wsum[k][1];
            }
            if (b < p.batch) pages[b + 1] = (int)min(pb + w, 0x7fffffffLL);
        }
    }
    __syncthreads();
}

// The sequence that owns item x: the last b with cu[b] <= x.
__device__ __forceinline__ int owner(const int* cu, int B, int x) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// A sequence that is left out, reported by one CTA.
__device__ __forceinline__ void report_skipped(const Fp8RowsParams& p, const int* rows) {
    if (blockIdx.x != 0) return;
    for (int b = threadIdx.x; b < p.batch; b += kThreads) {
        const long long Lq = p.q_lens[b];
        if (Lq > 0 && skipped(p, p.prefix_lens[b], Lq, rows[b])) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
    }
}

struct PageJob {
    long long at;    // where the page starts in the cache; -1: no page to write
    long long row;   // the row of the call that is the page's token 0 (may lie in front of the sequence's rows)
    int kept, end;   // tokens [0, kept) are there already, [kept, end) are new
};

}  // namespace

template <int D>
__global__ void __launch_bounds__(kThreads, 4) kv_append_fp8_kernel(Fp8RowsParams p, int run) {
    __shared__ int rows[kMaxBatch + 1];
    __shared__ int pages[kMaxBatch + 1];
    __shared__ long long wsum[kWarps][2];
    __shared__ PageJob jobs[kRun];
    constexpr int kUnits = 16 * D / 8 / 32;  // 8-element units of a lane
    constexpr int kPerRow = D / 8;           // ... of a token
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    scan_sequences<true>(p, rows, pages, wsum);
    report_skipped(p, rows);
    const int total = pages[p.batch];
    for (long long j0 = (long long)blockIdx.x * run; j0 < total; j0 += (long long)gridDim.x * run) {
        const int n_jobs = (int)min((long long)run, total - j0);
        __syncthreads();  // the run before has been worked through
        if (tid < n_jobs) {
            const int x = (int)j0 + tid, b = owner(pages, p.batch, x);
            const int n = p.prefix_lens[b], Lq = p.q_lens[b], col = n / 16 + (x - pages[b]);
            PageJob job;
            const int page = p.page_table[(long long)b * p.max_pages + col];
            job.kept = max(0, n - col * 16);
            job.end = min(16, n + Lq - col * 16);
            job.row = (long long)rows[b] - n + col * 16;
            job.at = -1;
            if ((unsigned)page < (unsigned)p.num_pages) job.at = fp8_block_offset(page, p.Hkv, 0, 0, D);  // never form an address from a bad id
            else atomicOr(p.status, FD_DEV_BAD_PAGE);
            jobs[tid] = job;
        }
        __syncthreads();
        const int items = n_jobs * 2 * p.Hkv;
        for (int it = warp; it < items; it += kWarps) {
            const int jb = it / (2 * p.Hkv), hw = it - jb * 2 * p.Hkv, h = hw >> 1, which = hw & 1;
            const PageJob job = jobs[jb];
            if (job.at < 0) continue;
            unsigned char* block = p.kv8 + job.at + (long long)hw * fp8_block_bytes(D);
            const __nv_bfloat16* src = which ? p.v : p.k;
            uint4 raw[kUnits];
            float amax = 0.f, old = 1.f;
            if (job.kept > 0) old = *reinterpret_cast<const float*>(block + 16 * D);
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int u = lane + 32 * i, tok = u / kPerRow, c = u % kPerRow;
                raw[i] = make_uint4(0, 0, 0, 0);
                if (tok >= job.kept && tok < job.end) {
                    raw[i] = *reinterpret_cast<const uint4*>(src + ((job.row + tok) * p.Hkv + h) * D + c * 8);
                } else if (tok < job.kept) {
                    const uint2 w = *reinterpret_cast<const uint2*>(block + tok * D + c * 8);
                    raw[i].x = w.x;
                    raw[i].y = w.y;
                }
            }
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int tok = (lane + 32 * i) / kPerRow;
                if (tok >= job.kept) {  // (a token that is not there is all zeros)
                    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k)  // (fmaxf drops a NaN)
                        amax = fmaxf(amax, fmaxf(fabsf(__uint_as_float(w[k] << 16)), fabsf(__uint_as_float(w[k] & 0xffff0000u))));
                } else {
                    const uint32_t w[2] = {raw[i].x, raw[i].y};
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t a, c;
                        e4m3x4_to_half(w[k], a, c);
                        const float2 fa = __half22float2(as_half2(a)), fc = __half22float2(as_half2(c));
                        const float m = fmaxf(fmaxf(fabsf(fa.x), fabsf(fa.y)), fmaxf(fabsf(fc.x), fabsf(fc.y)));
                        amax = fmaxf(amax, m * old);
                    }
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            const int e = fp8_scale_exp(amax);
            const float scale = exp2_int(e), inv = exp2_int(-e);
            const bool moved = job.kept > 0 && old != scale;
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int u = lane + 32 * i, tok = u / kPerRow, c = u % kPerRow;
                if (tok >= job.end || (tok < job.kept && !moved)) continue;
                uint2 out;
                if (tok >= job.kept) {
                    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                    uint32_t r[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) r[k] = to_e4m3x2(__uint_as_float(w[k] << 16) * inv, __uint_as_float(w[k] & 0xffff0000u) * inv);
                    out = make_uint2(r[0] | r[1] << 16, r[2] | r[3] << 16);
                } else {
                    const float f = old * inv;
                    const uint32_t w[2] = {raw[i].x, raw[i].y};
                    uint32_t r[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t a, d;
                        e4m3x4_to_half(w[k], a, d);
                        const float2 fa = __half22float2(as_half2(a)), fd_ = __half22float2(as_half2(d));
                        r[k] = to_e4m3x2(fa.x * f, fa.y * f) | to_e4m3x2(fd_.x * f, fd_.y * f) << 16;
                    }
                    out = make_uint2(r[0], r[1]);
                }
                *reinterpret_cast<uint2*>(block + tok * D + c * 8) = out;
            }
            if (lane == 0) *reinterpret_cast<uint4*>(block + 16 * D) = make_uint4(__float_as_uint(scale), 0, 0, 0);
        }
    }
}

__global__ void __launch_bounds__(kThreads, 4) kv_read_fp8_kernel(Fp8RowsParams p, int run) {
    __shared__ int rows[kMaxBatch + 1];
    __shared__ long long wsum[kWarps][2];
    __shared__ long long s_page[kRun];  // where the row's page starts in the cache; -1: no page to read
    __shared__ int s_tok[kRun];         // its token there
    const int tid = threadIdx.x;
    scan_sequences<false>(p, rows, nullptr, wsum);
    report_skipped(p, rows);
    const int g_shift = p.d == 64 ? 2 : 3, per_head = 1 << g_shift;  // 16-element groups of a head
    const int per_row = 2 * p.Hkv * per_head, block = fp8_block_bytes(p.d);
    const long long total = min(rows[p.batch], p.total_rows);
    for (long long r0 = (long long)blockIdx.x * run; r0 < total; r0 += (long long)gridDim.x * run) {
        const int n_rows = (int)min((long long)run, total - r0);
        __syncthreads();  // the run before has been worked through
        if (tid < n_rows) {
            const int row = (int)(r0 + tid), b = owner(rows, p.batch, row);
            const int n = p.prefix_lens[b], Lq = p.q_lens[b];
            long long at = -1;
            int tok = 0;
            if (!skipped(p, n, Lq, rows[b])) {
                const int j = n + row - rows[b], page = p.page_table[(long long)b * p.max_pages + (j >> 4)];
                tok = j & 15;
                if ((unsigned)page < (unsigned)p.num_pages) at = fp8_block_offset(page, p.Hkv, 0, 0, p.d);
                else atomicOr(p.status, FD_DEV_BAD_PAGE);
            }
            s_page[tid] = at;
            s_tok[tid] = tok;
        }
        __syncthreads();
        // a row's groups: head, K or V, group; a thread walks the run's with a stride, keeping row and group apart without a division
        int i = tid / per_row, g = tid - i * per_row;
        const int di = kThreads / per_row, dg = kThreads - di * per_row;
        for (; i < n_rows; i += di, g += dg) {
            if (g >= per_row) { g -= per_row; ++i; if (i >= n_rows) break; }
            const int hw = g >> g_shift, e = (g & (per_head - 1)) * 16, h = hw >> 1;
            const long long at = s_page[i];
            uint4 w = make_uint4(0, 0, 0, 0);
            float scale = 0.f;
            if (at >= 0) {
                const unsigned char* b = p.kv8 + at + (long long)hw * block;
                w = *reinterpret_cast<const uint4*>(b + s_tok[i] * p.d + e);
                scale = *reinterpret_cast<const float*>(b + 16 * p.d);
            }
            const uint32_t in[4] = {w.x, w.y, w.z, w.w};
            __align__(16) __nv_bfloat162 v[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t a, c;
                e4m3x4_to_half(in[k], a, c);
                const float2 fa = __half22float2(as_half2(a)), fc = __half22float2(as_half2(c));
                v[2 * k] = __floats2bfloat162_rn(fa.x * scale, fa.y * scale);  // (exact: four significant bits)
                v[2 * k + 1] = __floats2bfloat162_rn(fc.x * scale, fc.y * scale);
            }
            __nv_bfloat16* dst = ((hw & 1) ? p.v : p.k) + ((r0 + i) * p.Hkv + h) * p.d + e;
            reinterpret_cast<uint4*>(dst)[0] = reinterpret_cast<const uint4*>(v)[0];
            reinterpret_cast<uint4*>(dst)[1] = reinterpret_cast<const uint4*>(v)[1];
        }
    }
}

void launch_kv_append_fp8(const Fp8RowsParams& p, cudaStream_t s) {
    // pages that the rows can reach into, at most: every row may start one, and 16 rows of a sequence at least end one
    const long long most = std::min<long long>(p.total_rows, p.total_rows / 16 + 2LL * p.batch), resident = 4LL * p.n_sms;
    // a run: a page at a time while there are CTAs left for each, so that a page's 2 Hkv blocks go to the warps of one CTA
    const int run = (int)std::max(1LL, std::min<long long>(kRun, (most + resident - 1) / resident));
    const int grid = (int)std::max(1LL, std::min((most + run - 1) / run, resident));
    if (p.d == 64) kv_append_fp8_kernel<64><<<grid, kThreads, 0, s>>>(p, run);
    else kv_append_fp8_kernel<128><<<grid, kThreads, 0, s>>>(p, run);
}

void launch_kv_read_fp8(const Fp8RowsParams& p, cudaStream_t s) {
    const long long resident = 4LL * p.n_sms;
    const int run = (int)std::max(1LL, std::min<long long>(kRun, (p.total_rows + resident - 1) / resident));
    const int grid = (int)std::max(1LL, std::min((p.total_rows + run - 1LL) / run, resident));
    kv_read_fp8_kernel<<<grid, kThreads, 0, s>>>(p, run);
}

}  // namespace fd
