// Page reservation: pages for the query blocks out of a free list, and the cache slot and the position of every query row.
//
// Everything follows from the lengths by two scans over the sequences (rows, pages needed), so every CTA makes the scans
// for itself in shared memory and then works on its own share of the rows: no CTA depends on another, and one launch
// does for one row as for a million.  The row that opens a page (position a multiple of 16) writes the page's table entry.
// Only the counter of the free list is written by the CTA that finishes last: the caller may pass the same word for the
// count before and after, so nobody may write it while others still read it.
// Bound by its launch and the chain of the scans: 3.8 us for one sequence, 5.4 for 64, 6.1 for 256 prompts of 530 k rows
// (floor 0.8: 8 bytes a row), calls replayed from a graph.
#include <algorithm>

#include "fd_internal.cuh"

namespace fd {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxBatch = 4096;  // what fd_create allows

struct ReserveSmem {
    int rows[kMaxBatch + 1];  // exclusive scan of the query rows
    int need[kMaxBatch + 1];  // exclusive scan of the pages needed
};

}  // namespace

__global__ void __launch_bounds__(kThreads) reserve_kernel(ReserveParams p) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    ReserveSmem& sc = *reinterpret_cast<ReserveSmem*>(smem_raw);
    __shared__ long long wsum[kWarps][2];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.batch;
    if (tid == 0) { sc.rows[0] = 0; sc.need[0] = 0; }
    const int n_free = *p.n_free, n_freed = p.n_freed ? *p.n_freed : 0;
    bool bad = n_free < 0 || n_freed < 0 || (long long)n_free + n_freed > p.num_pages;
    // ---- the two scans, 256 sequences at a time
    long long rows0 = 0, need0 = 0;
    for (int base = 0; base < B; base += kThreads) {
        const int b = base + tid;
        long long r = 0, w = 0;
        if (b < B) {
            const long long n = p.prefix_lens[b], L = p.q_lens[b], M = p.n_mask[b], nb = p.n_blocks ? p.n_blocks[b] : 1;
            if (n < 0 || L < 0 || M < 0 || M > L || L > p.max_q_len || n + L > (long long)p.max_pages * 16 || nb < 0 ||
                (nb > 1 && (M % nb != 0 || nb > L - M))) {
                bad = true;
            } else {
                r = L;
                w = (n + L + 15) / 16 - (n + 15) / 16;
            }
        }
        long long ir = r, iw = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long ur = __shfl_up_sync(0xffffffffu, ir, o), uw = __shfl_up_sync(0xffffffffu, iw, o);
            if (lane >= o) { ir += ur; iw += uw; }
        }
        __syncthreads();  // wsum may still be read from the previous round
        if (lane == 31) { wsum[warp][0] = ir; wsum[warp][1] = iw; }
        __syncthreads();
        long long orow = rows0, oneed = need0;
        for (int k = 0; k < kWarps; ++k) {
            if (k < warp) { orow += wsum[k][0]; oneed += wsum[k][1]; }
            rows0 += wsum[k][0];
            need0 += wsum[k][1];
        }
        if (b < B) {  // (a total beyond 32 bits cannot match total_rows: the call is refused below)
            sc.rows[b + 1] = (int)min(orow + ir, 0x7fffffffLL);
            sc.need[b + 1] = (int)min(oneed + iw, 0x7fffffffLL);
        }
    }
    bad = __syncthreads_or(bad) != 0 || rows0 != p.total_rows;
    const int top = bad ? n_free : n_free + n_freed;      // ids on the list once the released ones are pushed
    const bool shorted = !bad && need0 > top;
    const int left = bad || shorted ? top : top - (int)need0;  // ... and after the call
    // an id of the list at place i, whether it has been pushed to the array yet or not
    auto list_at = [&](int i) { return i < n_free ? p.free_pages[i] : p.freed[i - n_free]; };
    bool bad_page = false;

    // ---- rows, four in a row per thread: one search, 16-byte stores
    const long long stride = (long long)gridDim.x * kThreads;
    const bool wide = ((reinterpret_cast<uintptr_t>(p.slot_map) | reinterpret_cast<uintptr_t>(p.positions)) & 15) == 0;
    for (long long row0 = 4 * ((long long)blockIdx.x * kThreads + tid); row0 < p.total_rows; row0 += 4 * stride) {
        int slot[4] = {-1, -1, -1, -1}, position[4] = {-1, -1, -1, -1};
        const int count = (int)min(4LL, p.total_rows - row0);
        if (!bad) {
            int lo = 0, hi = B;  // the sequence that owns the first row: the last one that starts at or before it
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (sc.rows[mid] <= row0) lo = mid; else hi = mid;
            }
            int b = lo - 1, n = 0, C = 0, M = 0, first = 0, last_page = -1, id = -1, end = 0, start = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k >= count) break;
                const int row = (int)(row0 + k);
                if (k == 0 || row >= end) {  // on to the sequence of this row (past empty ones)
                    do ++b; while (sc.rows[b + 1] <= row);
                    start = sc.rows[b];
                    end = sc.rows[b + 1];
                    n = p.prefix_lens[b];
                    M = p.n_mask[b];
                    C = end - start - M;
                    first = (n + 15) >> 4;
                    last_page = -1;
                }
                const int i = row - start, pos = n + i, page = pos >> 4;
                position[k] = pos;
                if (i >= C) {
                    const int nb = p.n_blocks ? max(p.n_blocks[b], 1) : 1, each = M / nb;
                    const int g = (i - C) / each, u = (i - C) - g * each;
                    position[k] = n + (C - nb + g) + 1 + u;
                }
                if (!shorted) {
                    int32_t* entry = p.page_table + (long long)b * p.max_pages + page;
                    if (page != last_page) {
                        last_page = page;
                        id = page >= first ? list_at(top - 1 - (sc.need[b] + page - first)) : *entry;
                        if ((unsigned)id >= (unsigned)p.num_pages) { bad_page = true; id = -1; }
                    }
                    if (page >= first && (pos & 15) == 0) *entry = id;
                    if (id >= 0) slot[k] = id * 16 + (pos & 15);
                }
            }
        }
        if (wide && count == 4) {
            *reinterpret_cast<int4*>(p.slot_map + row0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
            *reinterpret_cast<int4*>(p.positions + row0) = make_int4(position[0], position[1], position[2], position[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < count) { p.slot_map[row0 + k] = slot[k]; p.positions[row0 + k] = position[k]; }
        }
    }
    // ---- released ids that stay on the list (the others have been handed out from where the commit wrote them)
    if (!bad)
        for (long long i = (long long)blockIdx.x * kThreads + tid; i < n_freed && n_free + i < left; i += stride)
            p.free_pages[n_free + i] = p.freed[i];
    if (bad_page) atomicOr(p.status, FD_DEV_BAD_PAGE);
    if (blockIdx.x == 0 && tid == 0) {
        if (bad) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
        if (shorted) atomicOr(p.status, FD_DEV_NO_PAGES);
    }
    if (gridDim.x == 1) {
        if (tid == 0) *p.n_free_out = left;  // (every thread read the count before the barriers above)
        return;
    }
    __syncthreads();
    if (tid == 0) {
        s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
        if (s_last) {
            *p.ticket = 0;
            *p.n_free_out = left;
        }
    }
}

void launch_reserve(const ReserveParams& p, cudaStream_t s) {
    const long long work = (p.total_rows + 4 * kThreads - 1) / (4 * kThreads);
    const int grid = (int)std::max<long long>(1, std::min<long long>(work, 4LL * p.n_sms));
    reserve_kernel<<<grid, kThreads, sizeof(ReserveSmem), s>>>(p);
}

}  // namespace fd
