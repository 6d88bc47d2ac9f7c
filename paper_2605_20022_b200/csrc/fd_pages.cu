// The pages of a pool when sequences branch, end, and when the pool is compacted.
//
// A page is shared when several sequences name it: shared[id] counts its owners beyond the first, so pages that were never forked
// (and free ones) hold 0 and neither the reservation nor the commit, which touch a sequence's own last pages only, need to
// know of it.
//
// fork     every CTA makes the scan over the forks (which of them needs a page) for itself and copies its share of the table
//          entries: one launch, no CTA waits for another.  512 samples of 256 pages each 6.8 us, one sample 3.6.
// free     which occurrence of a shared page releases it must not depend on timing, so it takes passes over the occurrences with
//          barriers between them: count owners down, let a page without owners be claimed by its first occurrence, count the
//          claims, write the list.  Few pages: one CTA, one launch, 7 us for 64.  Many: a launch for each pass, 19 us for 131 k
//          -- bound by the random words of `shared`, an atomic for each page owned and three reads (one cluster of eight CTAs, with its
//          hardware barrier between the passes, took 98).
// compact  mark, count and rank, list the moves: passes over the ids, a thread-block cluster with its barrier between them, since they
//          are few; the tables follow in a launch over all SMs (24 k ids and 82 k table entries: 21 us the two).
// copy     16-byte words, four in flight a thread: 6400 pages of 33 KB in 72 us, 88 % of the measured copy bandwidth.
#include <algorithm>

#include "fd_fp8.cuh"
#include "fd_internal.cuh"
#include "fd_sm100.cuh"

namespace fd {

using namespace sm100;

namespace {

constexpr int kMaxBatch = 4096;  // what fd_create allows

// Exclusive prefix of v over the block's threads; *total their sum.  s: one int per warp.  All threads.
template <int THREADS>
__device__ __forceinline__ int block_scan(int v, int* s, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += u;
    }
    __syncthreads();  // s may still be read from the scan before
    if (lane == 31) s[warp] = inc;
    __syncthreads();
    int w = lane < THREADS / 32 ? s[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += u;
    }
    *total = __shfl_sync(0xffffffffu, w, THREADS / 32 - 1);
    const int before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    return inc - v + (warp ? before : 0);
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {  // every thread of every CTA; orders their global accesses too
    __threadfence();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The word at `p` in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ int peer_int(const int* p, uint32_t rank) {
    uint32_t a;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

}  // namespace

// ------------------------------------------------------------------------------------------------ fork
constexpr int kForkThreads = 256;

__global__ void __launch_bounds__(kForkThreads) fork_kernel(ForkParams p) {
    __shared__ int rank[kMaxBatch];        // free pages popped before this fork's
    __shared__ unsigned seen[kMaxBatch / 32], is_parent[kMaxBatch / 32];
    __shared__ int wsum[kForkThreads / 32];
    __shared__ int s_last;
    const int tid = threadIdx.x, N = p.n_forks;
    for (int i = tid; i < kMaxBatch / 32; i += kForkThreads) seen[i] = is_parent[i] = 0;
    __syncthreads();
    const int n_free = *p.n_free;
    bool bad = n_free < 0 || n_free > p.num_pages;
    int popped = 0;
    for (int base = 0; base < N; base += kForkThreads) {
        const int i = base + tid;
        int need = 0;
        if (i < N) {
            const int s = p.parents[i], t = p.children[i];
            if ((unsigned)s >= (unsigned)p.batch || (unsigned)t >= (unsigned)p.batch) {
                bad = true;
            } else {
                const int n = p.prefix_lens[s];
                if (n < 0 || (long long)n > (long long)p.max_pages * 16) bad = true;
                else need = (n & 15) != 0;
                atomicOr(&is_parent[s >> 5], 1u << (s & 31));
                if (atomicOr(&seen[t >> 5], 1u << (t & 31)) >> (t & 31) & 1u) bad = true;  // one child, two parents
            }
        }
        int sum;
        const int before = block_scan<kForkThreads>(need, wsum, &sum);
        if (i < N) rank[i] = popped + before;
        popped += sum;
    }
    __syncthreads();
    for (int i = tid; i < kMaxBatch / 32; i += kForkThreads)
        if (seen[i] & is_parent[i]) bad = true;  // (its length would be read and written in one call)
    bad = __syncthreads_or(bad) != 0;
    const bool shorted = !bad && popped > n_free;
    bool bad_page = false;
    const long long stride = (long long)gridDim.x * kForkThreads, first = (long long)blockIdx.x * kForkThreads + tid;
    if (bad || shorted) {
        for (long long i = first; i < N; i += stride) p.copy_src[i] = p.copy_dst[i] = -1;
    } else {
        // a warp a piece of a child's row: 32 entries at a time
        const int lane = tid & 31, pieces = (p.max_pages + 31) >> 5;
        const long long tasks = (long long)N * pieces;
        for (long long w = first >> 5; w < tasks; w += stride >> 5) {
            const int i = (int)(w / pieces), col = (int)(w - (long long)i * pieces) * 32 + lane;
            const int s = p.parents[i], t = p.children[i], n = p.prefix_lens[s], full = n >> 4;
            const int32_t* from = p.page_table + (long long)s * p.max_pages;
            if (col < p.max_pages) {
                int id = -1;
                if (col < full) {
                    id = from[col];
                    if ((unsigned)id < (unsigned)p.num_pages) atomicAdd(p.shared + id, 1);
                    else { id = -1; bad_page = true; }
                } else if (col == full && (n & 15)) {
                    id = p.free_pages[n_free - 1 - rank[i]];
                    int src = from[col];
                    if ((unsigned)id >= (unsigned)p.num_pages) { id = -1; bad_page = true; }
                    if ((unsigned)src >= (unsigned)p.num_pages) { src = -1; bad_page = true; }
                    p.copy_src[i] = id < 0 ? -1 : src;
                    p.copy_dst[i] = src < 0 ? -1 : id;
                }
                p.page_table[(long long)t * p.max_pages + col] = id;
            }
            if (col == 0) {
                p.prefix_lens[t] = n;
                if ((n & 15) == 0) p.copy_src[i] = p.copy_dst[i] = -1;
            }
        }
    }
    if (bad_page) atomicOr(p.status, FD_DEV_BAD_PAGE);
    if (blockIdx.x == 0 && tid == 0) {
        if (bad) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
        if (shorted) atomicOr(p.status, FD_DEV_NO_PAGES);
    }
    // the count is written by whoever finishes last: it may be the very word the others read
    __syncthreads();
    if (tid == 0) {
        s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
        if (s_last) {
            *p.ticket = 0;
            *p.n_free_out = bad || shorted ? n_free : n_free - popped;
        }
    }
}

void launch_kv_fork(const ForkParams& p, cudaStream_t s) {
    const long long work = ((long long)p.n_forks * ((p.max_pages + 31) / 32) + kForkThreads / 32 - 1) / (kForkThreads / 32);
    const int grid = (int)std::max<long long>(1, std::min<long long>(work, 4LL * p.n_sms));
    fork_kernel<<<grid, kForkThreads, 0, s>>>(p);
}

// ------------------------------------------------------------------------------------------------ free
// The occurrences of pages in the listed sequences, numbered e = 0 .. T - 1 (sequence by sequence, page by page); a warp takes a
// contiguous run of them.
constexpr int kFreeThreads = 512, kFreeSmallThreads = 1024;  // (one CTA alone: more loads in flight)
// Entries of the listed sequences' rows up to which one CTA does it in one launch (the lengths are on the device: what the sequences hold
// is not known here).  One CTA / four launches, random ids with one owner each, in a graph behind the copies that restore the books:
// 64 pages held of 64 entries 7.0 / 11.5 us, 1024 of 1024 8.2 / 14.4, 2048 of 4096 14.1 / 17.1, 4096 of 4096 21.6 / 23.1;
// 2048 of 8192 14.1 / 13.3, 4096 of 8192 22.1 / 18.1, 8192 of 8192 35.7 / 24.1.  (56 pages of 8 sequences with rows of 2048 entries take
// four launches: 12.)
constexpr long long kFreeSmall = 4096;
constexpr int kClaim = 0x40000000;  // a released page holds e - T - 1 - kClaim once occurrence e (of T) has claimed it: below any count

struct FreeShared {
    int cu[kMaxBatch + 1];  // exclusive scan of the pages of the listed sequences
    unsigned seen[kMaxBatch / 32];
    int wsum[32];
};

// Checks and scan.  Returns whether the call is to be refused (the same in every thread).
template <int THREADS>
__device__ __forceinline__ bool free_scan(const FreeParams& p, FreeShared& sh, int n_free, int* T) {
    const int tid = threadIdx.x, N = p.n_seqs;
    for (int i = tid; i < kMaxBatch / 32; i += THREADS) sh.seen[i] = 0;
    if (tid == 0) sh.cu[0] = 0;
    __syncthreads();
    bool bad = n_free < 0 || n_free > p.num_pages;
    long long total = 0;
    for (int base = 0; base < N; base += THREADS) {
        const int i = base + tid;
        int pages = 0;
        if (i < N) {
            const int b = p.seqs[i];
            if ((unsigned)b >= (unsigned)p.batch) {
                bad = true;
            } else {
                const int n = p.prefix_lens[b];
                if (n < 0 || (long long)n > (long long)p.max_pages * 16) bad = true;
                else pages = (n + 15) >> 4;
                if (atomicOr(&sh.seen[b >> 5], 1u << (b & 31)) >> (b & 31) & 1u) bad = true;  // listed twice
            }
        }
        if (pages > 0x1fffff) bad = true;  // (1024 of them must not pass 32 bits)
        pages = min(pages, 0x1fffff);
        int sum;
        const int before = block_scan<THREADS>(pages, sh.wsum, &sum);
        if (i < N) sh.cu[i + 1] = (int)min(total + before + pages, 0x3fffffffLL);
        total += sum;
    }
    *T = (int)min(total, 0x3fffffffLL);
    return __syncthreads_or(bad) != 0 || total >= kClaim / 2;
}

// f(e, entry, id) for this lane's occurrences of [lo, hi), ascending, four page ids in flight; ids outside the pool are passed on.
template <class F>
__device__ __forceinline__ void each_occurrence(const FreeParams& p, const FreeShared& sh, int lo, int hi, F f) {
    const int lane = threadIdx.x & 31;
    if (lo >= hi) return;
    int a = 0, z = p.n_seqs;  // the sequence that holds occurrence lo
    while (z - a > 1) {
        const int mid = (a + z) >> 1;
        if (sh.cu[mid] <= lo) a = mid; else z = mid;
    }
    int32_t* row = p.page_table + (long long)p.seqs[a] * p.max_pages;
    for (int base = lo; base < hi; base += 128) {
        int32_t* entry[4];
        int id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = base + u * 32 + lane;
            entry[u] = nullptr;
            id[u] = -1;
            if (e < hi) {
                if (e >= sh.cu[a + 1]) {
                    do ++a; while (e >= sh.cu[a + 1]);
                    row = p.page_table + (long long)p.seqs[a] * p.max_pages;
                }
                entry[u] = row + (e - sh.cu[a]);
                id[u] = *entry[u];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) f(base + u * 32 + lane, entry[u], id[u]);  // (entry nullptr: beyond the end; whole warps call)
    }
}

// Owners go.
__device__ __forceinline__ bool free_count_down(const FreeParams& p, const FreeShared& sh, int lo, int hi) {
    bool bad_page = false;
    each_occurrence(p, sh, lo, hi, [&](int, int32_t* entry, int id) {
        if (!entry) return;
        if ((unsigned)id >= (unsigned)p.num_pages || atomicSub(p.shared + id, 1) < 0) bad_page = true;  // (below 0: more owners than it has)
    });
    return bad_page;
}
// A page without owners goes to the list at its first occurrence.
__device__ __forceinline__ void free_claim(const FreeParams& p, const FreeShared& sh, int T, int lo, int hi) {
    each_occurrence(p, sh, lo, hi, [&](int e, int32_t* entry, int id) {
        if (entry && (unsigned)id < (unsigned)p.num_pages && __ldcg(p.shared + id) < 0) atomicMin(p.shared + id, e - T - 1 - kClaim);
    });
}
__device__ __forceinline__ bool free_claimed(const FreeParams& p, int T, int e, int32_t* entry, int id) {
    return entry && (unsigned)id < (unsigned)p.num_pages && __ldcg(p.shared + id) == e - T - 1 - kClaim;
}
__device__ __forceinline__ int free_claims(const FreeParams& p, const FreeShared& sh, int T, int lo, int hi) {  // of the warp's run, in every lane
    int n = 0;
    each_occurrence(p, sh, lo, hi, [&](int e, int32_t* entry, int id) { n += free_claimed(p, T, e, entry, id); });
    return __reduce_add_sync(0xffffffffu, n);
}
// The list: the last occurrence first, `end` the place behind the warp's run's.
__device__ __forceinline__ bool free_push(const FreeParams& p, const FreeShared& sh, int T, int lo, int hi, int end) {
    bool bad_page = false;
    each_occurrence(p, sh, lo, hi, [&](int e, int32_t* entry, int id) {
        const bool push = free_claimed(p, T, e, entry, id);
        const unsigned who = __ballot_sync(0xffffffffu, push);
        if (entry) *entry = -1;
        if (push) {
            const int at = end - 1 - __popc(who & ((1u << (threadIdx.x & 31)) - 1u));
            p.shared[id] = 0;  // (no other occurrence's claim: theirs compare unequal to this as well)
            if (at < p.num_pages) p.free_pages[at] = id;
            else bad_page = true;
        }
        end -= __popc(who);
    });
    return bad_page;
}
__device__ __forceinline__ void run_of(int warp, int warps, int T, int* lo, int* hi) {
    const int per = ((T + warps - 1) / warps + 31) & ~31;
    *lo = (int)min((long long)warp * per, (long long)T);
    *hi = (int)min((long long)*lo + per, (long long)T);
}

// Few pages: one CTA, one launch.
__global__ void __launch_bounds__(kFreeSmallThreads) free_small_kernel(FreeParams p) {
    __shared__ FreeShared sh;
    const int tid = threadIdx.x, warp = tid >> 5, n_free = *p.n_free;
    int T, lo, hi, all;
    if (free_scan<kFreeSmallThreads>(p, sh, n_free, &T)) {
        if (tid == 0) {
            atomicOr(p.status, FD_DEV_BAD_LENGTHS);
            *p.n_free_out = n_free;
        }
        return;
    }
    run_of(warp, kFreeSmallThreads / 32, T, &lo, &hi);
    bool bad_page = free_count_down(p, sh, lo, hi);
    __syncthreads();
    free_claim(p, sh, T, lo, hi);
    __syncthreads();
    const int mine = free_claims(p, sh, T, lo, hi);
    const int before = block_scan<kFreeSmallThreads>((tid & 31) == 0 ? mine : 0, sh.wsum, &all);
    // the warps behind this one push first: the run ends where theirs and its own have been pushed
    bad_page |= free_push(p, sh, T, lo, hi, n_free + all - __shfl_sync(0xffffffffu, before, 0));
    if (bad_page) atomicOr(p.status, FD_DEV_BAD_PAGE);
    for (int i = tid; i < p.n_seqs; i += kFreeSmallThreads) p.prefix_lens[p.seqs[i]] = 0;
    if (tid == 0) *p.n_free_out = min(n_free + all, p.num_pages);
}

// Many: a launch for each pass, the scan handed on through scratch (the last pass clears the lengths it was made from).
template <int PASS>
__global__ void __launch_bounds__(kFreeThreads) free_pass_kernel(FreeParams p) {
    __shared__ FreeShared sh;
    const int tid = threadIdx.x, warp = tid >> 5, N = p.n_seqs;
    constexpr int W = kFreeThreads / 32;
    int T, n_free;
    bool bad;
    if (PASS == 0) {
        n_free = *p.n_free;
        bad = free_scan<kFreeThreads>(p, sh, n_free, &T);
        if (blockIdx.x == 0) {
            for (int i = tid; i <= N; i += kFreeThreads) p.scratch->cu[i] = sh.cu[i];
            if (tid == 0) {
                p.scratch->bad = bad;
                p.scratch->total = T;
                p.scratch->n_free = n_free;
                if (bad) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
            }
        }
    } else {
        bad = p.scratch->bad != 0;
        T = p.scratch->total;
        n_free = p.scratch->n_free;
        for (int i = tid; i <= N && !bad; i += kFreeThreads) sh.cu[i] = p.scratch->cu[i];
        __syncthreads();
    }
    if (bad) {
        if (PASS == 3 && blockIdx.x == 0 && tid == 0) *p.n_free_out = n_free;
        return;
    }
    int lo, hi;
    run_of(blockIdx.x * W + warp, gridDim.x * W, T, &lo, &hi);
    if (PASS == 0) {
        if (free_count_down(p, sh, lo, hi)) atomicOr(p.status, FD_DEV_BAD_PAGE);
    } else if (PASS == 1) {
        free_claim(p, sh, T, lo, hi);
    } else if (PASS == 2) {
        const int mine = free_claims(p, sh, T, lo, hi);
        if ((tid & 31) == 0) p.scratch->count[blockIdx.x * W + warp] = mine;
    } else {
        // warps in front of this CTA's, and all: the counts' prefix sums
        int before = 0, all = 0;
        for (int i = tid; i < (int)gridDim.x * W; i += kFreeThreads) {
            const int n = p.scratch->count[i];
            all += n;
            if (i < (int)blockIdx.x * W) before += n;
        }
        int sum_before, sum_all;
        block_scan<kFreeThreads>(before, sh.wsum, &sum_before);
        block_scan<kFreeThreads>(all, sh.wsum, &sum_all);
        for (int w = 0; w < warp; ++w) sum_before += p.scratch->count[blockIdx.x * W + w];
        if (free_push(p, sh, T, lo, hi, n_free + sum_all - sum_before)) atomicOr(p.status, FD_DEV_BAD_PAGE);
        for (int i = blockIdx.x * kFreeThreads + tid; i < N; i += gridDim.x * kFreeThreads) p.prefix_lens[p.seqs[i]] = 0;
        if (blockIdx.x == 0 && tid == 0) *p.n_free_out = min(n_free + sum_all, p.num_pages);
    }
}

int launch_kv_free(const FreeParams& p, cudaStream_t s) {
    // (the lengths are on the device: the table's width bounds what a sequence holds)
    const long long most = (long long)p.n_seqs * p.max_pages;
    if (most <= kFreeSmall) {
        free_small_kernel<<<1, kFreeSmallThreads, 0, s>>>(p);
        return 1;
    }
    const int grid = (int)std::min<long long>((most + 4 * kFreeThreads - 1) / (4 * kFreeThreads), std::min(p.n_sms, 1024));
    int n = 0;
    for (auto pass : {free_pass_kernel<0>, free_pass_kernel<1>, free_pass_kernel<2>, free_pass_kernel<3>}) {
        if (launch(pass, grid, kFreeThreads, 0, s, p) != cudaSuccess) break;
        ++n;
    }
    return n;
}

// ------------------------------------------------------------------------------------------------ compact
constexpr int kClusterThreads = 1024, kMaxPageCluster = 8;

template <class K, class P>
static cudaError_t launch_cluster(K kernel, const P& p, int ctas, cudaStream_t s) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kClusterThreads);
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

__global__ void __launch_bounds__(kClusterThreads) compact_kernel(CompactParams p) {
    __shared__ int wsum[kClusterThreads / 32];
    __shared__ int s_holes, s_movers, s_bad;
    const int tid = threadIdx.x, R = (int)cluster_rank(), C = (int)cluster_size(), n = p.num_pages;
    const int per = ((n + C - 1) / C + 3) & ~3, lo = min(R * per, n), hi = min(lo + per, n);  // this CTA's ids
    const int n_free = *p.n_free;
    bool bad = n_free < 0 || n_free > n;  // the same in every CTA
    if (tid == 0) s_bad = 0;
    // ---- page_map: 1 for a page in use, 0 for a free one
    for (int i = lo + tid; i < hi; i += kClusterThreads) p.page_map[i] = 1;
    cluster_barrier();
    if (!bad) {
        bool mine = false;
        for (int k = R * kClusterThreads + tid; k < n_free; k += C * kClusterThreads) {
            const int id = p.free_pages[k];
            if ((unsigned)id >= (unsigned)n || atomicExch(p.page_map + id, 0) == 0) mine = true;  // outside the pool, or listed twice
        }
        if (mine) s_bad = 1;
    }
    cluster_barrier();
    for (int r = 0; r < C; ++r) bad = bad || peer_int(&s_bad, r) != 0;
    const int m = n - n_free;  // pages in use: ids below m are where they go
    if (!bad) {
        int holes = 0, movers = 0;
        for (int i = lo + tid; i < hi; i += kClusterThreads) {
            const bool live = __ldcg(p.page_map + i) != 0;
            holes += !live && i < m;
            movers += live && i >= m;
        }
        int c;
        block_scan<kClusterThreads>(holes, wsum, &c);
        if (tid == 0) s_holes = c;
        block_scan<kClusterThreads>(movers, wsum, &c);
        if (tid == 0) s_movers = c;
    }
    cluster_barrier();
    int holes = 0, movers = 0, all = 0;
    if (!bad) {
        for (int r = 0; r < C; ++r) {
            const int h = peer_int(&s_holes, r), v = peer_int(&s_movers, r);
            if (r < R) { holes += h; movers += v; }
            all += v;
        }
        if (all > p.max_copies) bad = true;  // (the same in every CTA)
    }
    if (!bad) {
        for (int base = lo; base < hi; base += kClusterThreads) {
            const int i = base + tid;
            const bool in = i < hi, live = in && __ldcg(p.page_map + i) != 0, hole = in && !live && i < m, mover = live && i >= m;
            int sum;
            const int bh = block_scan<kClusterThreads>(hole, wsum, &sum);
            if (hole) p.copy_dst[holes + bh] = i;
            holes += sum;
            const int bm = block_scan<kClusterThreads>(mover, wsum, &sum);
            if (mover) p.copy_src[movers + bm] = i;
            movers += sum;
            if (in) p.page_map[i] = live ? i : -1;
        }
    } else {
        for (int i = lo + tid; i < hi; i += kClusterThreads) p.page_map[i] = i;
    }
    const int moves = bad ? 0 : all;
    cluster_barrier();
    // ---- pages that move take their count of owners along (sources lie at or above m, targets below)
    for (int k = R * kClusterThreads + tid; k < moves; k += C * kClusterThreads) {
        const int from = __ldcg(p.copy_src + k), to = __ldcg(p.copy_dst + k);
        p.page_map[from] = to;
        if (p.shared) {
            p.shared[to] = p.shared[from];
            p.shared[from] = 0;
        }
    }
    for (int k = moves + R * kClusterThreads + tid; k < p.max_copies; k += C * kClusterThreads) p.copy_src[k] = p.copy_dst[k] = -1;
    if (R == 0 && tid == 0) {
        *p.n_copies = moves;
        *p.failed = bad;
        if (bad) atomicOr(p.status, n_free < 0 || n_free > n || all > p.max_copies ? FD_DEV_BAD_LENGTHS : FD_DEV_BAD_PAGE);
    }
    cluster_barrier();  // (a CTA's shared memory stays until its peers have read it)
}

// The tables and the free list after a compaction.
__global__ void __launch_bounds__(256) rename_kernel(CompactParams p) {
    if (*p.failed) return;
    const long long stride = (long long)gridDim.x * blockDim.x, first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    const int n_free = *p.n_free;
    for (long long i = first; i < (long long)p.batch * p.max_pages; i += stride) {
        const int id = p.page_table[i];
        if ((unsigned)id < (unsigned)p.num_pages) p.page_table[i] = p.page_map[id];
    }
    for (long long i = first; i < n_free; i += stride) p.free_pages[i] = p.num_pages - 1 - (int)i;
}

int launch_kv_compact(const CompactParams& p, cudaStream_t s) {
    if (launch_cluster(compact_kernel, p, p.num_pages <= 2 * kClusterThreads ? 1 : kMaxPageCluster, s) != cudaSuccess) return 0;
    const long long work = (std::max<long long>((long long)p.batch * p.max_pages, p.num_pages) + 1023) / 1024;
    const int grid = (int)std::max(1LL, std::min<long long>(work, 4LL * p.n_sms));
    return launch(rename_kernel, grid, 256, 0, s, p) == cudaSuccess ? 2 : 1;
}

// ------------------------------------------------------------------------------------------------ copy
// A CTA takes pieces of pages, as many words as its threads take in one round.
constexpr int kCopyThreads = 256;

__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(CopyPagesParams p, int pieces) {
    const int n = p.n_copies ? min(*p.n_copies, p.max_copies) : p.max_copies;
    const int words = (int)(p.page_bytes / 16);
    const int per = (words + pieces - 1) / pieces;
    for (long long t = blockIdx.x; t < (long long)n * pieces; t += gridDim.x) {
        const int k = (int)(t / pieces), w0 = (int)(t - (long long)k * pieces) * per, w1 = min(words, w0 + per);
        const int from = p.src[k], to = p.dst[k];
        if (from < 0 || to < 0) continue;
        if (from >= p.num_pages || to >= p.num_pages) {  // never form an address from a bad id
            if (threadIdx.x == 0) atomicOr(p.status, FD_DEV_BAD_PAGE);
            continue;
        }
        const uint4* a = reinterpret_cast<const uint4*>(p.cache + (long long)from * p.page_bytes);
        uint4* b = reinterpret_cast<uint4*>(p.cache + (long long)to * p.page_bytes);
        for (int w = w0 + threadIdx.x; w < w1; w += 4 * kCopyThreads) {
            uint4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (w + u * kCopyThreads < w1) v[u] = __ldcs(a + w + u * kCopyThreads);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (w + u * kCopyThreads < w1) __stcs(b + w + u * kCopyThreads, v[u]);
        }
    }
}

void launch_kv_copy_pages(const CopyPagesParams& p, cudaStream_t s) {
    if (p.max_copies == 0) return;
    const int pieces = (int)((p.page_bytes / 16 + 4 * kCopyThreads - 1) / (4 * kCopyThreads));  // one round of the threads each
    const int grid = (int)std::min<long long>((long long)p.max_copies * pieces, 8LL * p.n_sms);
    copy_pages_kernel<<<grid, kCopyThreads, 0, s>>>(p, pieces);
}

}  // namespace fd
