// What the tensor-core attention kernels share: pieces of work and their descriptors, the walk over a CTA's range, the plan a
// small call makes for itself, the Q load warp.
#pragma once

#include <cuda.h>

#include "fd_internal.cuh"
#include "fd_sm100.cuh"

namespace fd {

using namespace sm100;

// The plan of a call that plans for itself (at most kSelfPlanMaxRb sequences, one row block each), in shared memory.
struct SelfScans {
    int cu_q[kSelfPlanMaxRb + 1], cu_tiles[kSelfPlanMaxRb + 1], cu_ne[kSelfPlanMaxRb + 1];
    int fatal;
};
static_assert(sizeof(SelfScans) <= 304, "SelfScans must fit between the descriptor ring and the exchange buffer");
static_assert(sizeof(RowBlock) * kSelfPlanMaxRb <= 1024, "row blocks of a self-planned call must fit their slot");

// The tiles [s_c, e_c) a CTA works on and the row block that owns the first of them.
struct Range {
    int s_c, e_c, first;
};

struct Piece {
    int v, b, kvh, tile0, nt, n, Lq, M, nb, i0, Lv, kv_len, rows, row0, slot, seg_nt;  // v: row block; Lv: its block rows
    bool complete;
};

// Piece that starts at tile t.  `hint` is a row block at or before the one that owns t (pieces are walked in
// order, so the previous piece's row block will do): a short forward walk replaces a search.
__device__ __forceinline__ Piece decode_piece(const AttnParams& p, int n_rb, int t, int s_c, int e_c, int cta, int hint) {
    // p.plan may point into shared memory (a call that plans for itself): plain loads either way
    Piece pc;
    int lo = hint;
    while (lo + 1 < n_rb && p.Hkv * p.plan.cu_tiles[lo + 1] <= t) ++lo;
    pc.v = lo;
    const int ntiles = p.plan.cu_tiles[lo + 1] - p.plan.cu_tiles[lo];
    const int rem = t - p.Hkv * p.plan.cu_tiles[lo];
    pc.kvh = rem / ntiles;
    pc.tile0 = rem % ntiles;
    const int seg_start = t - pc.tile0, seg_end = seg_start + ntiles;
    const int t_end = min(e_c, seg_end);
    pc.nt = t_end - t;
    pc.seg_nt = ntiles;
    const int4* rbp = reinterpret_cast<const int4*>(p.plan.rb + lo);
    const int4 r0 = rbp[0], r1 = rbp[1];  // (b, i0, n, Lq), (M, nb, -, -)
    pc.b = r0.x;
    pc.i0 = r0.y;
    pc.n = r0.z;
    pc.Lq = r0.w;
    pc.M = r1.x;
    pc.nb = r1.y;
    pc.Lv = min(p.rb_rows, pc.Lq - pc.i0);
    pc.kv_len = pc.n + pc.Lq;
    pc.rows = pc.Lv * p.G;
    pc.row0 = p.plan.cu_q[lo];
    // with one cluster per segment every piece goes through the cluster merge, a piece that holds all tiles too
    pc.complete = (t == seg_start) && (t_end == seg_end) && p.cluster == 0;
    pc.slot = 2 * cta + (t == s_c ? 0 : 1);
    return pc;
}


__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Under programmatic dependent launch: block until the launch before this one on the stream has completed and its
// writes are visible.  Returns at once when that has happened already (or the launch was an ordinary one).
__device__ __forceinline__ void wait_prior_launch() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Warp-uniform bounded wait.
__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile int* abort) {
    const bool ok = mbar_wait(bar, parity, abort);
    return __all_sync(0xffffffffu, ok);
}

// Piece descriptors.  The Q load warp walks the pieces ahead of everyone, decodes each one (a chain of
// dependent global loads) and publishes it in a small ring in shared memory; the MMA warp and the softmax
// groups pick it up from there, so the decode is off their critical path at a piece boundary.  Slot
// reuse is safe: descriptor N + 1 is written after every QK^T of piece N - 1 has completed, hence the P V of the tile B tiles
// before its last (B: buffers of S).  Every consumer copies its descriptor to registers at piece start, so one that is not
// past piece N - 1 - B yet has copied that piece's: descriptors N - B to N + 1 must not share a slot, and with two buffers
// (bf16) four slots do, with three (FP4) eight.
template <int SLOTS, class Bars>
__device__ __forceinline__ void publish_piece(Bars* bars, Piece* ring, int n, const Piece& pc) {
    ring[n & (SLOTS - 1)] = pc;
    asm volatile("st.release.cta.shared::cta.s32 [%0], %1;" ::"r"(smem_u32(&bars->desc_n)), "r"(n + 1) : "memory");
}
template <class Bars>
__device__ __forceinline__ bool piece_published(Bars* bars, int n) {
    int v;
    asm volatile("ld.acquire.cta.shared::cta.s32 %0, [%1];" : "=r"(v) : "r"(smem_u32(&bars->desc_n)) : "memory");
    return v > n;
}
// Bounded like every other wait; false if it gave up (abort raised here or elsewhere).
template <class Bars>
__device__ __forceinline__ bool wait_piece(Bars* bars, int n, volatile int* abort) {
    if (piece_published(bars, n)) return true;
    const unsigned long long t0 = global_ns();
    for (uint32_t it = 1;; ++it) {
        if (piece_published(bars, n)) return true;
        if ((it & 15u) == 0u) {
            if (*abort) return false;
            if (global_ns() - t0 > kWaitLimitNs) break;
        }
    }
    *abort = 1;
    return false;
}

// ---------------------------------------------------------------------------------------------
// Roles.  Each walks the pieces of the CTA's tile range [s_c, e_c) in the same order and keeps
// its own copies of the running counters:
//   g0        KV tiles pushed through the rings before this piece      (ring slot and phase)
//   u_base[s] tiles stream s has processed before this piece           (phase of s_full / p_full / pv_done)
//   piece     pieces before this one                                   (phase of q_full / q_free / o_free)
// ---------------------------------------------------------------------------------------------
struct Walk {
    int t, g0, u_base[2], piece, b;
    __device__ __forceinline__ void advance(const Piece& pc) {
        b = pc.v;  // the row block: the next piece's walk starts from it
        g0 += pc.nt;
        u_base[0] += (pc.nt + 1) >> 1;
        u_base[1] += pc.nt >> 1;
        ++piece;
        t += pc.nt;
    }
};

// ---------------------------------------------------------------------------------------------
// A call that plans for itself (kTcSelfPlanned, kTcCluster): at most kSelfPlanMaxRb sequences, one row block
// each.  Warp 0 of every CTA checks the lengths and makes the scans the plan kernel would have made, into
// shared memory; the roles then read them through the same Plan pointers.  No launch, no dependency.
// ---------------------------------------------------------------------------------------------
template <int MODE>
__device__ __forceinline__ void self_plan(const AttnParams& p, SelfScans* sc, RowBlock* rbs, int* s_cs, int* s_first) {
    const int lane = threadIdx.x & 31, B = p.batch;
    const bool live = lane < B;
    long long n = 0, Lq = 0, M = 0, nb = 1;
    bool bad = false;
    if (live) {
        n = p.prefix_lens[lane]; Lq = p.q_lens[lane]; M = p.n_mask[lane];
        nb = p.n_blocks ? p.n_blocks[lane] : 1;
        bad = n < 0 || Lq < 0 || M < 0 || M > Lq || Lq > p.max_q_len || n + Lq > (long long)p.max_pages * 16;
        bad = bad || nb < 0 || (nb > 1 && (M % nb != 0 || nb > Lq - M));  // equal mask blocks, one hypothesis each
        if (bad) Lq = 0;
    }
    int q = (int)Lq, t = Lq > 0 ? (int)((n + Lq + kTileTokens - 1) / kTileTokens) : 0, ne = t > 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int uq = __shfl_up_sync(0xffffffffu, q, o), ut = __shfl_up_sync(0xffffffffu, t, o), un = __shfl_up_sync(0xffffffffu, ne, o);
        if (lane >= o) { q += uq; t += ut; ne += un; }
    }
    const int rows = __shfl_sync(0xffffffffu, q, 31);
    const bool fatal = __any_sync(0xffffffffu, bad) || rows != p.total_q_rows;
    if (live) {
        sc->cu_q[lane + 1] = q; sc->cu_tiles[lane + 1] = t; sc->cu_ne[lane + 1] = ne;
        const RowBlock rb = {lane, 0, (int)n, (int)Lq, (int)M, (int)nb, {0, 0}};
        rbs[lane] = rb;
    }
    if (lane == 0) {
        sc->cu_q[0] = 0; sc->cu_tiles[0] = 0; sc->cu_ne[0] = 0;
        sc->fatal = fatal;
        if (fatal && blockIdx.x == 0) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
    }
    if (MODE == kTcSelfPlanned) {
        // the range starts of this CTA and its neighbours, a lane each: the cuts the plan kernel would have made
        // (range_cut is shared with it and with the host), all in one go instead of one after the other
        __syncwarp();
        const int tiles = __shfl_sync(0xffffffffu, t, 31), nonempty = __shfl_sync(0xffffffffu, ne, 31);
        const long long k = p.piece_cost, W = (long long)p.Hkv * (tiles + k * nonempty);
        const int total = fatal ? 0 : tiles * p.Hkv;
        const int n_use = ranges_in_use(W, k, p.min_range_tiles, p.n_ctas);
        const int cc = (int)blockIdx.x - kCsWindow / 2 + 1 + lane;
        int start = 0, first = 0;
        if (cc >= 0 && cc <= p.n_ctas) {
            const int* ct_ = sc->cu_tiles;
            const int* ne_ = sc->cu_ne;
            start = (cc >= n_use || total == 0) ? total
                                                : range_cut(cc, n_use, W, B, p.Hkv, k, [ct_](int b) { return ct_[b]; }, [ne_](int b) { return ne_[b]; }, &first);
        }
        s_cs[lane] = start;
        if (cc == (int)blockIdx.x) *s_first = first;
    }
}

// Q load warp: the G * Lq rows of a piece -> shared memory, K-major, 128-byte swizzle.  q is seen as
// [T][Hq][d]; one TMA box is 64 elements of d x the G q-heads of the kv-head x q_box_t block rows, which
// lands as q_box_t * G consecutive 128-byte rows, row (i, g) at i * G + g: the order the MMA wants.  The
// last box of a piece may reach past the block (rows of the next sequence, or zeros past T): each query
// row only ever influences its own output row, and those rows are never stored.
template <int D, int SLOTS, class Bars>
__device__ __forceinline__ void q_role(const CUtensorMap& qmap, const AttnParams& p, int n_rb, unsigned char* sq, Bars* bars, Piece* ring,
                                       const Range rg, volatile int* abort) {
    constexpr int kHalves = D / 64;
    const int lane = threadIdx.x & 31, cta = blockIdx.x;
    const int bt = p.q_box_t;
    const int s_c = rg.s_c, e_c = rg.e_c;
    Walk w = {s_c, 0, {0, 0}, 0, rg.first};
    int issued = 0;
    Piece pc = decode_piece(p, n_rb, w.t, s_c, e_c, cta, w.b);
    if (lane == 0) publish_piece<SLOTS>(bars, ring, 0, pc);
    if (p.early == 1) wait_prior_launch();  // q may be written by it (p.early >= 2: it is known not to be)
    while (w.t < e_c) {
        if (w.piece > 0 && !wait_all(&bars->q_free, (w.piece - 1) & 1, abort)) break;
        const int nbox = (pc.Lv + bt - 1) / bt;
        if (lane == 0) mbar_arrive_expect_tx(&bars->q_full, nbox * bt * p.G * 128 * kHalves);
        __syncwarp();
        for (int e = lane; e < nbox * kHalves; e += 32) {
            const int j = e / kHalves, half = e % kHalves;
            tma_load_3d(sq + half * (kMaxRows * 128) + j * bt * p.G * 128, &qmap, half * 64, pc.kvh * p.G, pc.row0 + j * bt, &bars->q_full);
        }
        issued = w.piece + 1;
        w.advance(pc);
        if (w.t < e_c) {
            // the next piece: descriptor for the other roles, and its Q rows on their way into L2
            pc = decode_piece(p, n_rb, w.t, s_c, e_c, cta, w.b);
            if (lane == 0) publish_piece<SLOTS>(bars, ring, w.piece, pc);
            const int nb2 = (pc.Lv + bt - 1) / bt;
            for (int e = lane; e < nb2 * kHalves; e += 32)
                tma_prefetch_3d(&qmap, (e % kHalves) * 64, pc.kvh * p.G, pc.row0 + (e / kHalves) * bt);
        }
    }
    if (*abort && issued > 0) {  // drain the last copy before the shared memory is given back
        const unsigned long long t0 = global_ns();
        for (uint32_t it = 0; it < kSpinLimit && global_ns() - t0 < kWaitLimitNs; ++it)
            if (mbar_try_wait(&bars->q_full, (issued - 1) & 1)) break;
    }
}

}  // namespace fd
