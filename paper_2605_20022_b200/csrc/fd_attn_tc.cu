// Tensor-core split-KV attention under the hybrid mask for sm_100a: TMA-staged KV pages,
// tcgen05 MMAs with accumulators in tensor memory, softmax in registers.
//
// Work decomposition.  The plan kernel cuts every sequence's query block into row blocks (as many
// block rows as fit a 128-row tile with their G q-heads; one per sequence unless the block is long),
// numbers all 128-token KV tiles of the call (row block, then kv-head, then position) and cuts them
// into one contiguous range per persistent CTA, of equal cost (tiles plus a start-up charge per
// segment).  A range is walked piece by piece, a piece being its intersection with one
// (row block, kv-head) segment.
//
// One piece.  The at most 128 query rows of a row block that share the kv-head (row r = block row
// r / G of q-head kvh * G + r % G) form the M = 128 operand of every MMA, so each KV tile is
// read from HBM once for all of them.  Per tile j of the piece:
//     producer warps: one for K, one for V; 8 lanes issue one TMA box each -- a whole page of the
//                     kv-head, both 64-wide halves of d (4 KB: the TMA unit's cost is mostly per
//                     box, measured 20.9 B/clk per SM with 2 KB boxes, 28.9 with 4 KB) -- into a
//                     128B-swizzled buffer [8-token group][half][8 rows][128 B] of a 3-deep ring
//                     per operand; a K buffer is released by the QK^T commit, a V buffer by P V;
//     MMA warp      : S_s = Q K^T (tcgen05.mma, A and B from shared memory, S in TMEM), and
//                     after the softmax O_s += P_s V (A = P from TMEM, B = V MN-major);
//     softmax group : 128 threads, one query row each: tcgen05.ld the row of S, hybrid mask
//                     from the row's (kind, index) -> first invisible key position, online
//                     softmax in the log2 domain, bf16 P written back over S in TMEM.
// Tiles alternate between two independent streams s = j & 1, each with its own softmax
// group, S/P buffer, (m, l) state and O accumulator in TMEM, so the tensor pipe works on one
// stream while the other is in its softmax; the two streams are merged in the epilogue.  A segment
// that several CTAs share is merged by whichever of them delivers its partial last (a counter, no waiting).  O is
// rescaled lazily (only when a row maximum grows by more than 2^8), which is exact because
// the same reference maximum is used for P, l and O.
//
// TMEM columns: S0/P0 [0,128)  S1/P1 [128,256)  O0 [256,256+d)  O1 [384,384+d).
//
// Pieces are pipelined as well: every role walks the CTA's pieces on its own and meets the others only
// through mbarriers.  The load warps run ahead through the K / V rings; a fourth helper warp brings
// the next piece's Q tile in (TMA) as soon as the last QK^T of the current piece has completed, has
// the piece after that prefetched into L2, and publishes every piece's descriptor for the MMA warp and
// the softmax groups; the MMA warp starts the next piece while the softmax groups are still in the
// epilogue of the current one (the first P V of a piece waits until the epilogue has read O).
//
// Every wait is bounded.  A wait that runs out raises a CTA-wide abort flag: all roles leave
// their loops, in-flight TMA copies are drained, TMEM is released and FD_DEV_TIMEOUT is set.
//
// 4-bit and 8-bit pages (wide formats).  Same walk, same epilogue and merges; a tile differs in three places.
//     loads    : codes and scales of a page come into a raw ring, K and V together: in 4 bits, where they lie side by side, by one
//                untiled bulk copy, 3.6 times fewer bytes than bf16; in 8 bits by one TMA box, the scales by plain loads;
//     widening : eight warps turn a raw tile into fp16 tiles in the layout the MMAs read.  code * scale is exact in
//                fp16 in both formats (fd_fp4.cuh, fd_fp8.cuh).  In 4 bits K and V; k_scale goes into the scale of the scores,
//                v_scale into the output; Q is converted to fp16 by the same warps, a row against a power of two of its own.  In
//                8 bits V alone: K's codes are an operand of the MMA as they are, against Q as a sum of two e4m3 tiles, and
//                the softmax multiplies the 16 columns of a page by its scale;
//     softmax  : P is fp16.  Three S / P buffers and one O; the groups take turns and share the reference of a row.
// TMEM columns: S / P buffers [0,128) [128,256) [256,384), O [384,384+d).
//
// What bounds the 4-bit form: the tensor pipe needs 1024 clocks a tile (d = 128, 128 rows), the exponentials as many, shared memory
// about 1550 (Q K^T reads 128 bytes a clock, widening writes what P V reads); measured are 2400 with full rows: a batch of
// 16 on a 32k prefix takes 330 us call after call, 834 TFLOP/s, 51 % of the measured cuBLAS burst rate, 1.9 TB/s of cache
// (283 us and 971 TFLOP/s in short runs, before the power cap lowers the clock).  What is missing is latency: each of softmax, P V, Q K^T and widening hands over through a barrier (150 to 300 clocks a hand-over) with five
// warps to a scheduler.  A piece costs 6.8 us more than its tiles (first and last tile in two passes, O drained before the
// next piece's first P V, code that is not in the instruction cache: unrolling the two-pass form made a batch of 64 go from
// 141 to 163 us).  By that fit a batch of 64 with 1-16 rows (133 us) spends 72 us on 68 tiles a CTA and 31 us on 4.5 pieces.  The
// merges' live accumulators spill (536 bytes stored in the planned form, 680 in the self-planned one), and builds that differ
// in a few instructions of the epilogue took from 132 to 151 us at batch 64.  Registers of the softmax warps 152 (all that the
// launch has): fewer spills, but 371 us on the 32k prefix.
// Measured and dropped, batch 16 on 32k / batch 64, one token each: S^T = K Q^T with K widened into TMEM, no K tile in shared
// memory, 394 / 95-115 us, but 155-183 us at up to 16 rows; two S buffers and two accumulators, as in the bf16 form, 344 / 159;
// four widening warps 472 / 190; four for K and four for V, 431 / 187.
//
// The 8-bit form (d = 128): batch 16 on 32k 319 us (3.4 TB/s of cache; 376 call after call, under the power cap), batch 64 127, batch 1 12.4.  Half
// the widening is gone, and what bounds it is the same: hand-overs and, at a piece's ends, code that is not in the instruction
// cache.  Measured on the way, batch 16 on 32k / batch 64: both widened as in 4 bits, K and V a bulk copy each 464 / 182; K as it is, one box a page
// 335 / 173; eight widening warps 346 / 144; scales a tile ahead, Q by a rolled loop, one form of the widening 327 / 132.
// Dropped: four widening warps and 176 registers for the softmax 309 / 146 (d = 64 99 us where eight take 77); two S buffers and two accumulators, the
// bf16 form's, whose whole row in registers spills at the 176 to 200 there are, 458 / 164; 152 or 160 registers for the softmax
// 389 / 139 to 142.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <vector>

#include "fd_attn_common.cuh"
#include "fd_fp4.cuh"
#include "fd_fp8.cuh"
#include "fd_internal.cuh"
#include "fd_sm100.cuh"

namespace fd {

using namespace sm100;

namespace {

// A format whose pages are widened on their way to the MMAs (FMT: FD_KV_*).
__host__ __device__ constexpr bool wide(int fmt) { return fmt != FD_KV_BF16; }

// warps 0-3 softmax group 0, 4-7 softmax group 1, 8 K loads, 9 V loads, 10 MMA, 11 Q loads
// (wide formats: 8 loads both, 9 issues P V, 10 issues Q K^T, 12-19 widen)
constexpr int kKWarp = 8, kVWarp = 9, kMmaWarp = 10, kQWarp = 11;
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr int kEarlyLoadMaxTiles = 96;     // longest range of a CTA that starts on its KV before the previous launch has completed
// Who issues the P V of a tile.  In a range of at least kGroupPvMinTiles tiles warp 0 of the softmax group that wrote P
// issues it, as soon as the group's P is whole: the MMA warp, which takes its waits in program order (K tile, then the
// P V that last read the S buffer), then never stands between a finished P and its P V (3-10 % per call from batch 8
// upwards).  In a shorter range -- and in the cluster form, whose CTAs have one to three tiles -- the MMA warp issues
// it: there the issue sits on the group's critical path for nothing (batch 1: +0.7 us per call when tried).
#ifndef FD_GROUP_PV_MIN_TILES
#define FD_GROUP_PV_MIN_TILES 6
#endif
constexpr int kGroupPvMinTiles = FD_GROUP_PV_MIN_TILES;
template <int MODE>
__device__ __forceinline__ bool pv_by_group(int range_tiles) { return MODE != kTcCluster && range_tiles >= kGroupPvMinTiles; }

// 1: Q K^T(j) waits for the completion of the P V whose P it overwrites; 0: it does not (see mma_role).
#ifndef FD_QK_MODE
#define FD_QK_MODE 1
#endif
// 1: the first fill of the K and V rings is staggered (see load_role)
#ifndef FD_STAGGER
#define FD_STAGGER 1
#endif

template <int D, int MODE, int FMT>
struct Cfg {
    // the warps behind warp 11 widen the tiles: K and V (FP4), or V alone (FP8)
    static constexpr int kWidenWarps = wide(FMT) ? 8 : 0;
    static constexpr int kThreads = 384 + 32 * kWidenWarps;
    // Registers per thread of the softmax warps, of warps 8-11 and of the widening warps.  What the groups take adds up to no more
    // than what the launch allocates: configure_kernel compares the two before the kernel's first launch.
    static constexpr int kRegSoftmax = wide(FMT) ? 144 : 224;
    static constexpr int kRegHelper = FMT == FD_KV_FP8 ? 64 : wide(FMT) ? 48 : 56;
    static constexpr int kRegWiden = 64;
    static constexpr int kRegTotal = 256 * kRegSoftmax + 128 * kRegHelper + 32 * kWidenWarps * kRegWiden;
    static_assert(kRegTotal <= 65536, "register split");
    // buffers in the K ring, and again in the V ring (wide formats: of widened tiles, fed from the raw ring)
    static constexpr int kStages = wide(FMT) ? (D == 128 ? 2 : 4) : (D == 128 ? 3 : 6);
    static constexpr int kQBytes = kMaxRows * D * 2;
    static constexpr int kKBytes = kTileTokens * D * 2;  // one K (or V) tile
    static constexpr int kRawStages = wide(FMT) ? (D == 128 ? 3 : 6) : 0;
    // one page of the kv-head in a stage: codes and scales of K and V, which lie side by side in the cache (FP4), or the codes (FP8)
    static constexpr int kRawPage = FMT == FD_KV_FP8 ? 2 * 16 * D : 2 * fp4_page_bytes(D);
    static constexpr int kRawBytes = 8 * kRawPage;           // ... of a tile
    // Behind Q: the K ring -- for FP8 the raw ring, whose K the MMAs read as it is -- then the V ring, then (FP4) the raw ring.
    static constexpr int kVOffset = kQBytes + (FMT == FD_KV_FP8 ? kRawStages * kRawBytes : kStages * kKBytes);
    static constexpr int kBarOffset = kVOffset + kStages * kKBytes + (FMT == FD_KV_FP4 ? kRawStages * kRawBytes : 0);
    static constexpr int kCsOffset = kBarOffset + 320;           // window of the CTA range starts
    static constexpr int kDescOffset = kBarOffset + 448;         // ring of piece descriptors
    static constexpr int kScanOffset = kBarOffset + 720;         // SelfScans: the scans of a call that plans for itself
    static constexpr int kExOffset = kBarOffset + 1024;          // [2][128] floats: stream exchange in the epilogue
    static constexpr int kRbOffset = kBarOffset + 2048;          // row blocks of a call that plans for itself
    static constexpr int kWideOffset = kRbOffset + 1024;         // wide formats: WideShared
    static constexpr int kSmemBytes = kRbOffset + 1024 + (wide(FMT) ? 5120 : 0);  // the dynamic shared memory is declared 1024-byte aligned
    static constexpr int kDescSlots = wide(FMT) ? 8 : 4;  // ring of piece descriptors: see publish_piece
    static constexpr int kHalves = D / 64;
    // A K or V tile in shared memory: [8-token group][half of d][8 rows][128 B] -- what one TMA box per page
    // (two groups) lands; for either half the 16 groups lie kGroupBytes apart, the stride the MMA descriptors name.
    static constexpr int kGroupBytes = kHalves * 1024;
    static constexpr int kPageBytes = 2 * kGroupBytes;
    static_assert(kSmemBytes <= 227 * 1024, "shared memory of one CTA");
};

struct Bars {
    uint64_t k_full[6], k_empty[6], v_full[6], v_empty[6];
    uint64_t s_full[2], p_full[2], pv_done[2];
    uint64_t q_full, q_free;   // Q tile of a piece landed / no longer read by any MMA
    uint64_t o_free;           // the epilogue of a piece has read O out of TMEM
    uint64_t merge_bar;        // the other pieces of a segment have been copied into shared memory (merger, last piece)
    uint32_t tmem_base;
    int abort;
    int epi_flag;              // per-epilogue decisions of thread 0: bit 0 merge, bit 1 leave
    int desc_n;                // piece descriptors published so far (written by the Q load warp)
    int piece_ok;              // thread 0 of the softmax groups: the descriptor of the next piece is there
    int first;                 // a call that plans for itself: the row block that owns the first tile of this CTA's range
    int bad;                   // bit (piece & 31): a load warp met a page id outside the pool in that piece (they run at most
                               // as many pieces ahead as there are tile buffers, 14; the softmax groups clear the bit once past it)
};
static_assert(sizeof(Bars) <= 320, "Bars must fit in front of the range-start window");

// What a call on pages of a wide format keeps beside Bars.
struct WideShared {
    uint64_t raw_full[6], raw_empty[6];  // a stage of codes and scales has landed / has been widened
    uint64_t q_ready;                    // the Q tile of a piece has been turned into fp16
    // Three S / P buffers and one O (columns 0, 128, 256; 384): tile g uses buffer g % 3, the groups take turns.
    uint64_t s_full[3], p_full[3], pv_done[3];
    uint64_t decided[4][2];              // [warp of a group][tile & 1]: the tile has settled its rows' references
    // Per query row: what its scores are multiplied by.  Slot = piece & 3: the Q of piece n is converted when every Q K^T of
    // piece n - 1 has completed, hence every P V up to three tiles before that, and those of piece n - 4 among them.
    float row_scale[4][kMaxRows];
    float ref[2][kMaxRows];              // [piece & 1] the reference of each row, -inf while it has none
    Piece ring[8];                       // piece descriptors
    uint64_t q_read;                     // FP8, d = 64: the Q tile of a piece is in registers
    // FP8: the scales of a tile's pages, K's then V's.  Slot = tile & 15: it is written for tile t when the raw stage of t is free, hence
    // V of the tile kRawStages before it widened, P V of the tile kStages before that one completed, and that tile's softmax done: of
    // tile t - 5 (d = 128) or t - 10.
    alignas(16) float sc[16][16];
};
static_assert(sizeof(WideShared) <= 5120, "WideShared must fit behind the row blocks");


// K (which = 0) or V (which = 1) load warp.
template <int D, int MODE>
__device__ __forceinline__ void load_role(const CUtensorMap& tmap, const AttnParams& p, int n_rb, unsigned char* ring, uint64_t* full,
                                          uint64_t* empty, int which, const Range rg, uint64_t* k0_full, int* bad, volatile int* abort) {
    using C = Cfg<D, MODE, false>;
    const int lane = threadIdx.x & 31, cta = blockIdx.x;
    constexpr int kOps = 8;  // pages of a tile: one box each
    const int pg = lane;
    int issued = 0;
    // the KV stream is read once: let it leave L2 first, so that Q, the split partials and the page
    // table (all re-read) stay resident next to a stream many times the size of the cache
    const uint64_t policy = make_policy_evict_first();
    const int s_c = rg.s_c, e_c = rg.e_c;
    Walk w = {s_c, 0, {0, 0}, 0, rg.first};
    bool ok = true;
    // p.early: the first piece and its first page ids are looked up while the launch before this one may still run;
    // p.early == 2: so is the KV pool itself -- that launch is known not to write it -- and this warp waits for it
    // only if it has something to write (a sequence to flag); p.early == 3: that launch is the KV append, which
    // writes the query block's own slots and nothing else: tiles of the prefix are read ahead, the wait comes before
    // the first tile that reaches into the block (pages are 16 tokens, tiles 128: no page lies in both kinds)
    bool waited = !p.early;
    bool bad_early = false;
    while (w.t < e_c && ok) {
        const Piece pc = decode_piece(p, n_rb, w.t, s_c, e_c, cta, w.b);
        const int32_t* table = p.page_table + (long long)pc.b * p.max_pages;
        // Page ids are fetched a batch of four tiles (32 pages, one per lane) at a time and one batch
        // ahead, so the table lookup -- a dependent global load -- never sits between a buffer becoming
        // free and its refill, not even while the ring is filling up at the start of a piece.
        auto load_ids = [&](int batch) -> int {
            const int j = batch * 4 + (lane >> 3);
            const int pos = ((pc.tile0 + j) * 8 + (lane & 7)) * 16;
            if (!(j < pc.nt && pos < pc.kv_len)) return -1;
            int id = table[pos >> 4];
            if ((unsigned)id >= (unsigned)p.num_pages) {  // never form an address from a bad id
                if (!waited && p.early >= 2) { wait_prior_launch(); waited = true; }
                if (waited) atomicOr(p.status, FD_DEV_BAD_PAGE); else bad_early = true;  // (no global write ahead of the prior launch)
                atomicOr(bad, 1 << (w.piece & 31));
                id = 0;
            }
            return id;
        };
        int ids_cur = load_ids(0), ids_next = load_ids(1);
        for (int j = 0; j < pc.nt; ++j) {
            const int g = w.g0 + j, st = g % C::kStages, use = g / C::kStages;
            if (j > 0 && (j & 3) == 0) { ids_cur = ids_next; ids_next = load_ids((j >> 2) + 1); }
            const int phys = __shfl_sync(0xffffffffu, ids_cur, (j & 3) * 8 + pg);
            if (!waited && (p.early == 1 || (p.early == 3 && (pc.tile0 + j + 1) * kTileTokens > pc.n))) {  // the launch before this one may write what this tile holds
                wait_prior_launch();
                waited = true;
                if (bad_early) atomicOr(p.status, FD_DEV_BAD_PAGE);
            }
            if (!wait_all(&empty[st], (use & 1) ^ 1, abort)) { ok = false; break; }
#if FD_STAGGER
            // The first fill of the rings is not issued all at once: every CTA of the grid starts at the same moment,
            // and 224 KB per SM in one burst makes the first K tile -- all the MMA warp needs to begin -- land with
            // the last of it.  K tiles 0 and 1 go out at once; the V tiles and the third K tile follow when K tile 0
            // has landed (V tile 0 is not needed before the first softmax is through).  A delay, not a dependency:
            // it ends by itself after a few microseconds.
            if (g == (which ? 0 : 2) && k0_full != nullptr) {
                const unsigned long long t0 = global_ns();
                while (!mbar_try_wait(k0_full, 0) && global_ns() - t0 < 4000ull) {}
                __syncwarp();
            }
#endif
            const int pos0 = (pc.tile0 + j) * kTileTokens;
            const int npg = min(8, (pc.kv_len - pos0 + 15) >> 4);
            if (lane == 0) mbar_arrive_expect_tx(&full[st], npg * (16 * D * 2));
            __syncwarp();
            if (lane < kOps && phys >= 0) {
                unsigned char* dst = ring + st * C::kKBytes + pg * C::kPageBytes;
                tma_load_4d_hint(dst, &tmap, 0, 0, 0, ((phys * 2 + which) * p.Hkv + pc.kvh) * 2, &full[st], policy);
            }
            issued = g + 1;
        }
        w.advance(pc);
    }
    if (*abort) {  // drain TMA copies still in flight before the shared memory is given back
        for (int g = max(0, issued - C::kStages); g < issued; ++g) {
            const int st = g % C::kStages, use = g / C::kStages;
            const unsigned long long t0 = global_ns();
            for (uint32_t it = 0; it < kSpinLimit && global_ns() - t0 < kWaitLimitNs; ++it)
                if (mbar_try_wait(&full[st], use & 1)) break;
        }
    }
}

// FP4 load warp: codes and scales of K and V of a page lie side by side in the cache, so one untiled bulk copy a page
// brings both (2304 bytes at d = 128).  Otherwise the K load warp's walk: see load_role.
template <int D, int MODE>
__device__ __forceinline__ void load_role_fp4(const AttnParams& p, int n_rb, unsigned char* raw, WideShared* f4, const Range rg,
                                              int* bad, volatile int* abort) {
    using C = Cfg<D, MODE, FD_KV_FP4>;
    const int lane = threadIdx.x & 31, cta = blockIdx.x;
    int issued = 0;
    const uint64_t policy = make_policy_evict_first();
    const int s_c = rg.s_c, e_c = rg.e_c;
    Walk w = {s_c, 0, {0, 0}, 0, rg.first};
    bool ok = true, waited = !p.early;
    bool bad_early = false;
    while (w.t < e_c && ok) {
        const Piece pc = decode_piece(p, n_rb, w.t, s_c, e_c, cta, w.b);
        const int32_t* table = p.page_table + (long long)pc.b * p.max_pages;
        auto load_ids = [&](int batch) -> int {  // four tiles (32 pages, one per lane), one batch ahead
            const int j = batch * 4 + (lane >> 3);
            const int pos = ((pc.tile0 + j) * 8 + (lane & 7)) * 16;
            if (!(j < pc.nt && pos < pc.kv_len)) return -1;
            int id = table[pos >> 4];
            if ((unsigned)id >= (unsigned)p.num_pages) {  // never form an address from a bad id
                if (!waited && p.early >= 2) { wait_prior_launch(); waited = true; }
                if (waited) atomicOr(p.status, FD_DEV_BAD_PAGE); else bad_early = true;
                atomicOr(bad, 1 << (w.piece & 31));
                id = 0;
            }
            return id;
        };
        int ids_cur = load_ids(0), ids_next = load_ids(1);
        for (int j = 0; j < pc.nt; ++j) {
            const int g = w.g0 + j, st = g % C::kRawStages, use = g / C::kRawStages;
            if (j > 0 && (j & 3) == 0) { ids_cur = ids_next; ids_next = load_ids((j >> 2) + 1); }
            const int phys = __shfl_sync(0xffffffffu, ids_cur, (j & 3) * 8 + (lane & 7));
            if (!waited && (p.early == 1 || (p.early == 3 && (pc.tile0 + j + 1) * kTileTokens > pc.n))) {
                wait_prior_launch();
                waited = true;
                if (bad_early) atomicOr(p.status, FD_DEV_BAD_PAGE);
            }
            if (!wait_all(&f4->raw_empty[st], (use & 1) ^ 1, abort)) { ok = false; break; }
            const int npg = min(8, (pc.kv_len - (pc.tile0 + j) * kTileTokens + 15) >> 4);
            if (lane == 0) mbar_arrive_expect_tx(&f4->raw_full[st], npg * C::kRawPage);
            __syncwarp();
            if (lane < 8 && phys >= 0)
                bulk_load_hint(raw + st * C::kRawBytes + lane * C::kRawPage, p.kvq + fp4_page_offset(phys, p.Hkv, pc.kvh, 0, D), C::kRawPage,
                               &f4->raw_full[st], policy);
            issued = g + 1;
        }
        w.advance(pc);
    }
    if (*abort) {  // drain copies still in flight before the shared memory is given back
        for (int g = max(0, issued - C::kRawStages); g < issued; ++g) {
            const unsigned long long t0 = global_ns();
            for (uint32_t it = 0; it < kSpinLimit && global_ns() - t0 < kWaitLimitNs; ++it)
                if (mbar_try_wait(&f4->raw_full[g % C::kRawStages], (g / C::kRawStages) & 1)) break;
        }
    }
}

// FP8 load warp.  One TMA box a page brings the codes of K and V, as [8-token group][K, V][8 rows][d]: the groups of K then lie a
// fixed stride apart, as those of V do, and K is an operand of Q K^T as it stands.  (Two untiled copies a page, K and V apart, took half as
// long again in all: what a copy costs the TMA unit is mostly per copy.)  The scales, 16 bytes behind the codes of either,
// come by plain loads, a tile ahead.
template <int D, int MODE>
__device__ __forceinline__ void load_role_fp8(const CUtensorMap& tmap, const AttnParams& p, int n_rb, unsigned char* raw, WideShared* f4, const Range rg,
                                              int* bad, volatile int* abort) {
    using C = Cfg<D, MODE, FD_KV_FP8>;
    const int lane = threadIdx.x & 31, cta = blockIdx.x;
    int issued = 0;
    const uint64_t policy = make_policy_evict_first();
    const int s_c = rg.s_c, e_c = rg.e_c;
    Walk w = {s_c, 0, {0, 0}, 0, rg.first};
    bool ok = true, waited = !p.early;
    bool bad_early = false;
    // The scale of page (lane & 7) of K (lanes 0-7) or V (8-15).  A page that no token owns has 1: its scores are masked, but -inf times
    // a stale scale need not be -inf.
    auto load_scale = [&](int phys, int kvh) -> float {
        if (lane >= 16 || phys < 0) return 1.f;
        return __ldcg(reinterpret_cast<const float*>(p.kvq + fp8_block_offset(phys, p.Hkv, kvh, lane >> 3, D) + 16 * D));
    };
    while (w.t < e_c && ok) {
        const Piece pc = decode_piece(p, n_rb, w.t, s_c, e_c, cta, w.b);
        const int32_t* table = p.page_table + (long long)pc.b * p.max_pages;
        auto load_ids = [&](int batch) -> int {  // four tiles (32 pages, one per lane), one batch ahead
            const int j = batch * 4 + (lane >> 3);
            const int pos = ((pc.tile0 + j) * 8 + (lane & 7)) * 16;
            if (!(j < pc.nt && pos < pc.kv_len)) return -1;
            int id = table[pos >> 4];
            if ((unsigned)id >= (unsigned)p.num_pages) {  // never form an address from a bad id
                if (!waited && p.early >= 2) { wait_prior_launch(); waited = true; }
                if (waited) atomicOr(p.status, FD_DEV_BAD_PAGE); else bad_early = true;
                atomicOr(bad, 1 << (w.piece & 31));
                id = 0;
            }
            return id;
        };
        int ids_cur = load_ids(0), ids_next = load_ids(1);
        auto needs_wait = [&](int j) { return !waited && (p.early == 1 || (p.early == 3 && (pc.tile0 + j + 1) * kTileTokens > pc.n)); };
        float sc = 1.f;
        bool have = false;  // sc is the next tile's
        for (int j = 0; j < pc.nt; ++j) {
            const int g = w.g0 + j, st = g % C::kRawStages, use = g / C::kRawStages;
            if (j > 0 && (j & 3) == 0) { ids_cur = ids_next; ids_next = load_ids((j >> 2) + 1); }
            const int phys = __shfl_sync(0xffffffffu, ids_cur, (j & 3) * 8 + (lane & 7));
            if (needs_wait(j)) {
                wait_prior_launch();
                waited = true;
                if (bad_early) atomicOr(p.status, FD_DEV_BAD_PAGE);
            }
            const float now = have ? sc : load_scale(phys, pc.kvh);
            have = j + 1 < pc.nt && !needs_wait(j + 1);
            if (have) sc = load_scale(__shfl_sync(0xffffffffu, (j & 3) == 3 ? ids_next : ids_cur, ((j + 1) & 3) * 8 + (lane & 7)), pc.kvh);
            if (!wait_all(&f4->raw_empty[st], (use & 1) ^ 1, abort)) { ok = false; break; }
            const int npg = min(8, (pc.kv_len - (pc.tile0 + j) * kTileTokens + 15) >> 4);
            if (lane == 0) mbar_arrive_expect_tx(&f4->raw_full[st], npg * C::kRawPage);
            __syncwarp();
            if (lane < 8 && phys >= 0) tma_load_5d_hint(raw + st * C::kRawBytes + lane * C::kRawPage, &tmap, 0, 0, 0, 0, phys * p.Hkv + pc.kvh, &f4->raw_full[st], policy);
            if (lane < 16) f4->sc[g & 15][lane] = now;
            __syncwarp();
            if (lane == 0) mbar_arrive(&f4->raw_full[st]);
            issued = g + 1;
        }
        w.advance(pc);
    }
    if (*abort) {  // drain copies still in flight before the shared memory is given back
        for (int g = max(0, issued - C::kRawStages); g < issued; ++g) {
            const unsigned long long t0 = global_ns();
            for (uint32_t it = 0; it < kSpinLimit && global_ns() - t0 < kWaitLimitNs; ++it)
                if (mbar_try_wait(&f4->raw_full[g % C::kRawStages], (g / C::kRawStages) & 1)) break;
        }
    }
}

// One K or V tile: codes and scales -> fp16 in the layout the MMA reads (code * scale is exact: fd_fp4.cuh).  A thread
// widens 32 elements of a token at a time (16 bytes of codes, two scales, four 16-byte stores).  Four neighbouring lanes
// share a token, so the reads are contiguous; of a 16-byte store's eight lanes -- two tokens, four chunks -- the
// chunks of the upper half of d store their words in the order 2 3 0 1, which puts all eight on different banks.
// ZERO_TAIL: tokens at or beyond `valid` become zeros (no token owns them: they may hold a NaN, and 0 * NaN is not 0).
constexpr int kWidenThreads = 256;

template <int D>
struct RawWords {  // a thread's part of a tile; all of it is read before anything is stored (a store orders the reads behind it)
    // (The raw tile is given back only when these words have been widened and stored.  Given back as soon as the reads had been
    // issued, with nothing yet depending on them, one call in twelve on many short sequences found words of the next tile.  Why is
    // not established; the order as it is needs no more than that a store waits for the words it stores.)
    static constexpr int kChunks = D / 32;  // 32-element chunks of a token
    static constexpr int kPasses = kTileTokens * kChunks / kWidenThreads;
    uint4 codes[kPasses];
    uint32_t sc[kPasses];
    __device__ __forceinline__ void load(const unsigned char* raw) {
        constexpr int kRawPage = 2 * fp4_page_bytes(D);
        const int t = (int)threadIdx.x - 384, c = t % kChunks;
#pragma unroll
        for (int it = 0; it < kPasses; ++it) {
            const int tok = t / kChunks + it * (kWidenThreads / kChunks);
            const unsigned char* page = raw + (tok >> 4) * kRawPage;
            codes[it] = *reinterpret_cast<const uint4*>(page + (tok & 15) * (D / 2) + c * 16);
            sc[it] = *reinterpret_cast<const uint16_t*>(page + fp4_scale_offset(D) + (tok & 15) * (D / 16) + c * 2);
        }
    }
};

template <int D, bool ZERO_TAIL>
__device__ __forceinline__ void widen_tile(const RawWords<D>& in, unsigned char* tile, int valid) {
    constexpr int kChunks = RawWords<D>::kChunks;
    constexpr int kHalves = D / 64;
    const int t = (int)threadIdx.x - 384, c = t % kChunks;
    const bool swap = kHalves == 2 && (c & 2);
#pragma unroll
    for (int it = 0; it < RawWords<D>::kPasses; ++it) {
        const int tok = t / kChunks + it * (kWidenThreads / kChunks);
        const __half2 s2 = as_half2(e4m3x2_to_half((uint16_t)in.sc[it]));
        const __half2 s_lo = __half2half2(__low2half(s2)), s_hi = __half2half2(__high2half(s2));
        const bool dead = ZERO_TAIL && tok >= valid;
        const uint4 cd = in.codes[it];
        const uint32_t wd[4] = {swap ? cd.z : cd.x, swap ? cd.w : cd.y, swap ? cd.x : cd.z, swap ? cd.y : cd.w};
        const __half2 s01 = swap ? s_hi : s_lo, s23 = swap ? s_lo : s_hi;
        unsigned char* row = tile + (tok >> 3) * (kHalves * 1024) + (c >> 1) * 1024 + (tok & 7) * 128;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t h[4];
            e2m1x8_to_half(wd[k], h);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = dead ? 0u : as_u32(__hmul2(as_half2(h[i]), k < 2 ? s01 : s23));
            const int unit = (c & 1) * 4 + (swap ? k ^ 2 : k);
            *reinterpret_cast<uint4*>(row + ((unit ^ (tok & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        }
    }
}

// The V tile of 8-bit pages: 16 codes a thread and pass.
// Which of a pass's tokens, and which 16 codes of its row, are a thread's.  d = 128: of eight lanes that read or write together four
// have half a row of token x, four of token x ^ 5.  The swizzle of the raw rows puts their chunks c ^ x on all eight places of a
// 128-byte line, and that of the widened ones their units 2 c + k ^ x as well.  d = 64: two rows of four chunks.
template <int D>
struct V8Map {
    static constexpr int kTokens = kWidenThreads / (D / 16);  // of a pass
    static constexpr int kPasses = kTileTokens / kTokens;
    int tok, c;
    __device__ __forceinline__ V8Map() {
        const int t = (int)threadIdx.x - 384;
        if (D == 128) {
            const int x = (t >> 4) & 3;
            tok = (t >> 6) * 8 + ((t & 4) ? x ^ 5 : x);
            c = (t & 3) + ((t & 8) >> 1);
        } else {
            tok = t >> 2;
            c = t & 3;
        }
    }
};

template <int D>
struct RawV8 {
    uint4 codes[V8Map<D>::kPasses];
    __device__ __forceinline__ void load(const unsigned char* raw) {
        const V8Map<D> m;
        const int r = m.tok & 7;
        const unsigned char* row = raw + (m.tok >> 3) * (2 * 8 * D) + 8 * D + r * D + ((m.c ^ (D == 128 ? r : r >> 1)) << 4);  // (the swizzle of the box)
#pragma unroll
        for (int it = 0; it < V8Map<D>::kPasses; ++it) codes[it] = *reinterpret_cast<const uint4*>(row + it * (V8Map<D>::kTokens / 8) * (2 * 8 * D));
    }
};

// Tokens at or beyond `valid` become zeros, as codes: a second form of the loop below, run once a piece, would not be in the instruction
// cache when its turn comes (2.4 us where this takes 0.6).
template <int D>
__device__ __forceinline__ void widen_v8(RawV8<D>& in, const float* v_scales, unsigned char* tile, int valid) {
    constexpr int kHalves = D / 64;
    const V8Map<D> m;
    const int r = m.tok & 7, unit = (m.c & 3) * 2;
    unsigned char* row = tile + (m.tok >> 3) * (kHalves * 1024) + (m.c >> 2) * 1024 + r * 128;
    if (valid < kTileTokens) {
#pragma unroll
        for (int it = 0; it < V8Map<D>::kPasses; ++it)
            if (m.tok + it * V8Map<D>::kTokens >= valid) in.codes[it] = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int it = 0; it < V8Map<D>::kPasses; ++it) {
        const __half2 s2 = __float2half2_rn(v_scales[(m.tok + it * V8Map<D>::kTokens) >> 4]);  // (a power of two from 2^-15 on: exact)
        const uint32_t wd[4] = {in.codes[it].x, in.codes[it].y, in.codes[it].z, in.codes[it].w};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t h[4];
            e4m3x4_to_half(wd[2 * k], h[0], h[1]);
            e4m3x4_to_half(wd[2 * k + 1], h[2], h[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = as_u32(__hmul2(as_half2(h[i]), s2));
            *reinterpret_cast<uint4*>(row + it * (V8Map<D>::kTokens / 8) * (kHalves * 1024) + (((unit + k) ^ r) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
        }
    }
}

// The Q tile of a piece for K in e4m3: q = hi + lo, both e4m3, in place -- rows of d bytes, hi's 128 rows then lo's.  A row is
// multiplied by the power of two that brings its largest element into [2^7, 2^8).  hi keeps four of bf16's eight bits, what is left
// has at most four and e4m3 holds it exactly where the element is at least 2^-9 of the largest; below that q is off by at most
// half a step of e4m3's smallest, 2^-17 of the largest element.  Q K^T is then two products at twice the rate of one in fp16, and K
// needs no widening.  Rows no query owns become zeros, as in q_to_half.
// d / 16 neighbouring lanes share a row, 16 elements each.  d = 128: a row lands on itself, and a rolled loop takes four rows a warp at a time
// -- this runs once a piece, and straight-line code for it took 6 us out of a cold instruction cache.  d = 64: a row of 64 bytes
// lands on what were other rows, so all warps read before any writes.
template <int D>
__device__ __forceinline__ bool q_to_e4m3(unsigned char* sq, float* row_scale, float scale_log2e, int rows, uint64_t* q_read, uint32_t parity,
                                          volatile int* abort) {
    constexpr int kLanes = D / 16, kRows = kWidenThreads / kLanes, kPasses = kMaxRows / kRows;
    const int t = (int)threadIdx.x - 384, c = t % kLanes;
    uint4 v[D == 64 ? kPasses : 1][2];
    auto read = [&](int n, uint4 (&x)[2]) {
        const int r = t / kLanes + n * kRows;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = 2 * c + i;
            x[i] = r < rows ? *reinterpret_cast<const uint4*>(sq + r * 128 + (u >> 3) * (kMaxRows * 128) + (((u & 7) ^ (r & 7)) << 4)) : make_uint4(0, 0, 0, 0);
        }
    };
    auto write = [&](int n, const uint4 (&x)[2]) {
        const int r = t / kLanes + n * kRows;
        const uint32_t wd[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
        uint32_t mx = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) mx = __vmaxu2(mx, wd[k] & 0x7fff7fffu);
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) mx = __vmaxu2(mx, __shfl_xor_sync(0xffffffffu, mx, o));  // (and all lanes of the row have read)
        const int e = max((int)(max(mx & 0xffffu, mx >> 16) >> 7), 14);        // biased exponent of the largest magnitude
        const float f = __uint_as_float((uint32_t)(127 + 134 - e) << 23);      // 2^(134 - e), e in [14, 255]
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float x0 = __uint_as_float(wd[2 * k] << 16) * f, x1 = __uint_as_float(wd[2 * k] & 0xffff0000u) * f;
            const float x2 = __uint_as_float(wd[2 * k + 1] << 16) * f, x3 = __uint_as_float(wd[2 * k + 1] & 0xffff0000u) * f;
            hi[k] = to_e4m3x2(x0, x1) | to_e4m3x2(x2, x3) << 16;
            uint32_t a, b;
            e4m3x4_to_half(hi[k], a, b);
            const float2 ha = __half22float2(as_half2(a)), hb = __half22float2(as_half2(b));
            lo[k] = to_e4m3x2(x0 - ha.x, x1 - ha.y) | to_e4m3x2(x2 - hb.x, x3 - hb.y) << 16;
        }
        unsigned char* at = sq + r * D + ((c ^ (D == 128 ? r & 7 : (r & 7) >> 1)) << 4);
        *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(at + kMaxRows * D) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        // (as in q_to_half; a row with an infinity or a NaN: NaN, since e4m3 has no infinity to hold)
        if (c == 0) row_scale[r] = e == 255 ? __uint_as_float(0x7fffffffu) : fminf(fmaxf(scale_log2e * exp2f((float)(e - 134)), 1.17549435e-38f), 3.4028234e38f);
    };
    if (D == 128) {
#pragma unroll 1
        for (int n = 0; n < kPasses; ++n) {
            read(n, v[0]);
            write(n, v[0]);
        }
    } else {
#pragma unroll
        for (int n = 0; n < kPasses; ++n) read(n, v[D == 64 ? n : 0]);
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(q_read);
        if (!wait_all(q_read, parity, abort)) return false;
#pragma unroll
        for (int n = 0; n < kPasses; ++n) write(n, v[D == 64 ? n : 0]);
    }
    return true;
}

// The Q tile of a piece, bf16 -> fp16 in place, kPer neighbouring threads a row (of two, the second starts at unit 4 of its
// part: its words then lie on the other banks).  A row is multiplied by the power of two that brings its
// largest element into [2^14, 2^15): bf16's 8 bits then fit fp16 exactly down to 2^-31 of that element (below, the loss is
// smaller than what the fp32 sum of the score drops), and the factor goes into the scale of the row's scores.
// Rows at or beyond `rows` are no query's: they hold the next sequences' rows or what a launch before this one left there.  They
// become zeros, whose scores settle at once: scores that keep rising, or are NaN, would send the warp's real rows through the
// two-pass softmax tile after tile (one row on a prefix of 60 000, 8 kv-heads: 137 us instead of 112).
template <int D>
__device__ __forceinline__ void q_to_half(unsigned char* sq, float* row_scale, float scale_log2e, int rows) {
    constexpr int kPer = kWidenThreads / kMaxRows, kUnits = D / 8 / kPer;  // 16-byte units of a row, per thread
    static_assert(kPer == 2, "two threads a row");
    const int t = (int)threadIdx.x - 384, r = t / kPer, part = t % kPer;
    auto at = [&](int i) -> uint4* {  // the thread's i-th unit
        const int u = part * kUnits + (kPer == 2 && part && kUnits >= 8 ? i ^ 4 : i);
        return reinterpret_cast<uint4*>(sq + r * 128 + (u >> 3) * (kMaxRows * 128) + (((u & 7) ^ (r & 7)) << 4));
    };
    const bool live = r < rows;
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
        const uint4 v = live ? *at(i) : make_uint4(0, 0, 0, 0);
        mx = __vmaxu2(mx, __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
    }
    if (kPer == 2) mx = __vmaxu2(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    const int e = max((int)(max(mx & 0xffffu, mx >> 16) >> 7), 14);  // biased exponent of the largest magnitude
    const float f = __uint_as_float((uint32_t)(127 + 141 - e) << 23);  // 2^(141 - e), e in [14, 255]
#pragma unroll
    for (int i0 = 0; i0 < kUnits; i0 += 4) {  // four words in flight: a store in place orders the loads behind it
        uint4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = live ? *at(i0 + i) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t* wd = reinterpret_cast<uint32_t*>(&v[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                wd[k] = as_u32(__floats2half2_rn(__uint_as_float(wd[k] << 16) * f, __uint_as_float(wd[k] & 0xffff0000u) * f));
            *at(i0 + i) = v[i];
        }
    }
    // never 0 (a hidden score is -inf, and 0 * -inf is not): a score of at most 2^35 times 2^-126 is 0 for every purpose
    if (part == 0) row_scale[r] = fminf(fmaxf(scale_log2e * exp2f((float)(e - 141)), 1.17549435e-38f), 3.4028234e38f);
}

// FP4: the widening warps.  K runs one tile ahead of V (the MMA warp needs K j + 1 before V j), and the next piece's first K tile
// is widened before its Q is touched, while that Q is still on its way.
template <int D, int MODE>
__device__ __forceinline__ void widen_role_fp4(const AttnParams& p, unsigned char* sq, unsigned char* sk, unsigned char* sv,
                                           const unsigned char* raw, Bars* bars, WideShared* f4, const Piece* ring, const Range rg,
                                           volatile int* abort) {
    using C = Cfg<D, MODE, FD_KV_FP4>;
    const int lane = threadIdx.x & 31;
    Walk w = {rg.s_c, 0, {0, 0}, 0, rg.first};
    while (w.t < rg.e_c) {
        if (!__all_sync(0xffffffffu, wait_piece(bars, w.piece, abort))) return;
        const Piece pc = ring[w.piece & (C::kDescSlots - 1)];
        auto do_k = [&](int j) -> bool {
            const int g = w.g0 + j, rs = g % C::kRawStages, st = g % C::kStages;
            if (!wait_all(&f4->raw_full[rs], (g / C::kRawStages) & 1, abort)) return false;
            RawWords<D> in;
            in.load(raw + rs * C::kRawBytes);
            if (!wait_all(&bars->k_empty[st], ((g / C::kStages) & 1) ^ 1, abort)) return false;
            widen_tile<D, false>(in, sk + st * C::kKBytes, 0);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->k_full[st]);
            return true;
        };
        auto do_v = [&](int j) -> bool {
            const int g = w.g0 + j, rs = g % C::kRawStages, st = g % C::kStages;
            RawWords<D> in;  // (the tile has landed: do_k has waited for it)
            in.load(raw + rs * C::kRawBytes + fp4_page_bytes(D));
            if (!wait_all(&bars->v_empty[st], ((g / C::kStages) & 1) ^ 1, abort)) return false;
            const int valid = pc.kv_len - (pc.tile0 + j) * kTileTokens;
            if (valid >= kTileTokens) widen_tile<D, false>(in, sv + st * C::kKBytes, 0);
            else widen_tile<D, true>(in, sv + st * C::kKBytes, valid);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&bars->v_full[st]);
                mbar_arrive(&f4->raw_empty[rs]);  // here, where every word read has been used, and not behind the reads: see RawWords
            }
            return true;
        };
        if (!do_k(0)) return;
        if (!wait_all(&bars->q_full, w.piece & 1, abort)) return;
        q_to_half<D>(sq, f4->row_scale[w.piece & 3], p.scale_log2e, pc.rows);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&f4->q_ready);
        for (int j = 0; j < pc.nt; ++j) {
            if (j + 1 < pc.nt && !do_k(j + 1)) return;
            if (!do_v(j)) return;
        }
        w.advance(pc);
    }
}

// FP8: the widening warps turn Q into two e4m3 tiles and widen V; K is read as it is.
template <int D, int MODE>
__device__ __forceinline__ void widen_role_fp8(const AttnParams& p, unsigned char* sq, unsigned char* sv, const unsigned char* raw, Bars* bars,
                                               WideShared* f4, const Piece* ring, const Range rg, volatile int* abort) {
    using C = Cfg<D, MODE, FD_KV_FP8>;
    const int lane = threadIdx.x & 31;
    Walk w = {rg.s_c, 0, {0, 0}, 0, rg.first};
    while (w.t < rg.e_c) {
        if (!__all_sync(0xffffffffu, wait_piece(bars, w.piece, abort))) return;
        const Piece pc = ring[w.piece & (C::kDescSlots - 1)];
        if (!wait_all(&bars->q_full, w.piece & 1, abort)) return;
        if (!q_to_e4m3<D>(sq, f4->row_scale[w.piece & 3], p.scale_log2e, pc.rows, &f4->q_read, w.piece & 1, abort)) return;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&f4->q_ready);
        for (int j = 0; j < pc.nt; ++j) {
            const int g = w.g0 + j, rs = g % C::kRawStages, st = g % C::kStages;
            if (!wait_all(&f4->raw_full[rs], (g / C::kRawStages) & 1, abort)) return;
            RawV8<D> in;
            in.load(raw + rs * C::kRawBytes);
            if (!wait_all(&bars->v_empty[st], ((g / C::kStages) & 1) ^ 1, abort)) return;
            const int valid = pc.kv_len - (pc.tile0 + j) * kTileTokens;
            widen_v8<D>(in, &f4->sc[g & 15][8], sv + st * C::kKBytes, valid);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&bars->v_full[st]);
                mbar_arrive(&f4->raw_empty[rs]);  // (where every word read has been used: see RawWords)
            }
        }
        w.advance(pc);
    }
}

// A segment's ragged last tile: V rows no token owns may hold NaN or stale data -- P is 0 there, but 0 * NaN is not.
// The warp that is about to issue the tile's P V zeroes them (the tile has landed) and fences the writes for the MMA.
template <class C>
__device__ __forceinline__ void zero_v_tail(unsigned char* vt, int valid, int lane) {
    if (valid >= kTileTokens) return;
    const int nbad = kTileTokens - valid;
    for (int e = lane; e < nbad * 8 * C::kHalves; e += 32) {
        const int r = valid + e / (8 * C::kHalves), wd = e % (8 * C::kHalves);
        *reinterpret_cast<uint4*>(vt + (r >> 3) * C::kGroupBytes + (wd >> 3) * 1024 + (r & 7) * 128 + ((wd & 7) << 4)) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
    __syncwarp();
}

// MMA issuing warp.
template <int D, int MODE, int FMT>
__device__ __forceinline__ void mma_role(const AttnParams& p, unsigned char* sq, unsigned char* sk, unsigned char* sv, Bars* bars,
                                         WideShared* f4, const Piece* ring, uint32_t tmem, const Range rg, volatile int* abort) {
    using C = Cfg<D, MODE, FMT>;
    const int lane = threadIdx.x & 31;
    constexpr uint32_t idesc_qk = wide(FMT) ? make_idesc_f16(128, kTileTokens, false) : make_idesc_bf16(128, kTileTokens, false);
    constexpr uint32_t idesc_pv = make_idesc_bf16(128, D, true);
    const uint32_t col_s[2] = {0u, 128u}, col_o[2] = {256u, 384u};
    const bool group_pv = wide(FMT) || pv_by_group<MODE>(rg.e_c - rg.s_c);  // wide formats: pv_role_wide
    if (p.early == 1) wait_prior_launch();  // (this role touches shared and tensor memory only; p.early >= 2 lets it run ahead)
    const uint64_t qd0 = FMT == FD_KV_FP8 ? make_smem_desc(smem_u32(sq), 16, 8 * D, D == 128 ? 2 : 4) : make_smem_desc(smem_u32(sq), 16, 1024);
    const int s_c = rg.s_c, e_c = rg.e_c;
    Walk w = {s_c, 0, {0, 0}, 0, rg.first};
    bool ok = true;
    while (w.t < e_c && ok) {
        if (!__all_sync(0xffffffffu, wait_piece(bars, w.piece, abort))) break;
        const Piece pc = ring[w.piece & (C::kDescSlots - 1)];
        if (!wait_all(wide(FMT) ? &f4->q_ready : &bars->q_full, w.piece & 1, abort)) break;
        auto issue_pv = [&](int jj) {  // (ranges whose P V this warp issues: see kGroupPvMinTiles)
            const int gg = w.g0 + jj, s = jj & 1, st = gg % C::kStages, u = w.u_base[s] + (jj >> 1);
            if (!wait_all(&bars->v_full[st], (gg / C::kStages) & 1, abort)) { ok = false; return; }
            unsigned char* vt = sv + st * C::kKBytes;
            zero_v_tail<C>(vt, pc.kv_len - (pc.tile0 + jj) * kTileTokens, lane);
            // the first P V of a stream in a piece overwrites O: the previous piece's epilogue must have read it
            if (jj < 2 && w.piece > 0 && !wait_all(&bars->o_free, (w.piece - 1) & 1, abort)) { ok = false; return; }
            // (descriptors are made before the last wait: what follows it is the MMA instructions alone.  The address
            // field of a descriptor is its low 14 bits, in 16-byte units, so a K step is an addition.)
            const uint64_t vd0 = make_smem_desc(smem_u32(vt), 1024, C::kGroupBytes);
            if (!wait_all(&bars->p_full[s], u & 1, abort)) { ok = false; return; }
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < kTileTokens / 16; ++kk)
                    // one page per K step: its two 8-token groups lie kGroupBytes apart, the two halves of d 1 KB apart
                    umma_ts(tmem + col_o[s], tmem + col_s[s] + kk * 8, vd0 + (uint64_t)((kk * C::kPageBytes) >> 4), idesc_pv, jj >= 2 || kk > 0);
                umma_commit(&bars->v_empty[st]);
                umma_commit(&bars->pv_done[s]);
            }
            __syncwarp();
        };
        for (int j = 0; j < pc.nt && ok; ++j) {
            const int g = w.g0 + j, st = g % C::kStages, use = g / C::kStages;
            const int s = j & 1;
            const int rs = g % (wide(FMT) ? C::kRawStages : 1);  // FP8: the raw stage that holds K
            if (FMT == FD_KV_FP8 ? !wait_all(&f4->raw_full[rs], (g / (wide(FMT) ? C::kRawStages : 1)) & 1, abort) : !wait_all(&bars->k_full[st], use & 1, abort)) { ok = false; break; }
            // S_s is written over P_s (its first 64 columns), which the P V of tile j - 2 of this stream reads, and
            // nothing orders two MMAs with different accumulators but the completion of the first: Q K^T waits for
            // that P V's completion barrier.  (FD_QK_MODE 0 drops the wait, relying on one thread's MMAs executing in
            // issue order: 3-5 % faster, but not a documented guarantee; kept for measurements only.  Tried as well:
            // Q K^T as two N = 64 halves with only the aliasing half behind the wait, 11 % slower; issuing whichever
            // MMA is ready first from a polling loop, 8 % slower -- the polling warp takes issue slots from the
            // softmax warps of its scheduler.)
            [[maybe_unused]] const int u_prev = w.u_base[s] + (j >> 1) - 1;  // the stream's previous tile, over all pieces
            const uint64_t kd0 = FMT == FD_KV_FP8 ? make_smem_desc(smem_u32(sk + rs * C::kRawBytes), 16, 16 * D, D == 128 ? 2 : 4)
                                                  : make_smem_desc(smem_u32(sk + st * C::kKBytes), 16, C::kGroupBytes);
#if FD_QK_MODE != 0
            if (!wide(FMT) && u_prev >= 0 && !wait_all(&bars->pv_done[s], u_prev & 1, abort)) { ok = false; break; }
#endif
            if (wide(FMT) && g >= 3 && !wait_all(&f4->pv_done[g % 3], ((g - 3) / 3) & 1, abort)) { ok = false; break; }
            const uint32_t s_col = wide(FMT) ? (uint32_t)(g % 3) * 128u : col_s[s];
            tc_fence_after();
            if (elect_one()) {
                if constexpr (FMT == FD_KV_FP8) {
                    constexpr uint32_t idesc = make_idesc_e4m3(128, kTileTokens);
#pragma unroll
                    for (int kk = 0; kk < 2 * (D / 32); ++kk) {  // hi's products, then lo's
                        const int step = kk % (D / 32) * 32;
                        umma_ss_f8(tmem + s_col, qd0 + (uint64_t)((kk / (D / 32) * (kMaxRows * D) + step) >> 4), kd0 + (uint64_t)(step >> 4), idesc, kk > 0);
                    }
                } else
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    constexpr int kQHalf = kMaxRows * 128;
                    umma_ss(tmem + s_col, qd0 + (uint64_t)(((kk >> 2) * kQHalf + (kk & 3) * 32) >> 4),
                            kd0 + (uint64_t)(((kk >> 2) * 1024 + (kk & 3) * 32) >> 4), idesc_qk, kk > 0);
                }
                umma_commit(FMT == FD_KV_FP8 ? &f4->raw_empty[rs] : &bars->k_empty[st]);
                umma_commit(wide(FMT) ? &f4->s_full[g % 3] : &bars->s_full[s]);
                if (j == pc.nt - 1) umma_commit(&bars->q_free);  // the next piece's Q may come in
            }
            __syncwarp();
            if (!group_pv && j >= 1) issue_pv(j - 1);
        }
        if (!group_pv && ok) issue_pv(pc.nt - 1);
        w.advance(pc);
    }
}

// Wide formats: the warp that issues P V, in tile order (they add into one O; and Q K^T of the tiles ahead does not stand behind them).
template <int D, int MODE, int FMT>
__device__ __forceinline__ void pv_role_wide(unsigned char* sv, Bars* bars, WideShared* f4, const Piece* ring, uint32_t tmem, const Range rg,
                                            volatile int* abort) {
    using C = Cfg<D, MODE, FMT>;
    constexpr uint32_t idesc = make_idesc_f16(128, D, true);
    Walk w = {rg.s_c, 0, {0, 0}, 0, rg.first};
    while (w.t < rg.e_c) {
        if (!__all_sync(0xffffffffu, wait_piece(bars, w.piece, abort))) return;
        const int nt = ring[w.piece & (C::kDescSlots - 1)].nt, v = ring[w.piece & (C::kDescSlots - 1)].v;
        for (int j = 0; j < nt; ++j) {
            const int g = w.g0 + j, st = g % C::kStages, b = g % 3;
            if (!wait_all(&bars->v_full[st], (g / C::kStages) & 1, abort)) return;
            // the first P V of a piece overwrites O: the previous piece's epilogue must have read it
            if (j == 0 && w.piece > 0 && !wait_all(&bars->o_free, (w.piece - 1) & 1, abort)) return;
            const uint64_t vd0 = make_smem_desc(smem_u32(sv + st * C::kKBytes), 1024, C::kGroupBytes);
            if (!wait_all(&f4->p_full[b], (g / 3) & 1, abort)) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < kTileTokens / 16; ++kk)
                    umma_ts(tmem + 384u, tmem + b * 128u + kk * 8, vd0 + (uint64_t)((kk * C::kPageBytes) >> 4), idesc, j > 0 || kk > 0);
                umma_commit(&bars->v_empty[st]);
                umma_commit(&f4->pv_done[b]);
            }
            __syncwarp();
        }
        w.g0 += nt;
        w.t += nt;
        w.b = v;
        ++w.piece;
    }
}

// ---------------------------------------------------------------------------------------------
// One cluster per segment (kTcCluster).  The CTAs of a cluster split the segment's tiles evenly.  Query row r of the
// segment is owned by CTA r / share of the cluster (share = ceil(128 / cluster size)).  Every CTA writes the
// unnormalised partial result of the rows it does not own -- O in fp32 and (m, l) -- to its two scratch slots in
// global memory, one block per owner, keeps the rows it owns in registers, and after ONE cluster barrier each owner
// brings the c - 1 blocks meant for it into its shared memory with bulk copies, combines them with its own part in
// rank order (fixed, so the result does not depend on timing) and writes the bf16 rows.  The cluster is there for the
// barrier and the co-scheduling; the bytes go through L2, because that is the faster carrier: an SM stores 64 KB to
// global memory in 0.9 us and a bulk copy lands it in 0.3 us, while the SM-to-SM path moved the same rows at about
// 20 GB/s per SM (3.5-5 us), with st.shared::cluster pushes as with ld.shared::cluster pulls.  No counters, no polling.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_ctarank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {  // every thread of every CTA of the cluster
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
constexpr int kMaxCluster = 16;
// Rows a CTA of a cluster of c owns (the last CTA may own fewer, or none).
__host__ __device__ constexpr int cluster_share(int c) { return (kMaxRows + c - 1) / c; }
// What one CTA hands one owner: the O rows as [d / 4 words][share rows][16 bytes], then (m, l) per row.
__host__ __device__ constexpr uint32_t cluster_block_bytes(int c, int d) { return (uint32_t)((cluster_share(c) * (d * 4 + 8) + 15) / 16 * 16); }
// Do the two scratch slots of a CTA, and the K ring where the blocks land, hold the c blocks of a cluster of c?
// (Wide formats: the K and V rings, which lie side by side and are both idle by then.)
__host__ __device__ constexpr bool cluster_fits(int c, int d, bool wide_format) {
    return (uint32_t)c * cluster_block_bytes(c, d) <= 2u * kMaxRows * d * 4 &&
           (uint32_t)c * cluster_block_bytes(c, d) <= (uint32_t)(wide_format ? (d == 128 ? 4 : 8) : (d == 128 ? 3 : 6)) * kTileTokens * d * 2;
}

// Addresses of the exchange.  In global memory: CTA `cta` of the grid owns scratch slots 2 cta and 2 cta + 1, one block
// per owner rank.  In shared memory: after the cluster barrier the K ring (idle by then) takes the c blocks meant for
// this CTA, block c from rank c; its own block it has written there itself.
template <int D>
struct Exchange {
    unsigned char* g_base;  // scratch of this CTA
    unsigned char* land;    // the K ring (generic address)
    uint32_t land_s;        // ... and its shared-memory address
    int share;
    uint32_t block;
    __device__ __forceinline__ unsigned char* g_block(int dest) const { return g_base + (size_t)dest * block; }
    __device__ __forceinline__ static uint32_t o_off(int share_, int rl, int word) { return (uint32_t)(word * share_ + rl) * 16; }
    __device__ __forceinline__ uint32_t ml_off(int rl) const { return (uint32_t)share * D * 4 + (uint32_t)rl * 8; }
};

// Owner side, after the cluster barrier: warp 0 brings the peers' blocks in, a lane per peer.
template <int D>
__device__ __forceinline__ void cluster_fetch(const AttnParams& p, const Exchange<D>& ex, Bars* bars, int rank) {
    const int C = p.cluster, c = threadIdx.x & 31;
    if (c == 0) mbar_arrive_expect_tx(&bars->merge_bar, (uint32_t)(C - 1) * ex.block);
    __syncwarp();
    if (c < C && c != rank) {
        fence_proxy_async_all();  // the peers' plain stores, acquired at the barrier, before the bulk copy that reads them
        const long long cta_stride = (long long)2 * kMaxRows * D * 4;  // two scratch slots per CTA
        bulk_load(ex.land + (size_t)c * ex.block, ex.g_base + (c - rank) * cta_stride + (long long)rank * ex.block, ex.block, &bars->merge_bar);
    }
}

// Owner side, once the blocks have landed: the eight warps of the softmax groups share the rows this CTA owns, a row
// per D / 4 lanes, a lane per 16-byte word (its 8-byte bf16 stores form one contiguous run per row).  Lane c of a row's
// group holds part c's (m, l) and weight, handed round by shuffles; the c parts are combined in rank order.
template <int D>
__device__ __forceinline__ void cluster_reduce(const AttnParams& p, const Exchange<D>& ex, int rank, int rows, int kvh, int row0) {
    constexpr int kLpr = D / 4;              // lanes per row (>= the largest cluster)
    constexpr int kRowsPerWarp = 32 / kLpr;
    static_assert(kLpr >= kMaxCluster, "one lane per part");
    const int C = p.cluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int word = lane % kLpr;
    const int r_lo = rank * ex.share, n_own = min(ex.share, rows - r_lo);  // rows [r_lo, r_lo + n_own) are this CTA's
    for (int rl0 = 0; rl0 < n_own; rl0 += 8 * kRowsPerWarp) {              // uniform over the warp: it shuffles
        const int rl = rl0 + warp * kRowsPerWarp + lane / kLpr;
        const bool act = rl < n_own;
        const int rl_c = act ? rl : 0;
        float2 q = make_float2(-INFINITY, 0.f);
        if (act && word < C) q = *reinterpret_cast<const float2*>(ex.land + (size_t)word * ex.block + ex.ml_off(rl_c));
        float m = q.x;
        int flagged = q.y < 0.f;  // some CTA of the cluster met a page id outside the pool (it sent l < 0)
#pragma unroll
        for (int o = kLpr / 2; o > 0; o >>= 1) {
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o, kLpr));
            flagged |= __shfl_xor_sync(0xffffffffu, flagged, o, kLpr);
        }
        const float w = q.x == -INFINITY ? 0.f : exp2f(q.x - m);  // a part that saw no visible key for the row counts nothing
        float l = w * q.y;
#pragma unroll
        for (int o = kLpr / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o, kLpr);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        const unsigned char* o0 = ex.land + Exchange<D>::o_off(ex.share, rl_c, word);
        for (int c0 = 0; c0 < C; c0 += 4) {
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const float4*>(o0 + (size_t)min(c0 + k, C - 1) * ex.block);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float wc = __shfl_sync(0xffffffffu, w, min(c0 + k, C - 1), kLpr);
                if (c0 + k < C && wc != 0.f) {  // (by selection: the O rows of a part without weight may hold anything)
                    acc.x += wc * v[k].x; acc.y += wc * v[k].y; acc.z += wc * v[k].z; acc.w += wc * v[k].w;
                }
            }
        }
        if (!act) continue;
        float inv = l > 0.f ? p.out_scale / l : 0.f;
        if (flagged) {  // by assignment: what came from a stand-in page may be inf or NaN
            inv = 0.f;
            acc = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        const int r = r_lo + rl;
        __nv_bfloat16* dst = p.out + ((long long)(row0 + r / p.G) * p.Hq + kvh * p.G + r % p.G) * D + word * 4;
        __align__(8) __nv_bfloat162 v2[2] = {__floats2bfloat162_rn(acc.x * inv, acc.y * inv), __floats2bfloat162_rn(acc.z * inv, acc.w * inv)};
        *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(v2);
    }
}

// Merge of a split segment from shared memory (the merger at the last piece of its range, when the Q tile and the
// rings are idle).  The staging area holds kRound O arrays of partial slots ([D / 4][128 rows][4 floats]) and behind
// them the (m[128], l[128]) pairs: first this CTA's own, then those of the n_other other pieces in CTA order.  The O
// arrays come in rounds of kRound pieces (bulk copies issued by thread 0 through issue_round, completion on merge_bar);
// this CTA's own piece -- the own_pos-th of the segment in CTA order -- is in registers (own: the thread's D / 2
// columns).  Same arithmetic, same order as merge_row: the result does not depend on who merges.  Called by all 256
// threads of the softmax groups (it holds barriers); `active`: the thread has a row to write.
template <int D, int MODE, int FMT>
struct Stage {
    static constexpr uint32_t kBytes = Cfg<D, MODE, FMT>::kQBytes + 2 * Cfg<D, MODE, FMT>::kStages * Cfg<D, MODE, FMT>::kKBytes;
    static constexpr uint32_t kPieceBytes = kMaxRows * D * 4;
    static constexpr int kRound = (kBytes - 8192) / kPieceBytes;
    static constexpr uint32_t kMlOffset = kRound * kPieceBytes;
    static constexpr int kMaxOthers = (kBytes - kMlOffset) / (2 * kMaxRows * 4) - 1;
};

template <int D, int MODE, int FMT, class IssueRound>
__device__ __forceinline__ void merge_staged(const AttnParams& p, Bars* bars, const unsigned char* stage, int n_other, int own_pos,
                                             const float* own, int r, int cg, bool active, bool bad, int kvh, int row0,
                                             volatile int* abort, IssueRound issue_round) {
    using S = Stage<D, MODE, FMT>;
    constexpr int CW = D / 2;
    const float* ml = reinterpret_cast<const float*>(stage + S::kMlOffset);  // [1 + n_other][2][128]
    float acc[CW];
#pragma unroll
    for (int c = 0; c < CW; ++c) acc[c] = 0.f;
    float m = -INFINITY, l = 0.f;
    auto add_own = [&]() {
        const float mp = ml[r], lp = ml[kMaxRows + r];
        const float w = (mp == -INFINITY) ? 0.f : exp2f(mp - m);
        l += w * lp;
#pragma unroll
        for (int k = 0; k < CW; ++k) acc[k] += w * own[k];
    };
    for (int round = 0, k0 = 0;; ++round, k0 += S::kRound) {
        if (!wait_all(&bars->merge_bar, round & 1, abort)) return;  // uniform: every thread sees the same outcome or leaves
        if (round == 0 && active) {
            m = ml[r];
            for (int k = 0; k < n_other; ++k) m = fmaxf(m, ml[(1 + k) * 2 * kMaxRows + r]);
        }
        const int k1 = min(n_other, k0 + S::kRound);
        if (active) {
            for (int k = k0; k < k1; ++k) {
                if (k == own_pos) add_own();
                const float mp = ml[(1 + k) * 2 * kMaxRows + r], lp = ml[(1 + k) * 2 * kMaxRows + kMaxRows + r];
                const float w = (mp == -INFINITY) ? 0.f : exp2f(mp - m);
                l += w * lp;
                const float4* o = reinterpret_cast<const float4*>(stage + (size_t)(k - k0) * S::kPieceBytes) + ((cg * CW) >> 2) * kMaxRows + r;
#pragma unroll
                for (int q = 0; q < CW / 4; ++q) {
                    const float4 v = o[q * kMaxRows];
                    acc[4 * q] += w * v.x;
                    acc[4 * q + 1] += w * v.y;
                    acc[4 * q + 2] += w * v.z;
                    acc[4 * q + 3] += w * v.w;
                }
            }
        }
        if (k1 == n_other) break;
        named_bar_sync(1, 256);  // everyone has read this round's O arrays: the next round may land on them
        if (threadIdx.x == 0) issue_round(round + 1);
    }
    if (!active) return;
    if (own_pos == n_other) add_own();
    __nv_bfloat16* dst = p.out + ((long long)(row0 + r / p.G) * p.Hq + kvh * p.G + r % p.G) * D + cg * CW;
    if (bad) {  // a page id of this sequence was bad: defined output, zeros (by assignment)
#pragma unroll
        for (int c = 0; c < CW; ++c) acc[c] = 0.f;
        store_cols_bf16<CW>(dst, acc, 0.f);
        return;
    }
    store_cols_bf16<CW>(dst, acc, p.out_scale / l);
}

// Two weights in the 16-bit type of the P V product.
template <int FMT>
__device__ __forceinline__ uint32_t pack16(float2 v) {
    if (wide(FMT)) return as_u32(__floats2half2_rn(v.x, v.y));
    const __nv_bfloat162 b = __floats2bfloat162_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&b);
}

// One row of a tile in the kernel of the wide formats.  Both groups add into one O (three S / P buffers instead of two and a second
// accumulator: a group then finds its next S ready, where the chain softmax -> P V -> Q K^T of its own buffer used to stand
// between two of its tiles), so a row's reference -- what its scores are taken against -- is shared by the two threads of
// the row, and its changes have to follow the order of the tiles: a tile settles its reference after the tile before it
// has (decided), and stores its weights only then.  The reference is raised when a score passes it by more than the
// threshold, which is rare, so the weights are formed beforehand against the reference as it stands and only kept --
// packed, half the size of the scores -- if nothing has changed.  Otherwise, and in the first tile of a piece (no
// reference yet) and the tiles the mask cuts, S is gone over twice: for the maximum, then for the weights, written as
// they are formed (a chunk's weights only ever land on scores that have been read).
// m, l: the reference and the sum of this thread's weights so far.
// FP8: S stands for the codes of K, page_scale holds what the 16 columns of each page are multiplied by.
template <int D, int FMT>
__device__ __forceinline__ void softmax_tile_wide(uint32_t s_addr, uint32_t o_addr, float c, float head, const float* page_scale, bool masked, int lim, int blo, int bhi,
                                                 int j, volatile float* ref, uint64_t* decided_before, uint32_t before_parity, uint64_t* decided,
                                                 uint64_t* pv_before, uint32_t pv_parity, volatile int* abort, float& m, float& l) {
    const int lane = threadIdx.x & 31;
    float ps[FMT == FD_KV_FP8 ? 8 : 1];
    if (FMT == FD_KV_FP8) {
#pragma unroll
        for (int k = 0; k < 8; k += 4) *reinterpret_cast<float4*>(ps + k) = *reinterpret_cast<const float4*>(page_scale + k);
    }
    // the largest of a chunk's scores, whose first page is `page`
    auto take_max = [&](const auto& sv, float& a, float& b, [[maybe_unused]] int page) {
        constexpr int N = sizeof(sv) / 4;
        if constexpr (FMT == FD_KV_FP8) {
#pragma unroll
            for (int k0 = 0; k0 < N; k0 += 16) {
                float x = -INFINITY, y = -INFINITY;
#pragma unroll
                for (int k = k0; k < k0 + 16; k += 4) {
                    x = max3(x, __uint_as_float(sv[k]), __uint_as_float(sv[k + 1]));
                    y = max3(y, __uint_as_float(sv[k + 2]), __uint_as_float(sv[k + 3]));
                }
                a = fmaxf(a, fmaxf(x, y) * ps[page + k0 / 16]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                a = max3(a, __uint_as_float(sv[k]), __uint_as_float(sv[k + 1]));
                b = max3(b, __uint_as_float(sv[k + 2]), __uint_as_float(sv[k + 3]));
            }
        }
    };
    auto weights = [&](const auto& x, float2 c2, float2 nm2, float2& sum0, float2& sum1, uint32_t* pk, [[maybe_unused]] int page) {
#pragma unroll
        for (int k = 0; k < (int)(sizeof(x) / 4); k += 4) {
            if (FMT == FD_KV_FP8 && k % 16 == 0) c2 = make_float2(c * ps[page + k / 16], c * ps[page + k / 16]);
            const float2 xa = __ffma2_rn(make_float2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), c2, nm2);
            const float2 xb = __ffma2_rn(make_float2(__uint_as_float(x[k + 2]), __uint_as_float(x[k + 3])), c2, nm2);
            const float2 pa = make_float2(ex2_approx(xa.x), ex2_approx(xa.y)), pb = make_float2(ex2_approx(xb.x), ex2_approx(xb.y));
            sum0 = __fadd2_rn(sum0, pa);
            sum1 = __fadd2_rn(sum1, pb);
            pk[k >> 1] = pack16<true>(pa);
            pk[(k >> 1) + 1] = pack16<true>(pb);
        }
    };
    auto rebase = [&](float to) {  // this thread's sum, from the reference it was formed against
        if (m != to) {
            l = __fmul_rn(l, m == -INFINITY ? 0.f : exp2f(m - to));  // (rounded by itself: both passes below then add to the same)
            m = to;
        }
    };
    const float2 c2 = make_float2(c, c);
    float now = *ref;
    bool slow = masked || __any_sync(0xffffffffu, now == -INFINITY);  // (warp-uniform: masked is)
    if (!slow) {
        const float2 nm2 = make_float2(-now, -now);
        float a = -INFINITY, b = -INFINITY;
        float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
        uint32_t pk[2][32], sv[2][16];
        tmem_ld16(s_addr, sv[0]);
#pragma unroll
        for (int ch = 0; ch < 8; ++ch) {
            tc_wait_ld();
            if (ch < 7) tmem_ld16(s_addr + (ch + 1) * 16, sv[(ch + 1) & 1]);
            take_max(sv[ch & 1], a, b, ch);
            weights(sv[ch & 1], c2, nm2, sum0, sum1, &pk[ch >> 2][(ch & 3) * 8], ch);
        }
        if (j > 0) (void)wait_all(decided_before, before_parity, abort);  // (an abort is acted upon by the caller's next wait)
        slow = __any_sync(0xffffffffu, *ref != now || fmaxf(a, b) * c - head > now + kRescaleThreshold);
        if (!slow) {
            if (lane == 0) mbar_arrive(decided);
            tmem_st32(s_addr, pk[0]);
            tmem_st32(s_addr + 32, pk[1]);
            rebase(now);
            l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
        }
    } else if (j > 0) {
        (void)wait_all(decided_before, before_parity, abort);
    }
    if (slow) {
        now = *ref;
        auto low_bits = [](int n) -> uint32_t { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; };
        auto load = [&](int ch, uint32_t (&sv)[32]) {
            tmem_ld32(s_addr + ch * 32, sv);
            tc_wait_ld();
            if (masked) {  // the columns of the chunk the row sees, as a bit each
                const uint32_t vis = low_bits(lim - ch * 32) | (low_bits(bhi - ch * 32) & ~low_bits(blo - ch * 32));
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (!((vis >> k) & 1u)) sv[k] = 0xff800000u;  // -inf by select: S may be NaN there
            }
        };
        // (these loops are not unrolled, and registers have no index: the chunk's two scales are read again)
        auto reload_scales = [&]([[maybe_unused]] int ch) {
            if constexpr (FMT == FD_KV_FP8) {
                const float2 two = *reinterpret_cast<const float2*>(page_scale + 2 * ch);
                ps[0] = two.x;
                ps[1] = two.y;
            }
        };
        float a = -INFINITY, b = -INFINITY;
#pragma unroll 1
        for (int ch = 0; ch < 4; ++ch) {
            uint32_t sv[32];
            load(ch, sv);
            reload_scales(ch);
            take_max(sv, a, b, 0);
        }
        const float m_new = fmaxf(a, b) * c - head;
        float alpha = 1.f, to = now;
        if (now == -INFINITY) {
            to = m_new;  // nothing accumulated yet (O is overwritten, or exactly zero)
        } else if (m_new > now + kRescaleThreshold) {
            alpha = exp2f(now - m_new);
            to = m_new;
        }
        if (j > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
            // every P V before this tile's has completed once the last one has, and this tile's waits for its weights
            (void)wait_all(pv_before, pv_parity, abort);
            tc_fence_after();
#pragma unroll 1
            for (int ch = 0; ch < D / 16; ++ch) {
                uint32_t o[16];
                tmem_ld16(o_addr + ch * 16, o);
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                tmem_st16(o_addr + ch * 16, o);
            }
            tc_wait_st();
        }
        if (to != now) *ref = to;
        __syncwarp();
        if (lane == 0) mbar_arrive(decided);
        rebase(to);
        const float mc = (to == -INFINITY) ? 0.f : to;
        const float2 nm2 = make_float2(-mc, -mc);
        float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
#pragma unroll 1
        for (int ch = 0; ch < 4; ++ch) {
            uint32_t sv[32], pk[16];
            load(ch, sv);
            reload_scales(ch);
            weights(sv, c2, nm2, sum0, sum1, pk, 0);
            tmem_st16(s_addr + ch * 16, pk);
        }
        l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
    }
    tc_wait_st();
}

// The two softmax groups (256 threads).
template <int D, int MODE, int FMT>
__device__ __forceinline__ void softmax_role(const AttnParams& p, Bars* bars, float* ex, int* s_cs, const CtaStarts cs, const Piece* ring,
                                             uint32_t tmem, const Range rg, const Exchange<D> exch, int cl_rank, unsigned char* stage,
                                             unsigned char* sv, WideShared* f4, volatile int* abort) {
    using C = Cfg<D, MODE, FMT>;
    constexpr uint32_t idesc_pv = make_idesc_bf16(128, D, true);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    const int s_c = rg.s_c, e_c = rg.e_c;
    const int s = warp >> 2;                  // stream
    const int r = (warp & 3) * 32 + lane;     // query row == TMEM lane
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t col_s[2] = {0u, 128u}, col_o[2] = {wide(FMT) ? 384u : 256u, 384u};
    int chain = 0;                            // wide formats: tiles this warp's rows have been through, both groups' (phase of decided)
    float c = p.scale_log2e;  // (wide formats: of this row and piece, from the conversion of q)
    // The wide formats hold P in fp16: everything is scaled by 2^7, so that weights between 2^-21 and, with the deferred rescaling, 2^15 keep
    // all of their bits; m carries the factor, so sums, partials and merges need not know
    constexpr float kHead = wide(FMT) ? 7.f : 0.f;
    // fill the window of range starts; the barrier below orders it before its first use
    if (MODE == kTcPlanned && tid < kCsWindow) {  // (a call that plans for itself has filled it while planning)
        const int cc = cs.base + tid;
        s_cs[tid] = (cc >= 0 && cc <= p.n_ctas) ? cs.g[cc] : 0;
    }
    bool cl_synced = false;
    // before any global write of this role (scratch, counters, out).  p.early == 2: the tiles of the first piece may be
    // worked through meanwhile -- tensor and shared memory only -- and the wait comes before its ticket and epilogue
    if (p.early == 1) wait_prior_launch();
    bool prior_done = p.early < 2;
    const bool group_pv = pv_by_group<MODE>(e_c - s_c);
    Walk w = {s_c, 0, {0, 0}, 0, 0};
    while (w.t < e_c) {
        // one thread waits for the descriptor, so that all 256 take the same decision
        if (tid == 0) bars->piece_ok = wait_piece(bars, w.piece, abort);
        named_bar_sync(1, 256);
        if (!bars->piece_ok) break;
        if (tid == 0 && bars->bad && w.piece > 0) atomicAnd(&bars->bad, ~(1 << ((w.piece - 1) & 31)));  // (all 256 threads are past that piece)
        const Piece pc = ring[w.piece & (C::kDescSlots - 1)];
        const bool warp_active = (warp & 3) * 32 < pc.rows;
        const int i = r / p.G;
        const RowMask rm = row_mask(pc.i0 + i, pc.n, pc.Lq, pc.M, pc.nb, r < pc.rows);
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        // Warps whose 32 rows are all padding do nothing per tile: warp 0 of the group (always active)
        // arrives on p_full for them, and they wait at the epilogue's hardware barrier, not by polling.
        const int n_idle_threads = 32 * (4 - min(4, (pc.rows + 31) >> 5));

        if constexpr (wide(FMT)) {
            for (int j = s; j < pc.nt && warp_active; j += 2) {
                const int g = w.g0 + j, b3 = g % 3, e = chain + j;
                if (!wait_all(&f4->s_full[b3], (g / 3) & 1, abort)) { ok = false; break; }
                tc_fence_after();
                if (j < 2) c = f4->row_scale[w.piece & 3][r];
                const int pos0 = (pc.tile0 + j) * kTileTokens;
                // masked: the tile reaches into the query block (or past kv_len): the row's mask applies, in tile-local columns
                softmax_tile_wide<D, FMT>(tmem + lane_base + b3 * 128u, tmem + lane_base + 384u, c, kHead, f4->sc[g & 15], pos0 + kTileTokens > pc.n, rm.limit - pos0,
                                    rm.blk_lo - pos0, rm.blk_hi - pos0, j, &f4->ref[w.piece & 1][r], &f4->decided[warp & 3][(e - 1) & 1],
                                    (uint32_t)((e - 1) >> 1) & 1u, &f4->decided[warp & 3][e & 1], &f4->pv_done[(g + 2) % 3], (uint32_t)((g - 1) / 3) & 1u,
                                    abort, m, l);
                tc_fence_before();
                mbar_arrive(&f4->p_full[b3]);
                if ((warp & 3) == 0 && lane == 0 && n_idle_threads) mbar_arrive_cnt(&f4->p_full[b3], n_idle_threads);
            }
            if (warp_active) chain += pc.nt;
        }
        for (int j = s; j < pc.nt && warp_active && !wide(FMT); j += 2) {
            const int u = w.u_base[s] + (j >> 1);
            if (!wait_all(&bars->s_full[s], u & 1, abort)) { ok = false; break; }
            tc_fence_after();
            {
                const int pos0 = (pc.tile0 + j) * kTileTokens;
                // tile reaches into the query block (or past kv_len): the row's mask applies, in tile-local columns
                const bool masked = pos0 + kTileTokens > pc.n;
                const int lim = rm.limit - pos0, blo = rm.blk_lo - pos0, bhi = rm.blk_hi - pos0;
                const uint32_t s_addr = tmem + lane_base + col_s[s];

                // ---- the whole row of S in one round trip: TMEM loads queue behind the MMAs in flight,
                //      so every ld -> wait pair costs up to one MMA tile; registers come from setmaxnreg
                uint32_t sv[4][32];
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_addr + ch * 32, sv[ch]);
                tc_wait_ld();
                if (masked) {
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch)
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (ch * 32 + k >= lim && (ch * 32 + k < blo || ch * 32 + k >= bhi)) sv[ch][k] = 0xff800000u;  // -inf by select: S may be NaN there
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};  // three-input max: 64 instructions per row
#pragma unroll
                for (int ch = 0; ch < 4; ++ch)
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {
                        mx[0] = max3(mx[0], __uint_as_float(sv[ch][k]), __uint_as_float(sv[ch][k + 1]));
                        mx[1] = max3(mx[1], __uint_as_float(sv[ch][k + 2]), __uint_as_float(sv[ch][k + 3]));
                        mx[2] = max3(mx[2], __uint_as_float(sv[ch][k + 4]), __uint_as_float(sv[ch][k + 5]));
                        mx[3] = max3(mx[3], __uint_as_float(sv[ch][k + 6]), __uint_as_float(sv[ch][k + 7]));
                    }
                const float m_new = fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c);
                float alpha = 1.f;
                if (j < 2 || m == -INFINITY) {
                    m = m_new;  // nothing accumulated yet (O is overwritten, or exactly zero)
                } else if (m_new > m + kRescaleThreshold) {
                    alpha = exp2f(m - m_new);
                    m = m_new;
                }
                if (__any_sync(0xffffffffu, alpha != 1.f)) {
                    // previous PV of this stream has completed (S/P buffer reuse orders it), so O is quiescent
#pragma unroll 1
                    for (int ch = 0; ch < D / 16; ++ch) {
                        uint32_t o[16];
                        tmem_ld16(tmem + lane_base + col_o[s] + ch * 16, o);
                        tc_wait_ld();
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                        tmem_st16(tmem + lane_base + col_o[s] + ch * 16, o);
                    }
                    l *= alpha;
                }

                // ---- P = exp2(S * c - m), row sum, bf16 P written over S (64 tokens -> 32 columns)
                const float mc = (m == -INFINITY) ? 0.f : m;
                const float2 c2 = make_float2(c, c), nm2 = make_float2(-mc, -mc);
                float2 sum0 = make_float2(0.f, 0.f), sum1 = make_float2(0.f, 0.f);
#pragma unroll
                for (int hp = 0; hp < 2; ++hp) {
                    uint32_t pk[32];
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        const float2 xa = __ffma2_rn(make_float2(__uint_as_float(sv[2 * hp][k]), __uint_as_float(sv[2 * hp][k + 1])), c2, nm2);
                        const float2 xb = __ffma2_rn(make_float2(__uint_as_float(sv[2 * hp + 1][k]), __uint_as_float(sv[2 * hp + 1][k + 1])), c2, nm2);
                        const float2 pa = make_float2(ex2_approx(xa.x), ex2_approx(xa.y));
                        const float2 pb = make_float2(ex2_approx(xb.x), ex2_approx(xb.y));
                        sum0 = __fadd2_rn(sum0, pa);
                        sum1 = __fadd2_rn(sum1, pb);
                        pk[k >> 1] = pack16<false>(pa);
                        pk[16 + (k >> 1)] = pack16<false>(pb);
                    }
                    tmem_st32(s_addr + hp * 32, pk);  // overwrites S columns that are already in registers
                }
                l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
                tc_wait_st();
            }
            tc_fence_before();
            mbar_arrive(&bars->p_full[s]);
            if ((warp & 3) == 0 && lane == 0 && n_idle_threads) mbar_arrive_cnt(&bars->p_full[s], n_idle_threads);
            if ((warp & 3) == 0 && group_pv) {
                // ---- P V of this tile, issued by warp 0 of the group itself as soon as the group's P is whole: the MMA
                //      warp issues Q K^T only and never stands between a finished P and its P V
                const int gg = w.g0 + j, st = gg % C::kStages;
                unsigned char* vt = sv + st * C::kKBytes;
                if (!wait_all(&bars->v_full[st], (gg / C::kStages) & 1, abort)) { ok = false; break; }
                zero_v_tail<C>(vt, pc.kv_len - (pc.tile0 + j) * kTileTokens, lane);
                // the first P V of a stream in a piece overwrites O: the previous piece's epilogue (both groups) must have read it
                if (j < 2 && w.piece > 0 && !wait_all(&bars->o_free, (w.piece - 1) & 1, abort)) { ok = false; break; }
                // (the address field of a descriptor is its low 14 bits, in 16-byte units, so a K step is an addition)
                const uint64_t vd0 = make_smem_desc(smem_u32(vt), 1024, C::kGroupBytes);
                if (!wait_all(&bars->p_full[s], u & 1, abort)) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < kTileTokens / 16; ++kk)
                        // one page per K step: its two 8-token groups lie kGroupBytes apart, the two halves of d 1 KB apart
                        umma_ts(tmem + col_o[s], tmem + col_s[s] + kk * 8, vd0 + (uint64_t)((kk * C::kPageBytes) >> 4), idesc_pv, j >= 2 || kk > 0);
                    umma_commit(&bars->v_empty[st]);
                    umma_commit(&bars->pv_done[s]);
                }
                __syncwarp();
            }
        }

        // ---- epilogue: merge the two streams, then final rows, or a partial plus -- if this CTA is the
        //      last one to deliver a piece of the segment -- the merge of all its partials.
        //      All 256 threads take every named barrier, whatever happened before; decisions that must be
        //      uniform (leave, merge) are taken by thread 0 alone and published through shared memory.
        // A piece of a split segment: who merges is settled by a ticket.  Thread 0 draws it as soon as its own last
        // tile is done -- the atomic's round trip then hides behind the rest of the piece -- and the CTA that draws
        // the last ticket of the segment is the merger: every other piece of the segment belongs to a CTA that has
        // drawn before it, hence is running and will deliver its partial without depending on anyone.  The merger
        // keeps its own part in registers, waits (bounded) for the others' delivery count, and combines.
        if (!prior_done) { wait_prior_launch(); prior_done = true; }  // (all 256 threads; returns at once when it has completed)
        const int seg_t0 = w.t - pc.tile0, seg_t1 = seg_t0 + pc.seg_nt;
        int c_first = cta, c_last = cta, n_pieces = 1, ticket = -1;  // (no ticket drawn: never the merger)
        int* seg_cnt = p.plan.seg_count + 2 * (pc.v * p.Hkv + pc.kvh);  // [0] tickets drawn, [1] partials delivered
        using St = Stage<D, MODE, FMT>;
        if (MODE != kTcCluster && !pc.complete) {
            segment_ctas(cs, p.n_ctas, cta, seg_t0, seg_t1, c_first, c_last);
            if (tid == 0 && !*abort) {
                n_pieces = segment_pieces(cs, c_first, c_last, seg_t0, seg_t1);
                ticket = atomicAdd(seg_cnt, 1);
            }
        }
        if (wide(FMT) && warp_active) {  // P V are issued in tile order by one warp: the last one has completed
            const int g_last = w.g0 + pc.nt - 1;
            ok = ok && wait_all(&f4->pv_done[g_last % 3], (g_last / 3) & 1, abort);
        }
        if (!wide(FMT) && warp_active) {  // every P V of the piece has completed: the last one of each stream
            ok = ok && wait_all(&bars->pv_done[0], (w.u_base[0] + ((pc.nt + 1) >> 1) - 1) & 1, abort);
            if (pc.nt >= 2) ok = ok && wait_all(&bars->pv_done[1], (w.u_base[1] + (pc.nt >> 1) - 1) & 1, abort);
        }
        tc_fence_after();
        const bool two = pc.nt >= 2 && !wide(FMT);
        // Stream exchange: group 1 hands its (m, l) to group 0, which answers with the two scale factors.
        // A thread only ever touches the two slots of its own row, so one barrier each way is enough.
        if (s == 1) { ex[r] = m; ex[kMaxRows + r] = l; }
        if (tid == 0) bars->epi_flag = (*abort ? 2 : 0) | ((MODE != kTcCluster && !pc.complete && ticket == n_pieces - 1) ? 1 : 0) | ((n_pieces - 1) << 8);
        named_bar_sync(1, 256);
        const bool leave = (bars->epi_flag & 2) != 0;
        const bool merger = (bars->epi_flag & 1) != 0;
        const bool stage_ok = merger && w.t + pc.nt == e_c && (bars->epi_flag >> 8) <= St::kMaxOthers;  // uniform: from shared memory
        float a0 = 0.f, a1 = 0.f, mm = -INFINITY, L = 0.f;
        if (s == 0) {
            if constexpr (wide(FMT)) {
                // one O, against the row's last reference; the two threads' sums are brought there
                const float m1 = ex[r], l1 = ex[kMaxRows + r];
                mm = f4->ref[w.piece & 1][r];
                f4->ref[(w.piece + 1) & 1][r] = -INFINITY;  // (the next piece's: the one before this has long been read)
                // (8 bits: a row whose scores are all NaN has kept m at -inf and has NaN in l; it goes on as a part that was seen)
                const float none = FMT == FD_KV_FP8 ? l : 0.f, none1 = FMT == FD_KV_FP8 ? l1 : 0.f;
                L = (m == -INFINITY ? none : exp2f(m - mm) * l) + (pc.nt < 2 ? 0.f : m1 == -INFINITY ? none1 : exp2f(m1 - mm) * l1);
                if (FMT == FD_KV_FP8 && L != L) mm = 0.f;
                a0 = 1.f;
            } else {
                const float m1 = two ? ex[r] : -INFINITY, l1 = ex[kMaxRows + r];
                mm = fmaxf(m, m1);
                a0 = (m == -INFINITY) ? 0.f : exp2f(m - mm);
                a1 = (m1 == -INFINITY) ? 0.f : exp2f(m1 - mm);
                L = a0 * l + (two ? a1 * l1 : 0.f);
            }
            if (pc.complete) { const float inv = p.out_scale / L; a0 *= inv; a1 *= inv; }
            ex[r] = a0;
            ex[kMaxRows + r] = a1;
        }
        named_bar_sync(1, 256);
        if (s == 1) { a0 = ex[r]; a1 = ex[kMaxRows + r]; }
        constexpr int kChunks = D / 64;  // 32-column chunks per softmax group
        const bool do_read = !leave && warp_active;
        // the load warps of this CTA have seen every page id of the piece by now (read where it is used: no register is held for it)
        auto bad_piece = [&]() { return (*static_cast<volatile int*>(&bars->bad) >> (w.piece & 31)) & 1; };
        const bool zero_rows = bad_piece();
        float o[kChunks][32];  // this thread's row, its group's half of the columns
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
            const int col = s * (D / 2) + ch * 32;
            if (do_read) {
                uint32_t o0[32], o1[32];
                tmem_ld32(tmem + lane_base + col_o[0] + col, o0);
                if (two) tmem_ld32(tmem + lane_base + col_o[1] + col, o1);
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    o[ch][k] = __uint_as_float(o0[k]) * a0;
                    if (two) o[ch][k] = fmaf(__uint_as_float(o1[k]), a1, o[ch][k]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 32; ++k) o[ch][k] = 0.f;
            }
            if (ch == kChunks - 1) {
                tc_fence_before();
                mbar_arrive(&bars->o_free);           // O has been read: the next piece may overwrite it
            }
            if (MODE == kTcCluster) {
                // one cluster per segment: a row another CTA owns goes to this CTA's scratch block for that owner, a row
                // this CTA owns to its own block in the K ring, idle since the last MMA (consecutive rows of a block
                // are consecutive 16-byte words: the warp's stores coalesce, and spread over the banks)
                const int dest = r / exch.share;
                if (do_read && r < pc.rows) {
                    unsigned char* blk = dest != cl_rank ? exch.g_block(dest) : exch.land + (size_t)cl_rank * exch.block;
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        *reinterpret_cast<float4*>(blk + Exchange<D>::o_off(exch.share, r % exch.share, (col + k) >> 2)) =
                            make_float4(o[ch][k], o[ch][k + 1], o[ch][k + 2], o[ch][k + 3]);
                }
            } else if (do_read && r < pc.rows) {
                if (pc.complete) {
                    __nv_bfloat16* dst = p.out + ((long long)(pc.row0 + i) * p.Hq + pc.kvh * p.G + r % p.G) * D + col;
                    if (zero_rows) {  // by assignment: what was computed from a stand-in page may be inf or NaN
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[ch][k] = 0.f;
                    }
                    store_cols_bf16<32>(dst, o[ch], 1.f);
                } else if (!merger) {
                    float4* dst = partial_o4(p.part, D, pc.slot, col, r);
#pragma unroll
                    for (int k = 0; k < 32; k += 4) dst[(k >> 2) * kMaxRows] = make_float4(o[ch][k], o[ch][k + 1], o[ch][k + 2], o[ch][k + 3]);
                }
            }
        }
        if (MODE == kTcCluster) {
            const int dest = r / exch.share, rl = r % exch.share;
            // (m, l) of the row for its owner (which may be this CTA: then into its own shared memory); a row this CTA
            // could not compute (it is giving up) counts as "saw no key"; a CTA whose load warps met a page id outside
            // the pool says so with a negative l
            if (r < pc.rows && s == 0) {
                const float2 ml = !do_read ? make_float2(-INFINITY, 0.f) : make_float2(mm, bad_piece() ? -1.f : L);
                unsigned char* blk = dest != cl_rank ? exch.g_block(dest) : exch.land + (size_t)cl_rank * exch.block;
                *reinterpret_cast<float2*>(blk + exch.ml_off(rl)) = ml;
            }
            cluster_sync_all();  // all 256 threads, whatever happened before; the other warps of the CTA wait in the kernel body
            cl_synced = true;
            // (the cluster barrier is a barrier of this CTA's threads as well: its own block in the K ring is complete)
            if (warp == 0) cluster_fetch<D>(p, exch, bars, cl_rank);
            if (wait_all(&bars->merge_bar, 0, abort) && !leave) cluster_reduce<D>(p, exch, cl_rank, pc.rows, pc.kvh, pc.row0);
        } else if (do_read && r < pc.rows && !pc.complete && s == 0) {
            // (the merger too: both column halves of its row need them, and only this thread has them)
            if (stage_ok) {
                float* own_ml = reinterpret_cast<float*>(stage + St::kMlOffset);
                own_ml[r] = mm;
                own_ml[kMaxRows + r] = L;
            } else {
                p.part.m[pc.slot * kMaxRows + r] = mm;
                p.part.l[pc.slot * kMaxRows + r] = L;
            }
        }
        if (MODE != kTcCluster && !pc.complete) {
            if (!merger) {
                // deliver: the barrier orders the partial stores of all threads before thread 0's fence, the fence
                // before the count.  Nobody waits for the count's result: the CTA goes straight on to its next piece.
                named_bar_sync(1, 256);
                if (tid == 0 && !leave && !*abort) {
                    __threadfence();
                    atomicAdd(seg_cnt + 1, bad_piece() ? 0x10001 : 1);  // (the upper half: pieces that met a page id outside the pool)
                }
            } else {
                if (tid == 0) {
                    // the n - 1 other pieces: all drawn before ours, so their CTAs are past their last tile
                    const unsigned long long t_start = global_ns();
                    bool there = false;
                    int bad = 0;
                    for (uint32_t it = 0; !there; ++it) {
                        int v;
                        asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(seg_cnt + 1) : "memory");
                        there = (v & 0xffff) >= n_pieces - 1;
                        bad = v >> 16;
                        if (!there && (it & 15u) == 15u && (*abort || global_ns() - t_start > kWaitLimitNs)) break;
                    }
                    if (there) {
                        seg_cnt[0] = 0;  // everyone has drawn and delivered: ready for the next call
                        seg_cnt[1] = 0;
                        // go (8: zeros); read after the barrier below, so that all 256 threads decide alike
                        bars->epi_flag |= 4 | ((bad | bad_piece()) != 0) << 3;
                    } else {
                        *abort = 1;
                    }
                }
                // At the last piece of the range the Q tile and the K and V rings are idle (every load of this CTA has
                // been consumed): the other pieces (m, l, and the O arrays in rounds) are brought there by bulk copies, all
                // of a round in flight together, and the merge reads shared memory.  Read straight from L2 the merge is
                // a chain of dependent round trips (row maxima, then piece after piece), each 1-2 us while the other SMs
                // still stream: measured 7-9 us for two or three pieces.
                auto issue_round = [&](int round) {  // thread 0
                    const int k0 = round * St::kRound, k1 = min(n_pieces - 1, k0 + St::kRound);
                    mbar_arrive_expect_tx(&bars->merge_bar, (uint32_t)(k1 - k0) * St::kPieceBytes + (round == 0 ? (uint32_t)(n_pieces - 1) * 2 * kMaxRows * 4 : 0u));
                    int k = 0;
                    for (int c = c_first; c <= c_last; ++c) {
                        const int sc = cs.at(c), ec = cs.at(c + 1);
                        if (c == cta || max(sc, seg_t0) >= min(ec, seg_t1)) continue;
                        const int slot = 2 * c + (sc >= seg_t0 ? 0 : 1);
                        if (round == 0) {
                            unsigned char* mlk = stage + St::kMlOffset + (size_t)(1 + k) * 2 * kMaxRows * 4;
                            bulk_load(mlk, p.part.m + slot * kMaxRows, kMaxRows * 4, &bars->merge_bar);
                            bulk_load(mlk + kMaxRows * 4, p.part.l + slot * kMaxRows, kMaxRows * 4, &bars->merge_bar);
                        }
                        if (k >= k0 && k < k1)
                            bulk_load(stage + (size_t)(k - k0) * St::kPieceBytes, p.part.o + (size_t)slot * (St::kPieceBytes / 4), St::kPieceBytes,
                                      &bars->merge_bar);
                        ++k;
                    }
                };
                if (tid == 0 && (bars->epi_flag & 4) && stage_ok) {
                    fence_proxy_async_all();
                    issue_round(0);
                    int own_pos = 0;
                    for (int c = c_first; c < cta; ++c) own_pos += max(cs.at(c), seg_t0) < min(cs.at(c + 1), seg_t1);
                    bars->epi_flag |= own_pos << 16;
                }
                named_bar_sync(1, 256);  // orders the acquire before every thread's loads of the partials
                const int rr = tid & (kMaxRows - 1), cg = tid >> 7;
                // rr == r and cg == s: the columns a thread merges are the ones it holds in registers
                if ((bars->epi_flag & 4) && !leave) {
                    if (!stage_ok) {
                        if (rr < pc.rows)
                            merge_row<D, D / 2>(p, cs, c_first, c_last, (bars->epi_flag & 8) != 0, pc.kvh, pc.row0, seg_t0, seg_t1, rr, cg, &o[0][0], cta);
                    } else {
                        merge_staged<D, MODE, FMT>(p, bars, stage, (int)((bars->epi_flag >> 8) & 0xff), (int)(bars->epi_flag >> 16), &o[0][0], rr, cg,
                                              rr < pc.rows, (bars->epi_flag & 8) != 0, pc.kvh, pc.row0, abort, issue_round);
                    }
                }
            }
        }
        if (leave) break;
        w.advance(pc);
    }
    // a CTA that gave up before its epilogue still owes the cluster its arrival: the peers must not wait for ever
    if (MODE == kTcCluster && !cl_synced) cluster_sync_all();
}

template <int D, int MODE, int FMT>
__global__ void __launch_bounds__(Cfg<D, MODE, FMT>::kThreads, 1) attn_tc_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap qmap,
                                                              const AttnParams p_in) {
    using C = Cfg<D, MODE, FMT>;
    extern __shared__ __align__(1024) unsigned char smem[];  // the swizzled tiles need 1024-byte alignment
    unsigned char* sq = smem;
    unsigned char* sk = smem + C::kQBytes;                      // K ring
    unsigned char* sv = smem + C::kVOffset;                     // V ring
    Bars* bars = reinterpret_cast<Bars*>(smem + C::kBarOffset);
    float* ex = reinterpret_cast<float*>(smem + C::kExOffset);
    int* s_cs = reinterpret_cast<int*>(smem + C::kCsOffset);
    SelfScans* scans = reinterpret_cast<SelfScans*>(smem + C::kScanOffset);
    RowBlock* rbs = reinterpret_cast<RowBlock*>(smem + C::kRbOffset);
    WideShared* f4 = reinterpret_cast<WideShared*>(smem + C::kWideOffset);  // wide formats only
    Piece* ring = wide(FMT) ? f4->ring : reinterpret_cast<Piece*>(smem + C::kDescOffset);
    volatile int* abort = &bars->abort;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if ((smem_u32(smem) & 1023u) != 0u) {  // uniform; cannot happen with the declared alignment: leave before any barrier
        if (tid == 0) atomicOr(p_in.status, FD_DEV_TIMEOUT);
        return;
    }

    // ---- set-up that needs nothing from earlier kernels: under programmatic dependent launch it overlaps the
    //      tail of the previous launch on the stream (the plan kernel, or the previous layer's call);
    //      griddepcontrol.wait below is where that launch's results are needed
    if (warp == 1 && lane == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(&bars->k_full[i], wide(FMT) ? C::kWidenWarps : 1); mbar_init(&bars->k_empty[i], 1);  // wide formats: the widening warps
            mbar_init(&bars->v_full[i], wide(FMT) ? C::kWidenWarps : 1); mbar_init(&bars->v_empty[i], 1);
        }
        if (wide(FMT)) {
            for (int i = 0; i < C::kRawStages; ++i) {  // FP8: codes and scales come apart; Q K^T reads a stage, too
                mbar_init(&f4->raw_full[i], FMT == FD_KV_FP8 ? 2 : 1);
                mbar_init(&f4->raw_empty[i], C::kWidenWarps + (FMT == FD_KV_FP8 ? 1 : 0));
            }
            mbar_init(&f4->q_ready, C::kWidenWarps);
            mbar_init(&f4->q_read, C::kWidenWarps);
            for (int i = 0; i < 3; ++i) { mbar_init(&f4->s_full[i], 1); mbar_init(&f4->p_full[i], 128); mbar_init(&f4->pv_done[i], 1); }
            for (int i = 0; i < 4; ++i) { mbar_init(&f4->decided[i][0], 1); mbar_init(&f4->decided[i][1], 1); }
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars->s_full[i], 1);
            mbar_init(&bars->p_full[i], 128);
            mbar_init(&bars->pv_done[i], 1);
        }
        mbar_init(&bars->q_full, 1);
        mbar_init(&bars->q_free, 1);
        mbar_init(&bars->o_free, 256);
        mbar_init(&bars->merge_bar, 1);
        bars->abort = 0;
        bars->epi_flag = 0;
        bars->desc_n = 0;
        bars->piece_ok = 0;
        bars->bad = 0;
        mbar_fence_init();
    }
    if (warp == kMmaWarp) tmem_alloc(&bars->tmem_base, 512);
    if (wide(FMT) && tid < 2 * kMaxRows) f4->ref[tid / kMaxRows][tid % kMaxRows] = -INFINITY;
    if (warp == kKWarp && lane == 0) { prefetch_tmap(&tmap); prefetch_tmap(&qmap); }
    // a call that plans for itself: warp 0 does so meanwhile (it needs the earlier kernels' results -- the lengths --
    // and waits for them on its own; its global loads then overlap the set-up of the other warps)
    if (MODE != kTcPlanned && warp == 0) {
        if (!p_in.early) wait_prior_launch();
        self_plan<MODE>(p_in, scans, rbs, s_cs, &bars->first);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    // a dependent launch behind this one (the next layer's call) may bring its CTAs in as ours retire and do its
    // own set-up; it waits for this grid to complete before reading anything
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // Everything below the plan needs the results of the launch before this one.  Under a pinned plan that launch is
    // normally the previous layer's call (p.early): it writes neither the plan nor the lengths nor the page table, so
    // the work of this CTA, its first piece and its first page ids are looked up while it still runs -- three to five
    // dependent L2 round trips, 2.4 us -- and each role waits for it just before its first access to anything else.
    if (!p_in.early) wait_prior_launch();

    // ---- the work of this CTA
    AttnParams p = p_in;
    const int cta = blockIdx.x;
    int total, n_rb, fatal;
    Range rg = {0, 0, 0};
    CtaStarts cs = {};
    cs.s = s_cs;
    cs.base = cta - kCsWindow / 2 + 1;
    int cl_rank = 0, cl_rows = 0, cl_b = 0, cl_kvh = 0, cl_row0 = 0;  // kTcCluster: this CTA's place and its segment
    bool cl_idle = false;
    if (MODE == kTcPlanned) {
        const PlanHeader hdr = *p.plan.hdr;
        total = hdr.total_tiles; n_rb = hdr.n_rb; fatal = hdr.fatal;
        if (total) { rg.s_c = p.plan.cta_start[cta]; rg.e_c = p.plan.cta_start[cta + 1]; rg.first = p.plan.cta_first[cta]; }
        cs.g = p.plan.cta_start;
    } else {
        p.plan.rb = rbs; p.plan.cu_q = scans->cu_q; p.plan.cu_tiles = scans->cu_tiles; p.plan.cu_ne = scans->cu_ne;
        n_rb = p.batch;
        fatal = scans->fatal;
        const int tiles = scans->cu_tiles[n_rb], nonempty = scans->cu_ne[n_rb];
        total = fatal ? 0 : tiles * p.Hkv;
        if (MODE == kTcSelfPlanned) {
            // the ranges the plan kernel would have cut (range_cut is shared with it and with the host)
            cs.ct = scans->cu_tiles; cs.ne = scans->cu_ne;
            cs.n_rb = n_rb; cs.Hkv = p.Hkv; cs.k = p.piece_cost; cs.total = total;
            cs.W = (long long)p.Hkv * (tiles + (long long)p.piece_cost * nonempty);
            cs.n_use = ranges_in_use(cs.W, p.piece_cost, p.min_range_tiles, p.n_ctas);
            if (total) { rg.s_c = s_cs[cta - cs.base]; rg.e_c = s_cs[cta + 1 - cs.base]; rg.first = bars->first; }
        } else {
            // segment = cluster number; the cluster's CTAs take equal shares of its tiles, in rank order
            const int seg = cta / p.cluster, v = seg / p.Hkv;
            cl_rank = (int)cluster_ctarank();
            cl_kvh = seg % p.Hkv;
            cl_b = v;
            cl_rows = rbs[v].Lq * p.G;
            cl_row0 = scans->cu_q[v];
            const int T = total ? scans->cu_tiles[v + 1] - scans->cu_tiles[v] : 0;
            const int t_base = p.Hkv * scans->cu_tiles[v] + cl_kvh * T;
            // (T <= 2^23 tiles and at most 16 ranks: the products fit 32 bits)
            rg.s_c = t_base + (int)((unsigned)T * (unsigned)cl_rank / (unsigned)p.cluster);
            rg.e_c = t_base + (int)((unsigned)T * (unsigned)(cl_rank + 1) / (unsigned)p.cluster);
            rg.first = v;
            cl_idle = rg.s_c >= rg.e_c && T > 0;  // peers have tiles: stay for the merge
        }
    }
    // Reading q and the cache ahead of the launch before this one pays where a call is short (its start and the tail
    // of the call before it overlap); a CTA with a long range gains nothing and only takes bandwidth from the
    // stragglers of that call, which everyone then waits for (measured: + 1.5 % on 222 tiles per CTA).
    if (p.early >= 2 && rg.e_c - rg.s_c > kEarlyLoadMaxTiles) p.early = 1;
    if (rg.s_c >= rg.e_c && !cl_idle) {  // uniform (over the cluster too): no tile for this CTA, or nothing at all
        if (p.early) wait_prior_launch();
        if (total == 0 && fatal) {  // inconsistent lengths: a defined output, zeros
            const long long n16 = (long long)p.total_q_rows * p.Hq * D / 8;
            uint4* o = reinterpret_cast<uint4*>(p.out);
            for (long long i2 = (long long)blockIdx.x * blockDim.x + threadIdx.x; i2 < n16; i2 += (long long)gridDim.x * blockDim.x)
                o[i2] = make_uint4(0, 0, 0, 0);
        }
        __syncthreads();
        if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
        return;
    }
    Exchange<D> exch = {};
    if (MODE == kTcCluster) {
        exch.g_base = reinterpret_cast<unsigned char*>(p.part.o) + (size_t)cta * 2 * kMaxRows * D * 4;
        exch.land = sk;
        exch.land_s = smem_u32(sk);
        exch.share = cluster_share(p.cluster);
        exch.block = cluster_block_bytes(p.cluster, D);
    }
    if (MODE == kTcCluster && cl_idle) {
        // fewer tiles than CTAs in the cluster: this one tells every owner "saw no key" and combines the rows it owns
        if (p.early) wait_prior_launch();
        if (tid < cl_rows) {
            const int dest = tid / exch.share, rl = tid % exch.share;
            unsigned char* blk = dest != cl_rank ? exch.g_block(dest) : exch.land + (size_t)cl_rank * exch.block;
            *reinterpret_cast<float2*>(blk + exch.ml_off(rl)) = make_float2(-INFINITY, 0.f);
        }
        cluster_sync_all();  // (a CTA-wide barrier as well: the own block is complete)
        if (warp == 0) cluster_fetch<D>(p, exch, bars, cl_rank);
        if (tid < 2 * kMaxRows) {  // whole warps: the wait is warp-uniform
            if (wait_all(&bars->merge_bar, 0, abort)) cluster_reduce<D>(p, exch, cl_rank, cl_rows, cl_kvh, cl_row0);
        }
    } else if (warp < 8) {
        // Warp-specialised register budgets: the softmax groups keep a whole 128-column row of S in registers.
        // 8 x 32 x 224 + 4 x 32 x 56 = 384 x 168, what the launch allocated: the increase is served exactly by what
        // the decrease released (a request for more than that does not return).
        // Wide formats: see Cfg.
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegSoftmax));
        softmax_role<D, MODE, FMT>(p, bars, ex, s_cs, cs, ring, tmem, rg, exch, cl_rank, sq, sv, f4, abort);
    } else {
        if (wide(FMT) && warp >= 12) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegWiden));
        }
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegHelper));
        if constexpr (wide(FMT)) {
            unsigned char* raw = smem + (FMT == FD_KV_FP8 ? C::kQBytes : C::kVOffset + C::kStages * C::kKBytes);
            if (warp == kKWarp) {
                if constexpr (FMT == FD_KV_FP8) load_role_fp8<D, MODE>(tmap, p, n_rb, raw, f4, rg, &bars->bad, abort);
                else load_role_fp4<D, MODE>(p, n_rb, raw, f4, rg, &bars->bad, abort);
            } else if (warp == kVWarp) pv_role_wide<D, MODE, FMT>(sv, bars, f4, ring, tmem, rg, abort);
            else if (warp >= 12) {
                if constexpr (FMT == FD_KV_FP8) widen_role_fp8<D, MODE>(p, sq, sv, raw, bars, f4, ring, rg, abort);
                else widen_role_fp4<D, MODE>(p, sq, sk, sv, raw, bars, f4, ring, rg, abort);
            }
        } else {
            if (warp == kKWarp) load_role<D, MODE>(tmap, p, n_rb, sk, bars->k_full, bars->k_empty, 0, rg, &bars->k_full[0], &bars->bad, abort);
            else if (warp == kVWarp) load_role<D, MODE>(tmap, p, n_rb, sv, bars->v_full, bars->v_empty, 1, rg, &bars->k_full[0], &bars->bad, abort);
        }
        if (warp == kMmaWarp) mma_role<D, MODE, FMT>(p, sq, sk, sv, bars, f4, ring, tmem, rg, abort);
        else if (warp == kQWarp) q_role<D, C::kDescSlots>(qmap, p, n_rb, sq, bars, ring, rg, abort);
        if (MODE == kTcCluster) cluster_sync_all();  // the cluster barrier of the merge counts every thread
    }
    // ---- common tail: everything of this CTA has completed, or it is giving up
    if (*abort && tid == 0) atomicOr(p.status, FD_DEV_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
}

struct TmapEntry {
    const void* ptr;
    int n;  // KV pool: pages; q: rows
    CUtensorMap map;
};

// Tensor maps already encoded, keyed by (pointer, extent).  A model calls the attention once per layer with that
// layer's pool and q buffer, in the same order every step: the entry after the last hit is tried first, then the
// whole list; the list grows with the number of distinct operands (one per layer) and is recycled round-robin
// only past kMaxEntries.
struct TmapCache {
    static constexpr size_t kMaxEntries = 4096;
    std::vector<TmapEntry> e;
    size_t last = 0, victim = 0;
    const CUtensorMap* find(const void* ptr, int n) {
        const size_t cnt = e.size();
        for (size_t k = 0; k < cnt; ++k) {
            const size_t i = (last + 1 + k) % cnt;
            if (e[i].ptr == ptr && e[i].n == n) { last = i; return &e[i].map; }
        }
        return nullptr;
    }
    TmapEntry& slot() {
        if (e.size() < kMaxEntries) { e.emplace_back(); last = e.size() - 1; return e.back(); }
        last = victim;
        victim = (victim + 1) % kMaxEntries;
        return e[last];
    }
};

struct TcState {
    PFN_cuTensorMapEncodeTiled_v12000 encode;
    TmapCache kv, kv8, q;
    int d, hkv;
    const CUtensorMap* current;
    const CUtensorMap* qcurrent;
    // per cache format (FD_KV_*): set up by its first call
    bool ready[3];
    int max_clusters[3][kMaxCluster + 1];  // [C]: clusters of C CTAs of the cluster kernel the device holds at once (0 = not launchable)
};

template <int D, int MODE, int FMT>
cudaError_t configure_kernel() {
    cudaError_t e = cudaFuncSetAttribute(attn_tc_kernel<D, MODE, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, MODE, FMT>::kSmemBytes);
    if (e == cudaSuccess && MODE == kTcCluster)
        e = cudaFuncSetAttribute(attn_tc_kernel<D, MODE, FMT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    // the register split draws on what the launch allocates: a request beyond that would wait for ever
    cudaFuncAttributes attr = {};
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&attr, attn_tc_kernel<D, MODE, FMT>);
    if (e == cudaSuccess && attr.numRegs * Cfg<D, MODE, FMT>::kThreads < Cfg<D, MODE, FMT>::kRegTotal) e = cudaErrorInvalidConfiguration;
    return e;
}

// How many clusters of `c` CTAs of the cluster kernel can be resident together (0 if such a launch is refused).
template <int D, int FMT>
int query_clusters(int c, int n_sms) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = c; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((n_sms / c) * c);
    cfg.blockDim = dim3(Cfg<D, kTcCluster, FMT>::kThreads);
    cfg.dynamicSmemBytes = Cfg<D, kTcCluster, FMT>::kSmemBytes;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, attn_tc_kernel<D, kTcCluster, FMT>, &cfg) != cudaSuccess) { cudaGetLastError(); return 0; }
    return n;
}

template <int D, int MODE, int FMT>
void launch_mode(const TcState* st, const AttnParams& p, cudaStream_t s) {
    // Programmatic dependent launch: the CTAs may start while the previous launch on the stream (the plan kernel,
    // or the previous layer's call) is still running; they do their set-up and then wait for it inside the kernel.
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.n_ctas);
    cfg.blockDim = dim3(Cfg<D, MODE, FMT>::kThreads);
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.dynamicSmemBytes = Cfg<D, MODE, FMT>::kSmemBytes;
    if (MODE == kTcCluster) {
        cfg.gridDim = dim3(p.batch * p.Hkv * p.cluster);  // one cluster per (sequence, kv-head) segment
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = p.cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cudaLaunchKernelEx(&cfg, attn_tc_kernel<D, MODE, FMT>, *st->current, *st->qcurrent, p);
}

template <int D, int FMT>
cudaError_t configure_format(TcState* st) {
    cudaError_t e = configure_kernel<D, kTcPlanned, FMT>();
    if (e == cudaSuccess) e = configure_kernel<D, kTcSelfPlanned, FMT>();
    if (e == cudaSuccess) e = configure_kernel<D, kTcCluster, FMT>();
    if (e != cudaSuccess) return e;
    int n_sms = 0, dev = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, dev);
    for (int c = 0; c <= kMaxCluster; ++c) st->max_clusters[FMT][c] = c >= 2 && cluster_fits(c, D, wide(FMT)) ? query_clusters<D, FMT>(c, n_sms) : 0;
    st->ready[FMT] = true;
    return cudaSuccess;
}

template <int D, int FMT>
void launch_format(const TcState* st, const AttnParams& p, int mode, cudaStream_t s) {
    if (mode == kTcCluster) launch_mode<D, kTcCluster, FMT>(st, p, s);
    else if (mode == kTcSelfPlanned) launch_mode<D, kTcSelfPlanned, FMT>(st, p, s);
    else launch_mode<D, kTcPlanned, FMT>(st, p, s);
}

}  // namespace

bool attn_tc_supported(int d, int G, int max_q_len) {
    (void)max_q_len;  // any length: a long query block is cut into row blocks of kMaxRows / G block rows
    return (d == 64 || d == 128) && G <= kMaxRows;
}

// Looks up (or encodes) the tensor map of this KV pool: a 4-D view [groups of 8 rows][d / 64 halves][8 rows][64]
// with a box of one page of one kv-head (two groups, both halves) and 128-byte swizzle.
cudaError_t attn_tc_prepare(void** state, const AttnParams& p) {
    TcState* st = static_cast<TcState*>(*state);
    if (!st) {
        st = new TcState();
        st->encode = nullptr;
        cudaDriverEntryPointQueryResult qres;
        cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", reinterpret_cast<void**>(&st->encode), cudaEnableDefault, &qres);
        if (e != cudaSuccess || !st->encode) { delete st; return e != cudaSuccess ? e : cudaErrorNotSupported; }
        st->d = p.d; st->hkv = p.Hkv;
        st->ready[0] = st->ready[1] = st->ready[2] = false;
        *state = st;
    }
    if (!st->ready[p.fmt]) {
        const cudaError_t e = p.d == 64 ? (p.fmt == FD_KV_FP8   ? configure_format<64, FD_KV_FP8>(st)
                                           : p.fmt == FD_KV_FP4 ? configure_format<64, FD_KV_FP4>(st)
                                                                : configure_format<64, FD_KV_BF16>(st))
                                        : (p.fmt == FD_KV_FP8   ? configure_format<128, FD_KV_FP8>(st)
                                           : p.fmt == FD_KV_FP4 ? configure_format<128, FD_KV_FP4>(st)
                                                                : configure_format<128, FD_KV_BF16>(st));
        if (e != cudaSuccess) return e;
    }
    // q: a 3-D view [T][Hq][d], box = 64 elements x G q-heads (one kv-head) x q_box_t block rows
    st->qcurrent = st->q.find(p.q, p.total_q_rows);
    if (!st->qcurrent) {
        CUtensorMap map;
        cuuint64_t dims[3] = {(cuuint64_t)p.d, (cuuint64_t)p.Hq, (cuuint64_t)(p.total_q_rows > 0 ? p.total_q_rows : 1)};
        cuuint64_t strides[2] = {(cuuint64_t)p.d * 2, (cuuint64_t)p.Hq * p.d * 2};
        cuuint32_t box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)p.q_box_t};
        cuuint32_t estr[3] = {1, 1, 1};
        const CUresult r = st->encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(p.q), dims, strides, box, estr,
                                      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (r != CUDA_SUCCESS) return cudaErrorInvalidValue;
        TmapEntry& e = st->q.slot();
        e.ptr = p.q;
        e.n = p.total_q_rows;
        e.map = map;
        st->qcurrent = &e.map;
    }
    if (p.fmt == FD_KV_FP4) {  // pages come by untiled bulk copies: no map of the pool (the kernel's first map goes unused)
        st->current = st->qcurrent;
        return cudaSuccess;
    }
    if (p.fmt == FD_KV_FP8) {
        // d bytes x 8 rows x (K, V) x two groups of 8 rows x (page, kv-head): a box is the codes of a page and head
        st->current = st->kv8.find(p.kvq, p.num_pages);
        if (st->current) return cudaSuccess;
        CUtensorMap map;
        const cuuint64_t block = (cuuint64_t)fp8_block_bytes(p.d);
        cuuint64_t dims[5] = {(cuuint64_t)p.d, 8, 2, 2, (cuuint64_t)p.num_pages * p.Hkv};
        cuuint64_t strides[4] = {(cuuint64_t)p.d, block, (cuuint64_t)p.d * 8, 2 * block};
        cuuint32_t box[5] = {(cuuint32_t)p.d, 8, 2, 2, 1};
        cuuint32_t estr[5] = {1, 1, 1, 1, 1};
        const CUresult r = st->encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, const_cast<unsigned char*>(p.kvq), dims, strides, box, estr,
                                      CU_TENSOR_MAP_INTERLEAVE_NONE, p.d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                      CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (r != CUDA_SUCCESS) return cudaErrorInvalidValue;
        TmapEntry& e = st->kv8.slot();
        e.ptr = p.kvq;
        e.n = p.num_pages;
        e.map = map;
        st->current = &e.map;
        return cudaSuccess;
    }
    st->current = st->kv.find(p.kv, p.num_pages);
    if (st->current) return cudaSuccess;
    // 64 elements x 8 rows x the 64-wide halves of d x groups of 8 rows: a box of two groups is one page of one
    // kv-head and lands as [group][half][8 rows][128 B]
    CUtensorMap map;
    cuuint64_t dims[4] = {64, 8, (cuuint64_t)p.d / 64, (cuuint64_t)p.num_pages * 2 * p.Hkv * 2};
    cuuint64_t strides[3] = {(cuuint64_t)p.d * 2, 128, (cuuint64_t)p.d * 2 * 8};
    cuuint32_t box[4] = {64, 8, (cuuint32_t)p.d / 64, 2};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    const CUresult r = st->encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<__nv_bfloat16*>(p.kv), dims, strides, box, estr,
                                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return cudaErrorInvalidValue;
    TmapEntry& e = st->kv.slot();
    e.ptr = p.kv;
    e.n = p.num_pages;
    e.map = map;
    st->current = &e.map;
    return cudaSuccess;
}

// CTAs per cluster for a call with one cluster per segment: the largest size (any, not only powers of two: a GPC holds
// a limited number of clusters of each size) for which all clusters of the call are resident together, so every SM it
// can use streams at once and a CTA has the fewest tiles; 0 if there is none.
int attn_tc_cluster_size(const void* state, int fmt, int n_segments, int n_sms) {
    const TcState* st = static_cast<const TcState*>(state);
    if (!st || n_segments <= 0) return 0;
    for (int c = kMaxCluster; c >= 2; --c)
        if (n_segments * c <= n_sms && st->max_clusters[fmt][c] >= n_segments) return c;
    return 0;
}

void launch_attn_tc(void* state, const AttnParams& p, int mode, cudaStream_t s) {
    if (p.batch == 0) return;
    const TcState* st = static_cast<const TcState*>(state);
    if (p.fmt == FD_KV_FP8) p.d == 64 ? launch_format<64, FD_KV_FP8>(st, p, mode, s) : launch_format<128, FD_KV_FP8>(st, p, mode, s);
    else if (p.fmt == FD_KV_FP4) p.d == 64 ? launch_format<64, FD_KV_FP4>(st, p, mode, s) : launch_format<128, FD_KV_FP4>(st, p, mode, s);
    else p.d == 64 ? launch_format<64, FD_KV_BF16>(st, p, mode, s) : launch_format<128, FD_KV_BF16>(st, p, mode, s);
}

void attn_tc_free(void* state) { delete static_cast<TcState*>(state); }

// Self-test of the bounded wait: one warp waits on an mbarrier that nothing will ever arrive on.
// The wait gives up after `limit_ns`, the kernel raises FD_DEV_TIMEOUT and returns normally.
__global__ void wait_timeout_selftest_kernel(int* status, unsigned long long limit_ns) {
    __shared__ uint64_t bar;
    __shared__ int abort_flag;
    if (threadIdx.x == 0) { mbar_init(&bar, 1); abort_flag = 0; mbar_fence_init(); }
    __syncthreads();
    const bool ok = mbar_wait_ns(&bar, 0, &abort_flag, limit_ns);
    __syncwarp();
    if (threadIdx.x == 0 && !ok) atomicOr(status, FD_DEV_TIMEOUT);
}

void launch_wait_timeout_selftest(int* status, unsigned long long limit_ns, cudaStream_t s) {
    wait_timeout_selftest_kernel<<<1, 32, 0, s>>>(status, limit_ns);
}

}  // namespace fd
