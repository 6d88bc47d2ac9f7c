// Causal attention of packed sequences on the tensor cores: the prompt on its way in.
//
// A CTA works on two row tiles at a time (fd_prompt.cuh), each a stream of its own: 128 query rows, a softmax warpgroup, S, P and O
// in tensor memory, an MMA-issuing warp.  Both streams read the same K and V tiles, brought in by TMA through one ring, so a tile's
// bytes serve 256 rows, and while one stream is in its softmax the tensor pipe works on the other.  Per tile and stream:
//     S = Q K^T      tcgen05.mma, Q and K from shared memory, S in tensor memory
//     P = exp2(..)   a thread a row: the row of S in registers, causal mask in the tiles the row's last key cuts, running maximum and
//                    sum in fp32; P goes to tensor memory in bf16 (V is bf16, and the operands of an MMA are of one type)
//     O += P V       A = P from tensor memory, B = V MN-major; O is rescaled only when a row's maximum has grown by more than 2^8
// S and P do not share columns, so S of the next tile is made as soon as the softmax has read this one's: a warpgroup finds it ready
// when it has written P, and the hand-overs (P -> product, product -> S, S -> softmax, 300 to 500 clocks each) run beside the
// exponentials.  At d = 128 that leaves room for tiles of 80 keys: two streams of S (80 columns), P (40) and O (128).  With
// tiles of 128 keys and P over S, a stream went through all of it once a tile, 5200 clocks of which the products are 1024.
// Roles: warps 0-3 and 4-7 softmax of streams 0 and 1, 8 K and V loads, 9 and 10 MMAs of streams 0 and 1, 11 Q loads, the
// descriptors of the items, which every role copies from a ring in shared memory, and the look through V tiles (below).
//
// Keys behind a row's last one get a weight of 0, but 0 times an infinity is not 0: in the tiles that the mask cuts for any row of the
// item a warp looks for values that are not finite among the keys some row must not see, puts zeros in their place, and the
// epilogue adds what each row does see of them.
//
// A call of few items (a short chunk behind a long prefix: 8 items for one of 64 tokens at 8 kv-heads) is split along the keys: `parts`
// CTAs share an item, each takes an equal share of its tiles and leaves (m, l, O) in scratch memory, which a second kernel combines in
// the order of the parts: 64 tokens behind 8128 take 25 us, where one CTA an item takes 125.  (Combined by the last CTA to deliver,
// one SM read what all had written, 54 us, and the code for it cost the softmax warps registers: 3 to 5 % on every other call.)  All items of
// a call are shared among the same number of CTAs, or none: from more than half as many items as CTAs on, none is (behind 3584 keys,
// 8 kv-heads: 512 tokens 48 us for a floor of 19, 640 74 for 25, 1200 121 for 50, 2048 154 for 93).
//
// What it reaches (32 heads over 8 of 128), in runs of 10 ms / call after call for seconds, when the power cap lowers the clock: a prompt
// of 32768 tokens 7.4 / 8.4 ms, 1.19 / 1.05 PFLOP/s, where the library's dense product of 8192 reaches 1.63 / 1.39 on the same machine;
// 8192 tokens 486 / 556 us, 1.13 / 0.99; 2048 44 / 45 us, 0.78 / 0.76; 16 ragged prompts of 100 to 4000 tokens 612 / 712 us; 17 tokens 8.4
// us.  What bounds it: 128 keys of a stream take 1880 clocks of a SM, in which the tensor pipe and the exponential
// unit are busy for 1024 each; in the rest both wait for hand-overs between a stream's softmax and its products, which two streams
// cover in part.  Short prompts wait besides for an item's ends (Q's load, the epilogue) that nothing overlaps.
// Tried and dropped (PFLOP/s at 32768 tokens, call after call, this form 1.05): a quarter of the exponentials by a polynomial on the FMA
// pipe 1.03, half of them 0.99; the next row of S loaded in front of P's stores 0.97; the streams' exponentials taking turns, no gain; one
// pass over S against a guessed maximum (spills: 8192 tokens 860 us, 584 without at that time); at d = 64 tiles of 96 keys (472 us for 406).
//
// Every wait is bounded: one that runs out raises a CTA-wide flag, the roles leave, copies in flight are drained, tensor memory is
// given back, FD_DEV_TIMEOUT is set.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <new>

#include "fd_attn_common.cuh"
#include "fd_prompt.cuh"

namespace fd {

using namespace sm100;

namespace {

constexpr int kPThreads = 384, kPRegSoftmax = 224, kPRegHelper = 56;
constexpr float kPRescale = 8.0f;  // log2 units
// Calls of at most this many sequences plan for themselves, a lane a sequence: the one warp that hands out items makes the scans and
// sorts (17 tokens: 8.4 us; with the plan kernel in front, which larger batches have, 13.8).
constexpr int kSelfBatch = 32;

template <int D>
struct PCfg {
    static constexpr int kKeys = D == 128 ? 80 : 128;         // keys of a tile
    static constexpr int kHalves = D / 64;
    static constexpr int kQBytes = kMaxRows * D * 2;          // one Q tile
    static constexpr int kQHalf = kMaxRows * 128;             // 64 elements of d of its rows
    static constexpr int kTileBytes = kKeys * D * 2;          // one K or V tile
    static constexpr int kHalfBytes = kKeys * 128;
    static constexpr int kStages = D == 128 ? 7 : 10;         // tiles in the ring: K and V in turn
    static constexpr int kOutOffset = 2 * kQBytes + kStages * kTileBytes;  // a softmax warp's 32 rows x 32 columns on their way out
    static constexpr int kBarOffset = kOutOffset + 8 * 2048;
    static constexpr int kSmemBytes = kBarOffset + 2048;
    // tensor memory, columns: S, P and O of stream s
    static constexpr uint32_t kStream = D == 128 ? 128 : 192;
    __device__ static constexpr uint32_t col_s(int s) { return s * kStream; }
    __device__ static constexpr uint32_t col_p(int s) { return s * kStream + kKeys; }
    __device__ static constexpr uint32_t col_o(int s) { return 2 * kStream + s * D; }
    static_assert(kKeys + kKeys / 2 <= kStream && 2 * kStream + 2 * D <= 512, "tensor memory");
    static_assert(kHalfBytes % 1024 == 0 && kSmemBytes <= 227 * 1024, "shared memory of one CTA");
};

// What the roles know of an item.  Keys are counted from the first one of this CTA's part.
struct ItemDesc {
    int kvh, row0, kv0, Lk;  // row0: the first output row of tile 0; kv-head -1: no more items
    int limit0;              // keys that token 0 of tile 0 sees
    int rows[2];             // query rows of the two tiles
    int tiles[2];            // key tiles they see
    int parts, pad;          // CTAs that share the item
};
// A part has at least kMinPartTiles tiles (64 tokens behind 936: 18.0 us, with at least four 19.4, unsplit 24.3); 16 parts at most (5
// tokens behind 14995: 23.6 us, at most eight 32.3).  Calls of fewer keys than kMinSplitTiles tiles hold are never split: the merge
// kernel is launched where the lengths, which are on the device, might ask for it, and costs 2 us (8 prompts of 40 tokens: 10.4 us
// without it, 12.4 with).
constexpr int kMaxParts = 16, kMinPartTiles = 2, kMinSplitTiles = 8;

struct PBars {
    uint64_t full[10], empty[10];
    uint64_t q_full[2], q_free[2], s_full[2], s_read[2], p_full[2], pv_done[2], o_free[2];
    uint64_t desc_full[4], desc_empty[4];
    uint64_t cut_full[8];  // a V tile that is to be looked through has landed; slot = number of such tiles & 7 (the ring holds five V tiles)
    ItemDesc desc[4];
    uint32_t tmem_base;
    int abort;
    unsigned odd[2];   // per stream, bit (item & 31): values that are not finite were taken out of a tile of the item
    int fatal;         // lengths inconsistent: no item is handed out, the output is zeros
    int plan[5 * kSelfBatch + 3];  // a call that plans for itself: its PromptPlan
};
static_assert(sizeof(PBars) <= 2048, "barriers, descriptors and the plan");

// A role's next item, copied from the ring.  Whole warps.
__device__ __forceinline__ bool next_item(PBars* bars, int n, ItemDesc& d, volatile int* abort) {
    if (!wait_all(&bars->desc_full[n & 3], (n >> 2) & 1, abort)) return false;
    d = bars->desc[n & 3];
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&bars->desc_empty[n & 3]);
    return d.kvh >= 0;
}

// Is V tile j of an item looked through before it is used?  Where the mask cuts it for a row of the item, or the sequence ends in it.
template <int D>
__device__ __forceinline__ bool is_cut(const ItemDesc& d, int j) { return (j + 1) * PCfg<D>::kKeys > min(d.limit0, d.Lk); }

// Looks through a V tile that has landed: of its rows [lo, valid), which some row of the item must not see, values that are not finite
// are reported to both streams and replaced by zeros; rows from `valid` on, another sequence's, become zeros.  One warp.
template <int D>
__device__ __forceinline__ void clean_tile(unsigned char* vt, int lo, int valid, PBars* bars, int item) {
    using C = PCfg<D>;
    const int lane = threadIdx.x & 31, n0 = lo * 8 * C::kHalves, n1 = min(valid, C::kKeys) * 8 * C::kHalves;
    auto at = [&](int e) -> uint4* {
        const int r = e / (8 * C::kHalves), w = e % (8 * C::kHalves);
        return reinterpret_cast<uint4*>(vt + (w >> 3) * C::kHalfBytes + r * 128 + (w & 7) * 16);
    };
    // bits 15 and 31: the element's exponent is all ones (its magnitude carries past 0x7f80)
    auto odd = [](uint32_t x) { return ((x & 0x7fff7fffu) + 0x00800080u) & 0x80008000u; };
    uint32_t any = 0;
#pragma unroll 4
    for (int e = n0 + lane; e < n1; e += 32) {
        const uint4 x = *at(e);
        any |= odd(x.x) | odd(x.y) | odd(x.z) | odd(x.w);
    }
    if (__any_sync(0xffffffffu, any != 0)) {
        if (lane < 2) atomicOr(&bars->odd[lane], 1u << (item & 31));
        auto keep = [&](uint32_t x) { const uint32_t o = odd(x) >> 15; return x & ~(o * 0xffffu); };
#pragma unroll 1
        for (int e = n0 + lane; e < n1; e += 32) {
            uint4 x = *at(e);
            *at(e) = make_uint4(keep(x.x), keep(x.y), keep(x.z), keep(x.w));
        }
    }
#pragma unroll 1
    for (int e = n1 + lane; e < C::kKeys * 8 * C::kHalves; e += 32) *at(e) = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    __syncwarp();
}

// The plan of a call of at most kSelfBatch sequences, by one warp.  Returns whether the lengths are consistent.
__device__ __forceinline__ bool self_plan_prompt(const PromptParams& p, PBars* bars, PromptPlan* pl) {
    const int lane = threadIdx.x & 31, B = p.batch;
    int* a = bars->plan;
    *pl = {a, a + kSelfBatch + 1, a + 2 * kSelfBatch + 2, a + 3 * kSelfBatch + 2, a + 4 * kSelfBatch + 2, nullptr};
    long long Lq = 0, Lk = 0;
    bool bad = false;
    if (lane < B) {
        Lq = p.q_lens[lane];
        Lk = p.kv_lens ? p.kv_lens[lane] : Lq;
        bad = Lq < 0 || Lk < 0;
    }
    long long sq = Lq, sk = Lk;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long uq = __shfl_up_sync(0xffffffffu, sq, o), uk = __shfl_up_sync(0xffffffffu, sk, o);
        if (lane >= o) { sq += uq; sk += uk; }
    }
    bad = __any_sync(0xffffffffu, bad) || __shfl_sync(0xffffffffu, sq, 31) != p.total_q || __shfl_sync(0xffffffffu, sk, 31) != p.total_kv;
    const int n = lane < B && !bad ? (int)((Lq + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens)) : -1;
    int rank = 0;  // sequences in front of this one: longer, or as long and earlier
#pragma unroll
    for (int o = 0; o < 32; ++o) {
        const int x = __shfl_sync(0xffffffffu, n, o);
        rank += x > n || (x == n && o < lane);
    }
    if (lane < B) {
        pl->cu_q[lane + 1] = (int)sq;
        pl->cu_kv[lane + 1] = (int)sk;
        pl->perm[rank] = lane;
        pl->blocks[rank] = n;
    }
    if (lane == 0) { pl->cu_q[0] = 0; pl->cu_kv[0] = 0; pl->pre[0] = 0; }
    __syncwarp();
    int pre = lane < B ? pl->blocks[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, pre, o);
        if (lane >= o) pre += u;
    }
    if (lane < B) pl->pre[lane + 1] = pre;
    __syncwarp();
    if (bad && lane == 0 && blockIdx.x == 0) atomicOr(p.status, FD_DEV_BAD_LENGTHS);
    return !bad;
}

template <int D>
__device__ __forceinline__ void prompt_q_role(const CUtensorMap& qmap, const PromptParams& p, unsigned char* sq, unsigned char* ring, PBars* bars, volatile int* abort) {
    using C = PCfg<D>;
    const int lane = threadIdx.x & 31;
    PromptPlan plan = p.plan;
    const bool fine = p.batch <= kSelfBatch ? self_plan_prompt(p, bars, &plan) : *p.plan.fatal == 0;
    if (!fine && lane == 0) bars->fatal = 1;
    const long long total = fine ? (long long)plan.pre[p.batch] * p.Hkv : 0;
    int turn = 0, loads[2] = {0, 0}, g = 0, cuts = 0, parts = 1;
    if (p.split && total > 0 && 2 * total <= gridDim.x) {  // (then at most that many sequences have items, the first in the plan's order)
        int longest = 0;
        for (int i = lane; i < min(p.batch, 1024); i += 32)
            if (plan.blocks[i] > 0) longest = max(longest, plan.cu_kv[plan.perm[i] + 1] - plan.cu_kv[plan.perm[i]]);
        longest = __reduce_max_sync(0xffffffffu, longest);
        const float tiles = (float)longest / C::kKeys;
        parts = max(1, min(min((int)(gridDim.x / total), (int)(tiles / kMinPartTiles)), kMaxParts));
    }
    if (p.split && blockIdx.x == 0 && lane == 0) *p.split = {parts, (int)total};
    // the next item, handed out; kv-head -1: there is none
    auto hand_out = [&](int n, ItemDesc& d) -> bool {
        long long t = parts > 1 ? (turn ? total : blockIdx.x / parts) : prompt_turn(turn, blockIdx.x, gridDim.x);
        while (parts == 1 && t >= total && (long long)turn * gridDim.x < total) t = prompt_turn(++turn, blockIdx.x, gridDim.x);
        ++turn;
        d = {-1, 0, 0, 0, 0, {0, 0}, {0, 0}, 1, 0};
        if (t < total) {
            const PromptItem it = prompt_item(plan, p.batch, p.Hkv, t);
            const int t0 = it.place * 2 * p.tile_tokens;
            d.kvh = it.kvh;
            d.row0 = it.row0 + t0;
            d.kv0 = it.kv0;
            d.Lk = it.Lk;
            d.limit0 = it.Lk - it.Lq + t0 + 1;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int toks = min(p.tile_tokens, it.Lq - t0 - s * p.tile_tokens);
                d.rows[s] = max(toks, 0) * p.G;
                d.tiles[s] = toks > 0 ? (max(d.limit0 + s * p.tile_tokens + toks - 1, 0) + C::kKeys - 1) / C::kKeys : 0;
            }
            if (parts > 1) {  // this CTA's tiles [lo, hi)
                const int nt = max(d.tiles[0], d.tiles[1]), part = blockIdx.x % parts;
                const int lo = (int)((long long)nt * part / parts), hi = (int)((long long)nt * (part + 1) / parts);
#pragma unroll
                for (int s = 0; s < 2; ++s) d.tiles[s] = max(min(d.tiles[s], hi) - lo, 0);
                d.kv0 += lo * C::kKeys;
                d.Lk -= lo * C::kKeys;
                d.limit0 -= lo * C::kKeys;
                d.parts = parts;
                if (part == 0 && lane == 0) p.split_items[t] = {d.row0, d.kvh, {d.rows[0], d.rows[1]}};
            }
        }
        if (n >= 4 && !wait_all(&bars->desc_empty[n & 3], ((n >> 2) + 1) & 1, abort)) return false;
        if (lane == 0) {
            bars->desc[n & 3] = d;
            mbar_arrive(&bars->desc_full[n & 3]);  // (release: the waiters read the descriptor behind it)
        }
        __syncwarp();
        return true;
    };
    auto load_q = [&](const ItemDesc& d) -> bool {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (d.tiles[s] == 0) continue;
            if (loads[s] > 0 && !wait_all(&bars->q_free[s], (loads[s] - 1) & 1, abort)) return false;
            if (lane == 0) {
                mbar_arrive_expect_tx(&bars->q_full[s], p.tile_tokens * p.G * 128 * C::kHalves);
#pragma unroll
                for (int h = 0; h < C::kHalves; ++h)
                    tma_load_3d(sq + s * C::kQBytes + h * C::kQHalf, &qmap, h * 64, d.kvh * p.G, d.row0 + s * p.tile_tokens, &bars->q_full[s]);
            }
            __syncwarp();
            ++loads[s];
        }
        return true;
    };
    ItemDesc d, next;
    bool ok = hand_out(0, d) && load_q(d);
    for (int n = 0; ok && d.kvh >= 0; ++n) {
        if (!hand_out(n + 1, next)) break;  // the loads run ahead into it
        // a bit of `odd` is used again 32 items on; the roles are at most the four items of the descriptor ring apart
        if (lane < 2) atomicAnd(&bars->odd[lane], ~(1u << ((n + 16) & 31)));
        const int nt = max(d.tiles[0], d.tiles[1]);
        for (int j = max(min(d.limit0, d.Lk) / C::kKeys, 0); ok && j < nt; ++j) {
            const int k = g + 2 * j + 1, st = k % C::kStages;
            ok = wait_all(&bars->cut_full[cuts & 7], (cuts >> 3) & 1, abort);
            if (!ok) break;
            clean_tile<D>(ring + st * C::kTileBytes, max(min(d.limit0 - j * C::kKeys, C::kKeys), 0), d.Lk - j * C::kKeys, bars, n);
            if (lane == 0) mbar_arrive(&bars->full[st]);
            ++cuts;
        }
        g += 2 * nt;
        ok = ok && load_q(next);
        d = next;
    }
    if (*abort)  // drain the copies in flight before the shared memory is given back
        for (int s = 0; s < 2; ++s)
            if (loads[s] > 0) {
                const unsigned long long t0 = global_ns();
                for (uint32_t i = 0; i < kSpinLimit && global_ns() - t0 < kWaitLimitNs; ++i)
                    if (mbar_try_wait(&bars->q_full[s], (loads[s] - 1) & 1)) break;
            }
}

template <int D>
__device__ __forceinline__ void prompt_load_role(const CUtensorMap& kmap, const CUtensorMap& vmap, unsigned char* ring, PBars* bars, volatile int* abort) {
    using C = PCfg<D>;
    const int lane = threadIdx.x & 31;
    int i = 0, cuts = 0;  // tiles pushed, V tiles among them that are looked through
    ItemDesc d;
    bool ok = true;
    for (int n = 0; ok && next_item(bars, n, d, abort); ++n) {
        const int nt = max(d.tiles[0], d.tiles[1]);
        for (int j = 0; j < 2 * nt; ++j, ++i) {
            const int st = i % C::kStages;
            if (!wait_all(&bars->empty[st], ((i / C::kStages) & 1) ^ 1, abort)) { ok = false; break; }
            const bool cut = (j & 1) && is_cut<D>(d, j >> 1);
            uint64_t* bar = cut ? &bars->cut_full[cuts & 7] : &bars->full[st];
            if (lane == 0) {
                mbar_arrive_expect_tx(bar, C::kTileBytes);
#pragma unroll
                for (int h = 0; h < C::kHalves; ++h)
                    tma_load_3d(ring + st * C::kTileBytes + h * C::kHalfBytes, (j & 1) ? &vmap : &kmap, h * 64, d.kvh, d.kv0 + (j >> 1) * C::kKeys, bar);
            }
            __syncwarp();
            cuts += cut;
        }
    }
    if (*abort) {  // copies still in flight: those of the ring's stages, on either kind of barrier
        const unsigned long long t0 = global_ns();
        for (int k = max(0, cuts - 8); k < cuts; ++k)
            for (uint32_t it = 0; it < kSpinLimit && global_ns() - t0 < kWaitLimitNs; ++it)
                if (mbar_try_wait(&bars->cut_full[k & 7], (k >> 3) & 1)) break;
        for (int k = max(0, i - C::kStages); k < i; ++k)  // (a stage whose tile nobody has looked through stays open: the limit ends it)
            for (uint32_t it = 0; it < kSpinLimit && global_ns() - t0 < kWaitLimitNs; ++it)
                if (mbar_try_wait(&bars->full[k % C::kStages], (k / C::kStages) & 1)) break;
    }
}

template <int D>
__device__ __forceinline__ void prompt_mma_role(int s, unsigned char* sq, unsigned char* ring, PBars* bars, uint32_t tmem, volatile int* abort) {
    using C = PCfg<D>;
    constexpr uint32_t idesc_qk = make_idesc_bf16(128, C::kKeys, false), idesc_pv = make_idesc_bf16(128, D, true);
    const int lane = threadIdx.x & 31;
    const uint32_t col_s = tmem + C::col_s(s), col_p = tmem + C::col_p(s), col_o = tmem + C::col_o(s);
    const uint64_t qd = make_smem_desc(smem_u32(sq + s * C::kQBytes), 16, 1024);
    int g = 0, u = 0, loads = 0;  // ring tiles, tiles of this stream, Q tiles of this stream before this item
    ItemDesc d;
    for (int n = 0; next_item(bars, n, d, abort); ++n) {
        const int mine = d.tiles[s], nt = max(d.tiles[0], d.tiles[1]);
        auto issue_qk = [&](int j) -> bool {
            const int k = g + 2 * j, st = k % C::kStages;
            if (!wait_all(&bars->full[st], (k / C::kStages) & 1, abort)) return false;
            // S of the tile before has been read
            if (u + j > 0 && !wait_all(&bars->s_read[s], (u + j - 1) & 1, abort)) return false;
            const uint64_t kd = make_smem_desc(smem_u32(ring + st * C::kTileBytes), 16, 1024);
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    umma_ss(col_s, qd + (uint64_t)(((kk >> 2) * C::kQHalf + (kk & 3) * 32) >> 4),
                            kd + (uint64_t)(((kk >> 2) * C::kHalfBytes + (kk & 3) * 32) >> 4), idesc_qk, kk > 0);
                umma_commit(&bars->s_full[s]);
                umma_commit(&bars->empty[st]);
                if (j == mine - 1) umma_commit(&bars->q_free[s]);
            }
            __syncwarp();
            return true;
        };
        auto issue_pv = [&](int j) -> bool {
            const int k = g + 2 * j + 1, st = k % C::kStages;
            if (!wait_all(&bars->full[st], (k / C::kStages) & 1, abort)) return false;
            unsigned char* vt = ring + st * C::kTileBytes;
            // the first product of an item overwrites O: the epilogue of the item before must have read it
            if (j == 0 && loads > 0 && !wait_all(&bars->o_free[s], (loads - 1) & 1, abort)) return false;
            const uint64_t vd = make_smem_desc(smem_u32(vt), C::kHalfBytes, 1024);
            if (!wait_all(&bars->p_full[s], (u + j) & 1, abort)) return false;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < C::kKeys / 16; ++kk)
                    umma_ts(col_o, col_p + kk * 8, vd + (uint64_t)((kk * 2048) >> 4), idesc_pv, j > 0 || kk > 0);
                umma_commit(&bars->pv_done[s]);
                umma_commit(&bars->empty[st]);
            }
            __syncwarp();
            return true;
        };
        if (mine > 0) {
            if (!wait_all(&bars->q_full[s], loads & 1, abort)) return;
            if (!issue_qk(0)) return;
            for (int j = 0; j < mine; ++j) {
                if (j + 1 < mine && !issue_qk(j + 1)) return;
                if (!issue_pv(j)) return;
            }
        }
        for (int k = g + 2 * mine; k < g + 2 * nt; ++k) {  // the other stream's alone (what has landed only: an arrival ahead would count for the tile before)
            if (!wait_all(&bars->full[k % C::kStages], (k / C::kStages) & 1, abort)) return;
            if (lane == 0) mbar_arrive(&bars->empty[k % C::kStages]);
        }
        g += 2 * nt;
        u += mine;
        loads += mine > 0;
    }
}

// One row of S: weights against the running maximum into P, sums.  Returns false if a wait gave up.
template <int D>
__device__ __forceinline__ bool prompt_softmax_tile(uint32_t s_addr, uint32_t p_addr, uint32_t o_addr, float c, int lim, bool first, uint64_t* s_read,
                                                    uint64_t* pv_done, uint32_t pv_parity, volatile int* abort, float& m, float& l) {
    constexpr int K = PCfg<D>::kKeys;
    uint32_t sv[K];
#pragma unroll
    for (int k = 0; k + 32 <= K; k += 32) tmem_ld32(s_addr + k, reinterpret_cast<uint32_t(&)[32]>(sv[k]));
    if (K % 32) tmem_ld16(s_addr + K / 32 * 32, reinterpret_cast<uint32_t(&)[16]>(sv[K / 32 * 32 % K]));
    tc_wait_ld();
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(s_read);
    if (__any_sync(0xffffffffu, lim < K)) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k >= lim) sv[k] = 0xff800000u;  // -inf by select: S may be NaN there
    }
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int k = 0; k < K; k += 8) {
        mx[0] = max3(mx[0], __uint_as_float(sv[k]), __uint_as_float(sv[k + 1]));
        mx[1] = max3(mx[1], __uint_as_float(sv[k + 2]), __uint_as_float(sv[k + 3]));
        mx[2] = max3(mx[2], __uint_as_float(sv[k + 4]), __uint_as_float(sv[k + 5]));
        mx[3] = max3(mx[3], __uint_as_float(sv[k + 6]), __uint_as_float(sv[k + 7]));
    }
    const float m_new = fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c);
    float alpha = 1.f;
    if (first || m == -INFINITY) {
        m = m_new;  // nothing accumulated yet (O is overwritten, or exactly zero)
    } else if (m_new > m + kPRescale) {
        alpha = exp2f(m - m_new);
        m = m_new;
    }
    if (__any_sync(0xffffffffu, alpha != 1.f)) {
        if (!wait_all(pv_done, pv_parity, abort)) return false;  // O is quiescent once the product of the tile before has completed
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
        l *= alpha;
    }
    const float mc = (m == -INFINITY) ? 0.f : m;
    const float2 c2 = make_float2(c, c), nm2 = make_float2(-mc, -mc);
    float2 sum0 = make_float2(0.f, 0.f), sum1 = make_float2(0.f, 0.f);
    uint32_t pk[K / 2];
#pragma unroll
    for (int k = 0; k < K; k += 4) {
        const float2 xa = __ffma2_rn(make_float2(__uint_as_float(sv[k]), __uint_as_float(sv[k + 1])), c2, nm2);
        const float2 xb = __ffma2_rn(make_float2(__uint_as_float(sv[k + 2]), __uint_as_float(sv[k + 3])), c2, nm2);
        const float2 pa = make_float2(ex2_approx(xa.x), ex2_approx(xa.y)), pb = make_float2(ex2_approx(xb.x), ex2_approx(xb.y));
        sum0 = __fadd2_rn(sum0, pa);
        sum1 = __fadd2_rn(sum1, pb);
        const __nv_bfloat162 ha = __floats2bfloat162_rn(pa.x, pa.y), hb = __floats2bfloat162_rn(pb.x, pb.y);
        pk[k >> 1] = *reinterpret_cast<const uint32_t*>(&ha);
        pk[(k >> 1) + 1] = *reinterpret_cast<const uint32_t*>(&hb);
    }
    l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
    if (!first) {  // P of the tile before has been read (an item's first: its epilogue has waited)
        if (!wait_all(pv_done, pv_parity, abort)) return false;
        tc_fence_after();
    }
    tmem_st32(p_addr, reinterpret_cast<uint32_t(&)[32]>(pk[0]));
    if (K == 128) tmem_st32(p_addr + 32, reinterpret_cast<uint32_t(&)[32]>(pk[K == 128 ? 32 : 0]));
    else tmem_st8(p_addr + 32, reinterpret_cast<uint32_t(&)[8]>(pk[K == 128 ? 0 : 32]));
    static_assert(K == 80 || K == 128, "columns of P");
    tc_wait_st();
    return true;
}

// What a row of the item sees of the values that were taken out of its tiles goes into its output, which stands in `dst` without them.
// (Their weights are positive: an infinity or a NaN of them is the sum's, whatever the rest.)
__device__ __forceinline__ float odd_sum(const PromptParams& p, const ItemDesc& d, int limit, int D, int c) {
    float x = 0.f;
    for (int j = max(d.limit0, 0); j < limit; ++j) {
        const float v = __bfloat162float(p.v[((long long)d.kv0 + j) * p.kv_stride + (long long)d.kvh * D + c]);
        if (!(fabsf(v) <= 3.4028234e38f)) x += v;
    }
    return x;
}

// A warp's rows of an item that several CTAs share: this CTA's part to scratch memory, for the merge kernel behind this one.  (m = -inf,
// l = 0: no key of the part is seen.)
template <int D>
__device__ __forceinline__ void deliver_part(const PromptParams& p, const ItemDesc& d, int s, int warp, bool live, bool odd, int limit, bool have, uint32_t o_addr,
                                             float m, float l) {
    const int r = warp * 32 + (threadIdx.x & 31), slot = 2 * blockIdx.x + s;
    float4* mine = partial_o4(p.part, D, slot, 0, r);
#pragma unroll 1
    for (int ch = 0; ch < D / 16 && have; ++ch) {
        uint32_t raw[16];
        tmem_ld16(o_addr + ch * 16, raw);
        tc_wait_ld();
#pragma unroll
        for (int k = 0; k < 16; k += 4)
            if (live)
                mine[(ch * 4 + (k >> 2)) * kMaxRows] =
                    make_float4(__uint_as_float(raw[k]), __uint_as_float(raw[k + 1]), __uint_as_float(raw[k + 2]), __uint_as_float(raw[k + 3]));
    }
    if (!live) return;
    const bool sees = have && limit > 0;
    // (scores that are all NaN or -inf leave m at -inf: the part counts all the same, and the row becomes NaN)
    p.part.m[slot * kMaxRows + r] = sees ? fmaxf(m, -3.4028234e38f) : -INFINITY;
    p.part.l[slot * kMaxRows + r] = sees ? l : 0.f;
    for (int c = 0; c < D && odd; ++c) {
        float* o = reinterpret_cast<float*>(mine + (c >> 2) * kMaxRows) + (c & 3);
        *o += odd_sum(p, d, limit, D, c);
    }
}

template <int D>
__device__ __forceinline__ void prompt_softmax_role(int s, const PromptParams& p, unsigned char* out_stage, PBars* bars, uint32_t tmem, volatile int* abort) {
    using C = PCfg<D>;
    const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, r = warp * 32 + lane, G = p.G;
    const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + C::col_s(s), p_addr = tmem + lane_base + C::col_p(s), o_addr = tmem + lane_base + C::col_o(s);
    const int tok = r / G;
    // Results leave through shared memory, 32 columns at a time: a thread has a row, but four neighbouring lanes write 64 bytes of one
    // row, eight rows an instruction (a thread's row by itself is a line of memory for every 16 bytes: 5000 clocks an item where this takes 2300).
    unsigned char* stage = out_stage + (threadIdx.x >> 5) * 2048;
    int off[4];  // where the rows that this lane writes start, from the item's first
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int R = warp * 32 + i * 8 + (lane >> 2);
        off[i] = (R / G * p.Hq + R % G) * D + (lane & 3) * 8;
    }
    int u = 0;
    ItemDesc d;
    for (int n = 0; next_item(bars, n, d, abort); ++n) {
        const int rows = d.rows[s], nt = d.tiles[s];
        if (rows == 0) continue;
        const bool live = r < rows, warp_live = warp * 32 < rows;
        const int limit = d.limit0 + s * p.tile_tokens + tok;
        // (a row that is no query's holds another sequence's: with a factor of 0 its scores never move its maximum)
        const float c = live ? p.scale_log2e : 0.f;
        float m = -INFINITY, l = 0.f;
        for (int j = 0; j < nt; ++j, ++u) {
            if (!wait_all(&bars->s_full[s], u & 1, abort)) return;
            tc_fence_after();
            if (warp_live) {
                if (!prompt_softmax_tile<D>(s_addr, p_addr, o_addr, c, live ? limit - j * C::kKeys : C::kKeys, j == 0, &bars->s_read[s], &bars->pv_done[s],
                                            (u - 1) & 1, abort, m, l))
                    return;
            } else {
                if (lane == 0) mbar_arrive(&bars->s_read[s]);
                // (every phase of pv_done is waited for, so that the epilogue's wait means the last one)
                if (j > 0 && !wait_all(&bars->pv_done[s], (u - 1) & 1, abort)) return;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->p_full[s]);
        }
        __nv_bfloat16* base = p.out + (((long long)d.row0 + s * p.tile_tokens) * p.Hq + d.kvh * G) * D;
        if (nt > 0) {
            if (!wait_all(&bars->pv_done[s], (u - 1) & 1, abort)) return;
            tc_fence_after();
        }
        const bool odd = (*static_cast<volatile unsigned*>(&bars->odd[s]) >> (n & 31) & 1u) != 0;
        const int odd_limit = min(limit, nt * C::kKeys);
        if (d.parts > 1) {  // (the CTA's only item)
            if (warp_live)
                deliver_part<D>(p, d, s, warp, live, odd, odd_limit, nt > 0, o_addr, m, l);
            continue;
        }
        const float inv = limit > 0 ? 1.f / l : 0.f;
#pragma unroll
        for (int ch = 0; ch < D / 32; ++ch) {
            uint32_t raw[32];
            if (nt > 0) {
                tmem_ld32(o_addr + ch * 32, raw);
                tc_wait_ld();
                if (ch == D / 32 - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars->o_free[s]);  // O has been read: the next item may overwrite it
                }
            }
            if (!warp_live) continue;
            __syncwarp();  // the chunk before has been read
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                __align__(16) __nv_bfloat162 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)  // (a row that sees no key: zeros)
                    v[k] = limit > 0 ? __floats2bfloat162_rn(__uint_as_float(raw[8 * q + 2 * k]) * inv, __uint_as_float(raw[8 * q + 2 * k + 1]) * inv)
                                     : __floats2bfloat162_rn(0.f, 0.f);
                *reinterpret_cast<uint4*>(stage + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = *reinterpret_cast<const uint4*>(v);
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = i * 8 + (lane >> 2);
                const uint4 v = *reinterpret_cast<const uint4*>(stage + row * 64 + (((lane & 3) ^ ((row >> 1) & 3)) << 4));
                if (warp * 32 + row < rows) *reinterpret_cast<uint4*>(base + off[i] + ch * 32) = v;
            }
        }
        if (odd) {
            __syncwarp();
            __nv_bfloat16* dst = base + ((long long)tok * p.Hq + r % G) * D;
            for (int c = 0; c < D && live; ++c) {
                const float x = odd_sum(p, d, odd_limit, D, c);
                if (x != 0.f) dst[c] = __float2bfloat16(__bfloat162float(dst[c]) + x);
            }
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kPThreads, 1) prompt_tc_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                                                                 const __grid_constant__ CUtensorMap vmap, const PromptParams p) {
    using C = PCfg<D>;
    extern __shared__ __align__(1024) unsigned char smem[];  // the swizzled tiles need 1024-byte alignment
    unsigned char* sq = smem;
    unsigned char* ring = smem + 2 * C::kQBytes;
    unsigned char* out_stage = smem + C::kOutOffset;
    PBars* bars = reinterpret_cast<PBars*>(smem + C::kBarOffset);
    volatile int* abort = &bars->abort;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if ((smem_u32(smem) & 1023u) != 0u) {  // uniform; cannot happen with the declared alignment: leave before any barrier
        if (tid == 0) atomicOr(p.status, FD_DEV_TIMEOUT);
        return;
    }
    if (warp == 8 && lane == 0) {
        for (int i = 0; i < C::kStages; ++i) { mbar_init(&bars->full[i], 1); mbar_init(&bars->empty[i], 2); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars->q_full[s], 1);
            mbar_init(&bars->q_free[s], 1);
            mbar_init(&bars->s_full[s], 1);
            mbar_init(&bars->s_read[s], 4);
            mbar_init(&bars->p_full[s], 4);
            mbar_init(&bars->pv_done[s], 1);
            mbar_init(&bars->o_free[s], 4);
        }
        for (int i = 0; i < 8; ++i) mbar_init(&bars->cut_full[i], 1);
        for (int i = 0; i < 4; ++i) { mbar_init(&bars->desc_full[i], 1); mbar_init(&bars->desc_empty[i], 11); }  // 8 softmax, 2 MMA, 1 load warps
        bars->abort = 0;
        bars->odd[0] = bars->odd[1] = 0;
        bars->fatal = 0;
        mbar_fence_init();
        prefetch_tmap(&qmap); prefetch_tmap(&kmap); prefetch_tmap(&vmap);
    }
    if (warp == 9) tmem_alloc(&bars->tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPRegSoftmax));
        prompt_softmax_role<D>(warp >> 2, p, out_stage, bars, tmem, abort);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPRegHelper));
        if (warp == 8) prompt_load_role<D>(kmap, vmap, ring, bars, abort);
        else if (warp == 11) prompt_q_role<D>(qmap, p, sq, ring, bars, abort);
        else prompt_mma_role<D>(warp - 9, sq, ring, bars, tmem, abort);
    }
    if (*abort && tid == 0) atomicOr(p.status, FD_DEV_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 512);
    if (bars->fatal) {  // inconsistent lengths: a defined output, zeros
        const long long n16 = (long long)p.total_q * p.Hq * D / 8;
        for (long long i = (long long)blockIdx.x * kPThreads + tid; i < n16; i += (long long)gridDim.x * kPThreads)
            reinterpret_cast<uint4*>(p.out)[i] = make_uint4(0, 0, 0, 0);
    }
}

// The parts of shared items combined: a block per (item, row tile) and 16 columns, a thread a row, the loads of four parts in flight.
template <int D>
__global__ void __launch_bounds__(kMaxRows) prompt_merge_kernel(const PromptParams p) {
    const PromptSplit sp = *p.split;
    const int item = blockIdx.x >> 1, s = blockIdx.x & 1, r = threadIdx.x, col = blockIdx.y * 16;
    if (sp.parts <= 1 || item >= sp.items) return;
    const PromptSplitItem it = p.split_items[item];
    if (r >= it.rows[s]) return;
    const int first = 2 * item * sp.parts + s;  // the parts' slots: every other one from here
    float top = -INFINITY, sum = 0.f, acc[16], m[kMaxParts];
#pragma unroll
    for (int q = 0; q < kMaxParts; ++q) m[q] = q < sp.parts ? p.part.m[(first + 2 * q) * kMaxRows + r] : -INFINITY;
#pragma unroll
    for (int q = 0; q < kMaxParts; ++q) top = fmaxf(top, m[q]);
#pragma unroll
    for (int k = 0; k < 16; ++k) acc[k] = 0.f;
#pragma unroll
    for (int q0 = 0; q0 < kMaxParts; q0 += 4) {
        if (q0 >= sp.parts) break;
        float4 v[4][4];
        float l[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int from = first + 2 * min(q0 + q, sp.parts - 1);
            l[q] = p.part.l[from * kMaxRows + r];
            const float4* o = partial_o4(p.part, D, from, col, r);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[q][k] = o[k * kMaxRows];
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (m[q0 + q] == -INFINITY) continue;  // (by selection: what stands there counts nothing)
            const float w = exp2f(m[q0 + q] - top);
            sum += w * l[q];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                acc[4 * k] += w * v[q][k].x;
                acc[4 * k + 1] += w * v[q][k].y;
                acc[4 * k + 2] += w * v[q][k].z;
                acc[4 * k + 3] += w * v[q][k].w;
            }
        }
    }
    const int tok = s * p.tile_tokens + r / p.G;
    store_cols_bf16<16>(p.out + (((long long)it.row0 + tok) * p.Hq + it.kvh * p.G + r % p.G) * D + col, acc, top == -INFINITY ? 0.f : 1.f / sum);
}

// Tensor maps already encoded, by what they were made from.
struct PromptMap {
    const void* ptr;
    long long stride;
    int rows, heads, box_heads, box_rows;
    CUtensorMap map;
};
struct PromptState {
    static constexpr int kSlots = 256;  // layers x (q, k, v) of a model, give or take
    PFN_cuTensorMapEncodeTiled_v12000 encode;
    PromptMap slots[kSlots];
};

}  // namespace

// The map of rows [rows][heads][d] with `stride` elements from row to row: a box of 64 elements, box_heads heads, box_rows rows.
static bool find_map(PromptState* st, const void* ptr, long long stride, int rows, int heads, int d, int box_heads, int box_rows, CUtensorMap* out) {
    const size_t h = (reinterpret_cast<uintptr_t>(ptr) >> 4) * 0x9e3779b97f4a7c15ull + (size_t)rows * 31 + (size_t)stride * 131 + box_heads;
    PromptMap& e = st->slots[(h >> 20) % PromptState::kSlots];
    if (e.ptr != ptr || e.stride != stride || e.rows != rows || e.heads != heads || e.box_heads != box_heads || e.box_rows != box_rows) {
        cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows};
        cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)stride * 2};
        cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
        cuuint32_t estr[3] = {1, 1, 1};
        e.ptr = nullptr;
        if (st->encode(&e.map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return false;
        e.ptr = ptr; e.stride = stride; e.rows = rows; e.heads = heads; e.box_heads = box_heads; e.box_rows = box_rows;
    }
    *out = e.map;
    return true;
}

cudaError_t prompt_tc_prepare(void** state, const PromptParams& p) {
    if (*state) return cudaSuccess;
    PromptState* st = new (std::nothrow) PromptState();
    if (!st) return cudaErrorMemoryAllocation;
    cudaDriverEntryPointQueryResult qres;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", reinterpret_cast<void**>(&st->encode), cudaEnableDefault, &qres);
    if (e == cudaSuccess && !st->encode) e = cudaErrorNotSupported;
    if (e == cudaSuccess)
        e = p.d == 64 ? cudaFuncSetAttribute(prompt_tc_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, PCfg<64>::kSmemBytes)
                      : cudaFuncSetAttribute(prompt_tc_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, PCfg<128>::kSmemBytes);
    // the register split draws on what the launch allocates: a request beyond that would wait for ever
    cudaFuncAttributes attr = {};
    if (e == cudaSuccess) e = p.d == 64 ? cudaFuncGetAttributes(&attr, prompt_tc_kernel<64>) : cudaFuncGetAttributes(&attr, prompt_tc_kernel<128>);
    if (e == cudaSuccess && attr.numRegs * kPThreads < 256 * kPRegSoftmax + 128 * kPRegHelper) e = cudaErrorInvalidConfiguration;
    if (e != cudaSuccess) { delete st; return e; }
    *state = st;
    return cudaSuccess;
}

bool prompt_tc_plans_itself(int batch) { return batch <= kSelfBatch; }

cudaError_t launch_prompt_tc(void* state, const PromptParams& p, int* launched, cudaStream_t s) {
    PromptState* st = static_cast<PromptState*>(state);
    CUtensorMap q, k, v;
    // (no keys at all: no item loads any, but a map has to name some memory)
    const __nv_bfloat16 *kp = p.total_kv ? p.k : p.q, *vp = p.total_kv ? p.v : p.q;
    const int kv_rows = p.total_kv ? p.total_kv : 1;
    if (!find_map(st, p.q, p.q_stride, p.total_q, p.Hq, p.d, p.G, p.tile_tokens, &q) ||
        !find_map(st, kp, p.kv_stride, kv_rows, p.Hkv, p.d, 1, p.d == 128 ? PCfg<128>::kKeys : PCfg<64>::kKeys, &k) ||
        !find_map(st, vp, p.kv_stride, kv_rows, p.Hkv, p.d, 1, p.d == 128 ? PCfg<128>::kKeys : PCfg<64>::kKeys, &v))
        return cudaErrorInvalidValue;
    // The lengths are on the device.  From the totals: there are at least total_q / (2 tile_tokens) blocks; where that leaves sharing
    // possible, the merge follows, and finds out.
    PromptParams a = p;
    const long long blocks = (p.total_q + 2LL * p.tile_tokens - 1) / (2 * p.tile_tokens);
    const bool may_split = 2 * blocks * p.Hkv <= p.n_ctas && p.total_kv >= kMinSplitTiles * PCfg<128>::kKeys;
    if (!may_split) a.split = nullptr;
    cudaError_t e = p.d == 64 ? launch(prompt_tc_kernel<64>, p.n_ctas, kPThreads, PCfg<64>::kSmemBytes, s, q, k, v, a)
                              : launch(prompt_tc_kernel<128>, p.n_ctas, kPThreads, PCfg<128>::kSmemBytes, s, q, k, v, a);
    *launched = e == cudaSuccess;
    if (may_split && e == cudaSuccess) {
        const dim3 grid(p.n_ctas / 2 * 2, p.d / 16);
        e = launch(p.d == 64 ? prompt_merge_kernel<64> : prompt_merge_kernel<128>, grid, kMaxRows, 0, s, a);
        *launched += e == cudaSuccess;
    }
    return e;
}

void prompt_tc_free(void* state) { delete static_cast<PromptState*>(state); }

}  // namespace fd
