// Causal attention of packed sequences on the tensor cores: the prompt on its way in.
//
// A CTA works on two row tiles at a time (fd_prompt.cuh), each a stream of its own: 128 query rows, a softmax warpgroup, an S / P
// buffer and an O accumulator in tensor memory, an MMA-issuing warp.  Both streams read the same K and V tiles (128 keys, brought
// in by TMA through one ring), so a tile's bytes serve 256 rows, and while one stream is in its softmax the tensor pipe works on
// the other.  Per tile and stream:
//     S = Q K^T      tcgen05.mma, Q and K from shared memory, S in tensor memory
//     P = exp2(..)   a thread a row: the row of S in registers, causal mask in the tiles the row's last key cuts, running maximum and
//                    sum in fp32; P goes back over S in bf16 (V is bf16, and the operands of an MMA are of one type)
//     O += P V       A = P from tensor memory, B = V MN-major; O is rescaled only when a row's maximum has grown by more than 2^8
// Roles: warps 0-3 and 4-7 softmax of streams 0 and 1, 8 K and V loads, 9 and 10 MMAs of streams 0 and 1, 11 Q loads and the
// descriptors of the items, which every role copies from a ring in shared memory.
// Tensor memory: S0 / P0 [0,128)  S1 / P1 [128,256)  O0 [256,256+d)  O1 [384,384+d).
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

constexpr int kPThreads = 384;
constexpr float kPRescale = 8.0f;  // log2 units

template <int D>
struct PCfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kTileTokens * D * 2;    // one K, V or Q tile
    static constexpr int kHalfBytes = kTileTokens * 128;      // 64 elements of d of its rows
    static constexpr int kStages = D == 128 ? 5 : 10;         // tiles in the ring: K and V in turn
    static constexpr int kBarOffset = (2 + kStages) * kTileBytes;
    static constexpr int kSmemBytes = kBarOffset + 1024;
    static_assert(kSmemBytes <= 227 * 1024, "shared memory of one CTA");
};

// What the roles know of an item.
struct ItemDesc {
    int kvh, row0, kv0, Lk;  // row0: the first output row of tile 0; kv-head -1: no more items
    int limit0;              // keys that token 0 of tile 0 sees
    int rows[2];             // query rows of the two tiles
    int tiles[2];            // key tiles they see
    int pad;
};

struct PBars {
    uint64_t full[10], empty[10];
    uint64_t q_full[2], q_free[2], s_full[2], p_full[2], pv_done[2], o_free[2];
    uint64_t desc_full[4], desc_empty[4];
    ItemDesc desc[4];
    uint32_t tmem_base;
    int abort;
};
static_assert(sizeof(PBars) <= 1024, "barriers and descriptors");

// A role's next item, copied from the ring.  Whole warps.
__device__ __forceinline__ bool next_item(PBars* bars, int n, ItemDesc& d, volatile int* abort) {
    if (!wait_all(&bars->desc_full[n & 3], (n >> 2) & 1, abort)) return false;
    d = bars->desc[n & 3];
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&bars->desc_empty[n & 3]);
    return d.kvh >= 0;
}

template <int D>
__device__ __forceinline__ void prompt_q_role(const CUtensorMap& qmap, const PromptParams& p, unsigned char* sq, PBars* bars, volatile int* abort) {
    using C = PCfg<D>;
    const int lane = threadIdx.x & 31;
    const long long total = *p.plan.fatal ? 0 : (long long)p.plan.pre[p.batch] * p.Hkv;
    int loads[2] = {0, 0};
    for (int turn = 0, n = 0;; ++turn) {
        const long long t = prompt_turn(turn, blockIdx.x, gridDim.x);
        const bool done = (long long)turn * gridDim.x >= total;
        if (!done && t >= total) continue;
        ItemDesc d = {-1, 0, 0, 0, 0, {0, 0}, {0, 0}, 0};
        if (!done) {
            const PromptItem it = prompt_item(p.plan, p.batch, p.Hkv, t);
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
                d.tiles[s] = toks > 0 ? (max(d.limit0 + s * p.tile_tokens + toks - 1, 0) + kTileTokens - 1) / kTileTokens : 0;
            }
        }
        if (n >= 4 && !wait_all(&bars->desc_empty[n & 3], ((n >> 2) + 1) & 1, abort)) break;
        if (lane == 0) {
            bars->desc[n & 3] = d;
            mbar_arrive(&bars->desc_full[n & 3]);  // (release: the waiters read the descriptor behind it)
        }
        __syncwarp();
        ++n;
        if (done) break;
        bool ok = true;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (d.tiles[s] == 0 || !ok) continue;
            if (loads[s] > 0 && !wait_all(&bars->q_free[s], (loads[s] - 1) & 1, abort)) { ok = false; continue; }
            if (lane == 0) {
                mbar_arrive_expect_tx(&bars->q_full[s], p.tile_tokens * p.G * 128 * C::kHalves);
#pragma unroll
                for (int h = 0; h < C::kHalves; ++h)
                    tma_load_3d(sq + s * C::kTileBytes + h * C::kHalfBytes, &qmap, h * 64, d.kvh * p.G, d.row0 + s * p.tile_tokens, &bars->q_full[s]);
            }
            __syncwarp();
            ++loads[s];
        }
        if (!ok) break;
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
    int i = 0;  // tiles pushed
    ItemDesc d;
    bool ok = true;
    for (int n = 0; ok && next_item(bars, n, d, abort); ++n) {
        const int nt = max(d.tiles[0], d.tiles[1]);
        for (int j = 0; j < 2 * nt; ++j, ++i) {
            const int st = i % C::kStages;
            if (!wait_all(&bars->empty[st], ((i / C::kStages) & 1) ^ 1, abort)) { ok = false; break; }
            if (lane == 0) {
                mbar_arrive_expect_tx(&bars->full[st], C::kTileBytes);
#pragma unroll
                for (int h = 0; h < C::kHalves; ++h)
                    tma_load_3d(ring + st * C::kTileBytes + h * C::kHalfBytes, (j & 1) ? &vmap : &kmap, h * 64, d.kvh, d.kv0 + (j >> 1) * kTileTokens,
                                &bars->full[st]);
            }
            __syncwarp();
        }
    }
    if (*abort)
        for (int k = max(0, i - C::kStages); k < i; ++k) {
            const unsigned long long t0 = global_ns();
            for (uint32_t it = 0; it < kSpinLimit && global_ns() - t0 < kWaitLimitNs; ++it)
                if (mbar_try_wait(&bars->full[k % C::kStages], (k / C::kStages) & 1)) break;
        }
}

template <int D>
__device__ __forceinline__ void prompt_mma_role(int s, unsigned char* sq, unsigned char* ring, PBars* bars, uint32_t tmem, volatile int* abort) {
    using C = PCfg<D>;
    constexpr uint32_t idesc_qk = make_idesc_bf16(128, kTileTokens, false), idesc_pv = make_idesc_bf16(128, D, true);
    const int lane = threadIdx.x & 31;
    const uint32_t col_s = tmem + s * 128u, col_o = tmem + 256u + s * 128u;
    const uint64_t qd = make_smem_desc(smem_u32(sq + s * C::kTileBytes), 16, 1024);
    int g = 0, u = 0, loads = 0;  // ring tiles, tiles of this stream, Q tiles of this stream before this item
    ItemDesc d;
    for (int n = 0; next_item(bars, n, d, abort); ++n) {
        const int mine = d.tiles[s], nt = max(d.tiles[0], d.tiles[1]);
        if (mine > 0 && !wait_all(&bars->q_full[s], loads & 1, abort)) return;
        for (int j = 0; j < nt; ++j, g += 2) {
            const int ks = g % C::kStages, vs = (g + 1) % C::kStages;
            if (!wait_all(&bars->full[ks], (g / C::kStages) & 1, abort)) return;
            if (j >= mine) {  // the other stream's alone (what has landed only: an arrival ahead would count for the tile before)
                if (lane == 0) mbar_arrive(&bars->empty[ks]);
                if (!wait_all(&bars->full[vs], ((g + 1) / C::kStages) & 1, abort)) return;
                if (lane == 0) mbar_arrive(&bars->empty[vs]);
                continue;
            }
            // S is written over the P of the tile before: its product has to have completed
            const uint64_t kd = make_smem_desc(smem_u32(ring + ks * C::kTileBytes), 16, 1024);
            if (u > 0 && !wait_all(&bars->pv_done[s], (u - 1) & 1, abort)) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint64_t off = (uint64_t)(((kk >> 2) * C::kHalfBytes + (kk & 3) * 32) >> 4);
                    umma_ss(col_s, qd + off, kd + off, idesc_qk, kk > 0);
                }
                umma_commit(&bars->s_full[s]);
                umma_commit(&bars->empty[ks]);
                if (j == mine - 1) umma_commit(&bars->q_free[s]);
            }
            __syncwarp();
            if (!wait_all(&bars->full[vs], ((g + 1) / C::kStages) & 1, abort)) return;
            unsigned char* vt = ring + vs * C::kTileBytes;
            const int valid = d.Lk - j * kTileTokens;
            if (valid < kTileTokens) {  // rows behind the sequence's last key are another's: P is 0 there, but 0 * NaN is not
                for (int e = lane; e < (kTileTokens - valid) * 8 * C::kHalves; e += 32) {
                    const int r = valid + e / (8 * C::kHalves), w = e % (8 * C::kHalves);
                    *reinterpret_cast<uint4*>(vt + (w >> 3) * C::kHalfBytes + r * 128 + (w & 7) * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_proxy_async_smem();
                __syncwarp();
            }
            // the first product of an item overwrites O: the epilogue of the item before must have read it
            if (j == 0 && loads > 0 && !wait_all(&bars->o_free[s], (loads - 1) & 1, abort)) return;
            const uint64_t vd = make_smem_desc(smem_u32(vt), C::kHalfBytes, 1024);
            if (!wait_all(&bars->p_full[s], u & 1, abort)) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < kTileTokens / 16; ++kk)
                    umma_ts(col_o, col_s + kk * 8, vd + (uint64_t)((kk * 2048) >> 4), idesc_pv, j > 0 || kk > 0);
                umma_commit(&bars->pv_done[s]);
                umma_commit(&bars->empty[vs]);
            }
            __syncwarp();
            ++u;
        }
        loads += mine > 0;
    }
}

// One row of S: weights against the running maximum, P over S, sums.
template <int D>
__device__ __forceinline__ void prompt_softmax_tile(uint32_t s_addr, uint32_t o_addr, float c, int lim, bool first, float& m, float& l) {
    uint32_t sv[4][32];
#pragma unroll
    for (int ch = 0; ch < 4; ++ch) tmem_ld32(s_addr + ch * 32, sv[ch]);
    tc_wait_ld();
    if (__any_sync(0xffffffffu, lim < kTileTokens)) {
#pragma unroll
        for (int ch = 0; ch < 4; ++ch)
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (ch * 32 + k >= lim) sv[ch][k] = 0xff800000u;  // -inf by select: S may be NaN there
    }
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
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
    if (first || m == -INFINITY) {
        m = m_new;  // nothing accumulated yet (O is overwritten, or exactly zero)
    } else if (m_new > m + kPRescale) {
        alpha = exp2f(m - m_new);
        m = m_new;
    }
    if (__any_sync(0xffffffffu, alpha != 1.f)) {
        // the product of the tile before has completed (S was written behind it), so O is quiescent
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
#pragma unroll
    for (int hp = 0; hp < 2; ++hp) {
        uint32_t pk[32];
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
            const float2 xa = __ffma2_rn(make_float2(__uint_as_float(sv[2 * hp][k]), __uint_as_float(sv[2 * hp][k + 1])), c2, nm2);
            const float2 xb = __ffma2_rn(make_float2(__uint_as_float(sv[2 * hp + 1][k]), __uint_as_float(sv[2 * hp + 1][k + 1])), c2, nm2);
            const float2 pa = make_float2(ex2_approx(xa.x), ex2_approx(xa.y)), pb = make_float2(ex2_approx(xb.x), ex2_approx(xb.y));
            sum0 = __fadd2_rn(sum0, pa);
            sum1 = __fadd2_rn(sum1, pb);
            const __nv_bfloat162 ha = __floats2bfloat162_rn(pa.x, pa.y), hb = __floats2bfloat162_rn(pb.x, pb.y);
            pk[k >> 1] = *reinterpret_cast<const uint32_t*>(&ha);
            pk[16 + (k >> 1)] = *reinterpret_cast<const uint32_t*>(&hb);
        }
        tmem_st32(s_addr + hp * 32, pk);  // over columns of S that are in registers
    }
    l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
    tc_wait_st();
}

template <int D>
__device__ __forceinline__ void prompt_softmax_role(int s, const PromptParams& p, PBars* bars, uint32_t tmem, volatile int* abort) {
    const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31, r = warp * 32 + lane, G = p.G;
    const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + s * 128u, o_addr = tmem + lane_base + 256u + s * 128u;
    const int tok = r / G;
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
            if (warp_live) prompt_softmax_tile<D>(s_addr, o_addr, c, live ? limit - j * kTileTokens : kTileTokens, j == 0, m, l);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->p_full[s]);
        }
        __nv_bfloat16* dst = p.out + (((long long)d.row0 + s * p.tile_tokens + tok) * p.Hq + d.kvh * G + r % G) * D;
        if (nt > 0) {
            if (!wait_all(&bars->pv_done[s], (u - 1) & 1, abort)) return;
            tc_fence_after();
        }
        const float inv = limit > 0 ? 1.f / l : 0.f;
#pragma unroll
        for (int ch = 0; ch < D / 32; ++ch) {
            float o[32];
            if (nt > 0) {
                uint32_t raw[32];
                tmem_ld32(o_addr + ch * 32, raw);
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = limit > 0 ? __uint_as_float(raw[k]) : 0.f;  // (a row that sees no key: zeros)
                if (ch == D / 32 - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars->o_free[s]);  // O has been read: the next item may overwrite it
                }
            } else {
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = 0.f;
            }
            if (live) store_cols_bf16<32>(dst + ch * 32, o, inv);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kPThreads, 1) prompt_tc_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                                                                 const __grid_constant__ CUtensorMap vmap, const PromptParams p) {
    using C = PCfg<D>;
    extern __shared__ __align__(1024) unsigned char smem[];  // the swizzled tiles need 1024-byte alignment
    unsigned char* sq = smem;
    unsigned char* ring = smem + 2 * C::kTileBytes;
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
            mbar_init(&bars->p_full[s], 4);
            mbar_init(&bars->pv_done[s], 1);
            mbar_init(&bars->o_free[s], 4);
        }
        for (int i = 0; i < 4; ++i) { mbar_init(&bars->desc_full[i], 1); mbar_init(&bars->desc_empty[i], 11); }  // 8 softmax, 2 MMA, 1 load warps
        bars->abort = 0;
        mbar_fence_init();
        prefetch_tmap(&qmap); prefetch_tmap(&kmap); prefetch_tmap(&vmap);
    }
    if (warp == 9) tmem_alloc(&bars->tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;
    if (*p.plan.fatal) {  // inconsistent lengths: a defined output, zeros (no role has started: the Q warp would find no item)
        const long long n16 = (long long)p.total_q * p.Hq * D / 8;
        for (long long i = (long long)blockIdx.x * kPThreads + tid; i < n16; i += (long long)gridDim.x * kPThreads)
            reinterpret_cast<uint4*>(p.out)[i] = make_uint4(0, 0, 0, 0);
    } else if (warp < 8) {
        // 8 x 32 x 224 + 4 x 32 x 56 = 384 x 168, what the launch allocated
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(224));
        prompt_softmax_role<D>(warp >> 2, p, bars, tmem, abort);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(56));
        if (warp == 8) prompt_load_role<D>(kmap, vmap, ring, bars, abort);
        else if (warp == 11) prompt_q_role<D>(qmap, p, sq, bars, abort);
        else prompt_mma_role<D>(warp - 9, sq, ring, bars, tmem, abort);
    }
    if (*abort && tid == 0) atomicOr(p.status, FD_DEV_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 512);
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
    const CUtensorMap *q, *k, *v;
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
    if (e != cudaSuccess) { delete st; return e; }
    *state = st;
    return cudaSuccess;
}

cudaError_t launch_prompt_tc(void* state, const PromptParams& p, cudaStream_t s) {
    PromptState* st = static_cast<PromptState*>(state);
    CUtensorMap q, k, v;
    // (no keys at all: no item loads any, but a map has to name some memory)
    const __nv_bfloat16 *kp = p.total_kv ? p.k : p.q, *vp = p.total_kv ? p.v : p.q;
    const int kv_rows = p.total_kv ? p.total_kv : 1;
    if (!find_map(st, p.q, p.q_stride, p.total_q, p.Hq, p.d, p.G, p.tile_tokens, &q) ||
        !find_map(st, kp, p.kv_stride, kv_rows, p.Hkv, p.d, 1, kTileTokens, &k) ||
        !find_map(st, vp, p.kv_stride, kv_rows, p.Hkv, p.d, 1, kTileTokens, &v))
        return cudaErrorInvalidValue;
    if (p.d == 64) prompt_tc_kernel<64><<<p.n_ctas, kPThreads, PCfg<64>::kSmemBytes, s>>>(q, k, v, p);
    else prompt_tc_kernel<128><<<p.n_ctas, kPThreads, PCfg<128>::kSmemBytes, s>>>(q, k, v, p);
    return cudaSuccess;
}

void prompt_tc_free(void* state) { delete static_cast<PromptState*>(state); }

}  // namespace fd
