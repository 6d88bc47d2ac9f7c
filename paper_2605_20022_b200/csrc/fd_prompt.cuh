// What the prompt attention kernels share: the call's parameters, its work list, the order in which the work is taken.
//
// A row tile is 128 / G consecutive tokens of a sequence times the G q-heads of one kv-head, at most 128 rows (row r = token r / G,
// head r % G): all of them read the same keys, whatever the ratio of heads.  A work item is a block of two neighbouring row tiles of
// one kv-head.  Under the causal mask the cost of a block of a whole prompt grows with its place in the sequence, so items are numbered from
// the last place down: first all blocks at the highest place that any sequence has, then the place below, ...  With the sequences sorted by
// their number of blocks, longest first, the blocks at places >= j number  S(r) - j r,  r the sequences that have more than j
// blocks and S the prefix sums of their numbers: a binary search finds an item from B numbers, no list of items is kept.
// CTA c of N takes items c, 2N - 1 - c, 2N + c, 4N - 1 - c, ...: the costs of a round of whole prompts fall steadily, and going back and
// forth evens them out.  Earlier keys (kv_lens) add to a block's cost and do not enter the order: where they differ much from sequence to
// sequence the CTAs finish apart (16 chunks of 64 tokens at 8 kv-heads, one behind 30000 keys, the others behind 300: 427 us, the time of the one
// sequence's 8 items, where an even share would be 25).
#pragma once

#include "fd_internal.cuh"

namespace fd {

struct PromptPlan {
    int* cu_q;    // [B + 1] first query row of each sequence
    int* cu_kv;   // [B + 1] first key row
    int* perm;    // [B] sequences by falling number of blocks
    int* blocks;  // [B] their numbers, in that order
    int* pre;     // [B + 1] exclusive prefix sums of them
    int* fatal;   // lengths inconsistent: the output is zeros
};

struct PromptItem {
    int b, kvh, place;  // sequence, kv-head, block of the sequence
    int Lq, Lk;         // its query rows and keys
    int row0, kv0;      // their first rows
};

// Blocks at places >= j, over the B sequences of the plan.
__device__ __forceinline__ int blocks_from(const PromptPlan& pl, int B, int j, int* count) {
    int lo = 0, hi = B;  // sequences with more than j blocks: a prefix of the order
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (pl.blocks[mid] > j) lo = mid + 1; else hi = mid;
    }
    *count = lo;
    return pl.pre[lo] - j * lo;
}

__device__ __forceinline__ PromptItem prompt_item(const PromptPlan& pl, int B, int Hkv, long long t) {
    PromptItem it;
    const int blk = (int)(t / Hkv);
    it.kvh = (int)(t - (long long)blk * Hkv);
    // the highest place j with more than blk blocks at places >= j
    int lo = 0, hi = pl.blocks[0], n;  // (blocks_from(lo) > blk, blocks_from(hi) <= blk)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (blocks_from(pl, B, mid, &n) > blk) lo = mid; else hi = mid;
    }
    const int above = blocks_from(pl, B, lo + 1, &n);
    it.place = lo;
    it.b = pl.perm[blk - above];
    it.row0 = pl.cu_q[it.b];
    it.Lq = pl.cu_q[it.b + 1] - it.row0;
    it.kv0 = pl.cu_kv[it.b];
    it.Lk = pl.cu_kv[it.b + 1] - it.kv0;
    return it;
}

// The i-th item of CTA c of n, or at or beyond the total when it has no more.
__device__ __forceinline__ long long prompt_turn(int i, int c, int n) { return (long long)i * n + ((i & 1) ? n - 1 - c : c); }

// What the merge of shared items needs to know.
struct PromptSplit {
    int parts, items;
};
struct PromptSplitItem {
    int row0, kvh, rows[2];
};

struct PromptParams {
    int batch, total_q, total_kv;
    int Hq, Hkv, G, d, tile_tokens;  // tokens of a row tile: kMaxRows / G
    float scale_log2e;
    const __nv_bfloat16 *q, *k, *v;
    long long q_stride, kv_stride;   // elements from one row to the next
    const int32_t* q_lens;
    const int32_t* kv_lens;          // nullptr: the same as q_lens
    __nv_bfloat16* out;
    PromptPlan plan;
    PartialView part;                // [2 n_ctas] slots: what a CTA computes of an item that several share
    PromptSplit* split;              // how the items were shared, or nullptr: none can be
    PromptSplitItem* split_items;    // [n_ctas / 2]
    int n_ctas;
    int* status;
};

cudaError_t launch_prompt_plan(const PromptParams& p, cudaStream_t s);
cudaError_t prompt_simt_prepare(int d);
void launch_prompt_simt(const PromptParams& p, cudaStream_t s);
cudaError_t prompt_tc_prepare(void** state, const PromptParams& p);
bool prompt_tc_plans_itself(int batch);  // (then the plan kernel is not needed)
cudaError_t launch_prompt_tc(void* state, const PromptParams& p, int* launched, cudaStream_t s);  // *launched: kernels
void prompt_tc_free(void* state);

}  // namespace fd
