/*
 * flexdraft.h -- C ABI of the FlexDraft decode-step hot path for NVIDIA B200 (sm_100a).
 *
 * One decode step of FlexDraft's parallel draft-and-verify decoding (paper Sec. 4.1,
 * "Inference"; Sec. 3 for the verification rule) is, per attention layer and per
 * sequence b, the attention of a query block
 *
 *        [ bonus token | k_b draft tokens | M_b mask tokens ]
 *          \____ C_b = k_b + 1 candidate rows ____/
 *
 * against that sequence's paged KV cache under the hybrid mask, followed, once per
 * step, by lossless verification of the drafts and by the commit / rollback of the KV
 * positions written for this block.  This library exports those three operations
 * (fd_attn_draft_verify, fd_verify_accept, fd_kv_commit) and the steps next to them: the
 * all-hypotheses form of the attention and the branch selection (Eq. 2), the draft-side
 * tail (Eq. 4, Eq. 5), verification by sampling at temperature > 0 (Sec. 3), the KV
 * append, and a whole step from host buffers.  Around them stand what a serving loop needs
 * next: pages out of a free list (fd_kv_reserve), norm, rotation and append in one pass
 * (fd_qk_norm_rope_append), and a cache held in 4 bits with the attention that reads it
 * (fd_kv_append_fp4, fd_kv_read_fp4, fd_attn_draft_verify_fp4).  Further out: the attention of
 * the prompts a sequence begins with (fd_attn_prompt), a cache held in 8 bits (fd_kv_append_fp8,
 * fd_kv_read_fp8, fd_attn_draft_verify_fp8), and the pages of sequences that branch and end
 * (fd_kv_fork, fd_kv_free, fd_kv_compact, fd_kv_copy_pages).  Everything runs in
 * hand-written CUDA kernels; there is no CPU fallback.
 *
 * Conventions (all entry points)
 *   - "device pointer": memory on the GPU that is current when fd_create() ran, owned
 *     by the caller.  "host pointer": ordinary host memory, owned by the caller.  That GPU
 *     must be the current one in every call on the context, and the stream one of its streams.
 *   - Calls are asynchronous on the given CUDA stream (a cudaStream_t passed as void*,
 *     NULL = the legacy default stream) and ordered by it.  Calls that share one fd_ctx
 *     must be issued on one stream, or be ordered by the caller: they share the context's
 *     scratch memory.
 *     A context is not thread-safe: one host thread at a time per fd_ctx.
 *   - The hot calls (fd_attn_draft_verify, fd_verify_accept, fd_kv_commit) never allocate
 *     and never synchronise; all scratch memory is sized by fd_create() from fd_config.
 *   - Errors the host can see (NULL pointer, size beyond the configured maximum,
 *     unsupported shape, misaligned pointer) return a code and launch nothing.
 *   - Errors only the device can see (lengths that contradict each other, a page id
 *     outside the pool, ...) never trap: the kernels skip the work, write a defined
 *     value (documented per call) and OR a FD_DEV_* bit into a sticky status word that
 *     fd_last_device_status() reads.
 *
 * Notation: B sequences; Hq q-heads, Hkv kv-heads, G = Hq/Hkv; d = head_dim; P = page_size
 * (16 tokens); V = vocab.  n_b = prefix_lens[b]; Lq_b = q_lens[b]; M_b = n_mask[b];
 * C_b = Lq_b - M_b; kv_len_b = n_b + Lq_b; T = sum_b Lq_b; R = sum_b C_b.
 */
#ifndef FLEXDRAFT_H
#define FLEXDRAFT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct fd_ctx fd_ctx; /* opaque; owns scratch memory and the device status word */

typedef enum {
    FD_OK = 0,
    FD_ERR_INVALID_ARG = 1,   /* NULL pointer, negative size, size beyond fd_config maximum */
    FD_ERR_UNSUPPORTED = 2,   /* shape outside what the kernels implement */
    FD_ERR_WORKSPACE = 3,     /* scratch memory could not be allocated */
    FD_ERR_CUDA = 4,          /* a CUDA runtime / driver call failed */
    FD_ERR_DEVICE_STATUS = 5, /* reserved */
    FD_ERR_STATIC_LIMIT = 6   /* fd_verify_accept_static: more rows or sequences than its fixed scratch holds */
} fd_status;

/* Bits of the sticky device status word. */
enum {
    FD_DEV_BAD_LENGTHS = 1,   /* lengths negative, n_mask > q_len, q_len > max_q_len, kv_len beyond the
                                 page table, or row totals that do not match the call's row count */
    FD_DEV_BAD_PAGE = 2,      /* a page id needed by a sequence is outside [0, num_pages) */
    FD_DEV_TIMEOUT = 4,       /* a bounded device-side wait ran out; the kernel returned early */
    FD_DEV_BAD_ACCEPT = 8,    /* fd_kv_commit: accepted_len[b] >= q_lens[b] */
    FD_DEV_NO_PAGES = 16      /* fd_kv_reserve, fd_kv_fork: the free list holds fewer pages than the call needs */
};

/* How a paged KV cache holds its values (fd_qk_norm_rope_append, fd_kv_copy_pages). */
enum {
    FD_KV_BF16 = 0,           /* [num_pages, 2, Hkv, P, d] bf16, the cache of fd_attn_draft_verify */
    FD_KV_FP4 = 1,            /* 4-bit pages, the cache of fd_attn_draft_verify_fp4 (see there) */
    FD_KV_FP8 = 2,            /* 8-bit pages, the cache of fd_attn_draft_verify_fp8 (see there; fd_kv_copy_pages only) */
    FD_KV_ROWS = 3            /* no cache: [2, num_pages * P, Hkv, d] bf16, K rows then V rows, row = slot; what fd_attn_prompt and
                                 fd_kv_append_fp8 take (fd_qk_norm_rope_append only) */
};

/* Which two elements of a head fd_qk_norm_rope_append rotates together (R = rot_dim). */
enum {
    FD_ROPE_HALVES = 0,       /* (i, i + R / 2) for i < R / 2 */
    FD_ROPE_ADJACENT = 1      /* (2 i, 2 i + 1) */
};

/* Which attention kernel fd_attn_draft_verify launches. */
enum {
    FD_ATTN_AUTO = 0,         /* tensor-core kernel when the shape allows it, else the SIMT kernel */
    FD_ATTN_SIMT = 1,         /* CUDA-core split-KV kernel (any supported shape) */
    FD_ATTN_TCGEN05 = 2,      /* tcgen05 / TMEM / TMA split-KV kernel (head_dim 64 or 128); how it finds its work is
                                 chosen per call, see FD_TC_* */
    FD_ATTN_TCGEN05_PLANNED = 3,      /* the same kernel, always on the plan kernel's work list (FD_TC_PLANNED) */
    FD_ATTN_TCGEN05_SELF_PLANNED = 4  /* the same kernel, planning for itself wherever the call is small enough
                                         (FD_TC_SELF_PLANNED), never one cluster per segment */
};

/* How a call of the tensor-core attention kernel found its work (fd_attn_last_mode).  All three give the same
 * result to within rounding order; the choice is about fixed cost.
 *   FD_TC_PLANNED       a one-CTA plan kernel (or fd_plan_pin, once per step) cuts all KV tiles of the call into
 *                       one range per SM ("stream-K"); ranges that share a (sequence, kv-head) segment leave
 *                       partial results in scratch memory and the last to arrive merges them.
 *   FD_TC_SELF_PLANNED  at most 24 sequences with query blocks of at most 128 / G rows: every CTA makes the same
 *                       cut itself in its prologue; one launch, nothing to wait for.
 *   FD_TC_CLUSTER       at most 18 segments (batch 1-2 at 8 kv-heads, the paper's parallel-mode operating point):
 *                       one thread-block cluster of up to 16 CTAs per segment splits its tiles evenly and merges
 *                       through distributed shared memory; one launch, no scratch memory, no counters. */
enum { FD_TC_PLANNED = 0, FD_TC_SELF_PLANNED = 1, FD_TC_CLUSTER = 2 };

typedef struct {
    int n_q_heads;            /* Hq */
    int n_kv_heads;           /* Hkv, divides Hq */
    int head_dim;             /* d: 64 or 128 */
    int page_size;            /* P: 16 */
    int vocab;                /* V >= 1 */
    int max_batch;            /* largest B of any call; at most 4096 */
    int max_q_len;            /* largest Lq_b, <= 4096.  Up to 128 / G block rows share one 128-row MMA tile; a
                                 longer query block is processed as several such row blocks, each streaming
                                 the sequence's KV on its own (the O(N^2) regime of preparing every hypothesis) */
    int max_pages_per_seq;    /* row length of page_table */
    float softmax_scale;      /* 0 selects 1/sqrt(d) */
    int attn_path;            /* FD_ATTN_* */
} fd_config;

/* Create a context on the current CUDA device.  Allocates all scratch memory: about 20 MB for
 * the attention (split partials, work list) plus, for the vocabulary sweeps, about 30 bytes per
 * (row, 4096-logit chunk) with max_batch * max_q_len rows -- 2 MB at batch 64, 32 rows and a
 * 152k vocabulary; size max_batch and max_q_len for the job.  *ctx is NULL on failure
 * (FD_ERR_WORKSPACE if the device has no room). */
fd_status fd_create(fd_ctx** ctx, const fd_config* cfg);

/* Free a context.  Synchronises the device first.  NULL is accepted. */
fd_status fd_destroy(fd_ctx* ctx);

/*
 * Attention of one target forward pass over the ragged query blocks (Sec. 4.1,
 * "Inference"; hybrid mask of Sec. 4.1 and the Fig. 2 caption).  For sequence b, q-head
 * h, block row i:
 *
 *     out[row0_b + i, h, :] = sum_{j in A_b(i)} softmax_j( scale * <q[row0_b+i, h], K_b[j, h/G]> ) V_b[j, h/G]
 *
 *     A_b(i), i <  C_b (candidate row): { j < n_b } U { n_b + t : t <= i }        causal; no mask token
 *     A_b(i), i >= C_b (mask row):      { j < kv_len_b }                          prefix, all candidates,
 *                                                                                 whole mask block
 *     K_b[j], V_b[j] = kv_cache[ page_table[b][j / P], 0 | 1, h / G, j % P, : ]
 *
 * The caller has already written K/V of all Lq_b query tokens (candidates first, then
 * mask tokens) at logical positions n_b .. n_b + Lq_b - 1 ("append, then attend"), with
 * positional encoding and norms applied.  Slots that no valid token owns may hold any
 * bit pattern (NaN included); they never influence the result.
 *
 *   batch          B, 0 <= B <= max_batch (B = 0 is a no-op)
 *   total_q_rows   T; must equal sum_b q_lens[b]
 *   q              device, [T, Hq, d] bf16, 16-byte aligned, sequence-major rows
 *   kv_cache       device, [num_pages, 2, Hkv, P, d] bf16, 128-byte aligned
 *   num_pages      size of the page pool
 *   page_table     device, [B, max_pages_per_seq] int32; entries beyond ceil(kv_len_b/P) are ignored
 *   prefix_lens, q_lens, n_mask   device, [B] int32
 *   out            device, [T, Hq, d] bf16, 16-byte aligned; fully overwritten
 *   stream         cudaStream_t
 *
 * Device-detected errors: a sequence with a page id outside the pool gets zeros in its
 * out rows (FD_DEV_BAD_PAGE); inconsistent lengths zero all T rows (FD_DEV_BAD_LENGTHS).
 * Arithmetic: bf16 inputs, fp32 scores / softmax / accumulation, bf16 output.
 */
fd_status fd_attn_draft_verify(fd_ctx* ctx, int batch, int total_q_rows,
                               const void* q, const void* kv_cache, int num_pages,
                               const int32_t* page_table, const int32_t* prefix_lens,
                               const int32_t* q_lens, const int32_t* n_mask,
                               void* out, void* stream);

/*
 * Optional: pin the work list of a step.  The attention call derives a work list (which CTA streams which
 * KV tiles) from the lengths alone; it is the same for every layer of a step.  fd_plan_pin computes it once;
 * until fd_plan_unpin, every fd_attn_draft_verify[_blocks] call with the same batch, total_q_rows and the
 * same four length pointers reuses it instead of recomputing it (a call with anything else that needs the plan
 * kernel recomputes and drops the pin; calls that plan for themselves, FD_TC_SELF_PLANNED and FD_TC_CLUSTER,
 * leave it alone).  The caller must not change the contents of the length arrays or of the page table while the
 * pin holds (from the second call it serves on, the kernel looks up its work and its first pages while the launch
 * before it on the stream is still running), and must unpin after a FD_DEV_TIMEOUT status (fd_last_device_status does so
 * itself when it reports that bit).  fd_kv_commit rewrites prefix_lens and therefore drops the pin
 * itself: the first attention call of the next step plans afresh (or is preceded by a new fd_plan_pin).
 * fd_kv_append leaves the lengths alone and keeps the pin.
 * Consecutive attention calls under one pin overlap on the device (fd_calls_back_to_back): a call starts while the call before it is still
 * finishing, and -- where its range of KV tiles is short -- reads its q and its cache ahead of that call's completion,
 * provided no earlier call since the pin wrote them (the library compares the `out` ranges of those calls with q and
 * kv_cache of this one; behind fd_kv_append, which writes the query block's own slots of the cache, the tiles that
 * lie wholly in the prefix are still read ahead, the ones that reach into the block after the append has completed).  fd_kv_append itself, behind an attention call of the chain, copies while that call finishes (its k_new /
 * v_new are checked against those `out` ranges in the same way).  Every write of an attention call (out, scratch)
 * waits for the launch before it, and the append waits for it before it ends, so results are those of calls run one
 * after the other.  What the library cannot see is a buffer written by the CALLER's own asynchronous work on another
 * stream: order such work before the call as usual.
 * The calls served by a pin must be ordered after fd_plan_pin (the
 * same stream, or streams the caller has ordered) and must not overlap one another: they share the context's
 * scratch memory, as all attention calls on one context do.
 * The paper does not describe a work list; this follows from "all layers of a step share the lengths".
 *
 *   prefix_lens, q_lens, n_mask   device, [B] int32;  n_blocks   device, [B] int32 or NULL
 */
fd_status fd_plan_pin(fd_ctx* ctx, int batch, int total_q_rows, const int32_t* prefix_lens, const int32_t* q_lens,
                      const int32_t* n_mask, const int32_t* n_blocks, void* stream);
fd_status fd_plan_unpin(fd_ctx* ctx);

/*
 * A whole step on device buffers in one call: for every layer the KV append (if k_new / v_new are given) and the
 * attention, on one work list (fd_plan_pin), then fd_verify_accept and fd_kv_commit -- the sequence of Sec. 4.1
 * "Inference" / Sec. 3, launched from C with nothing between the launches, so that consecutive calls overlap as under
 * fd_calls_back_to_back.  Everything a layer-by-layer caller gets from the single calls, this gives bit for bit.
 *
 *   q, k_new, v_new, kv_caches, out   HOST arrays of n_layers DEVICE pointers (k_new and v_new both NULL: no append);
 *                                     shapes per layer as fd_attn_draft_verify_blocks / fd_kv_append
 *   page_table, prefix_lens           device, in/out (the commit rewrites them)
 *   everything else                   device, as in the single calls; n_blocks may be NULL
 *
 * Asynchronous on `stream` like the single calls; errors as theirs (the first one is returned, later launches of the
 * step are skipped).
 */
fd_status fd_step_device(fd_ctx* ctx, int batch, int total_q_rows, int total_cand_rows, int n_layers,
                         const void* const* q, const void* const* k_new, const void* const* v_new,
                         void* const* kv_caches, void* const* out, int num_pages, int32_t* page_table,
                         int32_t* prefix_lens, const int32_t* q_lens, const int32_t* n_mask, const int32_t* n_blocks,
                         const float* logits, const int32_t* draft_tokens, int32_t* accepted_len,
                         int32_t* bonus_token, int32_t* freed_pages, int32_t* n_freed, void* stream);

/*
 * The caller's promise that lets consecutive calls overlap (default: off).  While on, the caller launches nothing of
 * its own on the stream between two calls on this context (a call on another context counts as the caller's own) --
 * the calls are back to back, as the layers of a benchmark step are, or as they are where everything between two
 * attention calls is itself ordered before the first of them.  The library then knows that the launch before a call is its own, and what that launch writes: see
 * fd_plan_pin (attention calls read q and the cache ahead, fd_kv_append copies under the tail of the attention call
 * before it) and fd_verify_accept (its sweep, like those of fd_verify_accept_sample and fd_draft_select, runs under
 * the tail of the attention call right before it).  Off, every call
 * waits for the launch before it before it reads anything but the pinned plan, the lengths and the page table: a
 * kernel of the caller's between two calls may then be any kernel, one that releases its dependents early included.
 * fd_step_host and fd_step_host_append, which launch nothing but this library's kernels, behave as if it were on.
 */
fd_status fd_calls_back_to_back(fd_ctx* ctx, int on);

/*
 * Host-side view of the work split, for schedulers and tests: how fd_attn_draft_verify cuts the 128-token KV
 * tiles of a call (numbered sequence-major, then kv-head, then position) into n_ranges contiguous ranges, one
 * per CTA of the tensor-core kernel.  Ranges have equal cost, a segment (sequence, kv-head) counting its tiles
 * plus a fixed start-up charge; a small call leaves the last ranges empty.  Runs on the CPU, touches no GPU.
 * The paper does not describe a work split; this is this library's own.
 *
 *   prefix_lens, q_lens   HOST, [B] int32 (a sequence has ceil((n_b + Lq_b) / 128) tiles per kv-head, none if Lq_b = 0)
 *   range_start           HOST, [n_ranges + 1] int32, out: first tile of every range; [n_ranges] = all tiles
 */
fd_status fd_plan_ranges_host(int batch, int n_kv_heads, const int32_t* prefix_lens, const int32_t* q_lens,
                              int n_ranges, int32_t* range_start);

/*
 * KV append, the step before the attention ("append, then attend").  The forward pass that verifies the
 * drafts also produces K/V for the query block; they enter the paged cache at logical positions
 * n_b .. n_b + Lq_b - 1 (candidates first, then mask tokens), where fd_attn_draft_verify reads them and
 * where, after fd_kv_commit has kept the accepted part, every later step finds them (Sec. 4.1
 * "Inference": the KV cache of the clean prefix is reused by all later steps).
 *
 *   k_new, v_new   device, [T, Hkv, d] bf16, 16-byte aligned, sequence-major rows
 *   kv_cache       device, [num_pages, 2, Hkv, P, d] bf16, in/out; only the slots of the block are written
 *   page_table     device, [B, max_pages_per_seq] int32: pages for positions up to n_b + Lq_b - 1 must be allocated
 *   prefix_lens, q_lens   device, [B] int32
 *
 * A sequence whose rows would pass T or the page table, or whose block is longer than max_q_len, is skipped
 * (FD_DEV_BAD_LENGTHS; append a longer one in pieces, n_b growing by what has been appended); a slot whose page
 * id is outside the pool is skipped (FD_DEV_BAD_PAGE).
 */
fd_status fd_kv_append(fd_ctx* ctx, int batch, int total_q_rows, const void* k_new, const void* v_new,
                       void* kv_cache, int num_pages, const int32_t* page_table,
                       const int32_t* prefix_lens, const int32_t* q_lens, void* stream);

/*
 * The same attention with several mask blocks per sequence: the parallel mode proper, in which the
 * forward pass that verifies the current draft also prepares one next-draft branch per hypothesis r
 * ("the first r drafts are accepted", Sec. 3 "Parallel speculative decoding", Eq. 2), each branch
 * conditioned on the prefix and on those r drafts only.
 *
 *   n_blocks   device, [B] int32, or NULL (= fd_attn_draft_verify).  nb_b = n_blocks[b]; 0 and 1 mean one
 *              block.  For nb_b > 1 the M_b mask rows are nb_b consecutive blocks of M_b / nb_b tokens
 *              (M_b divisible by nb_b, nb_b <= C_b); block g is the branch of hypothesis
 *              r = C_b - nb_b + g, so nb_b = C_b prepares every hypothesis r = 0..k_b.
 *
 *     A_b(i) for a mask row of block g:  { j < n_b } U { n_b + t : t <= r }  U  { its own block }
 *
 * (candidate row 0 is the known bonus token, candidate t the t-th draft); blocks never see each
 * other; candidate rows are as in fd_attn_draft_verify.  A query block may be as long as max_q_len
 * (the paper's full form, bonus + 16 drafts and 17 branches of 16 tokens, is 289 rows): 128 / G block
 * rows share one MMA tile per kv-head, a longer block is processed in several such row blocks.
 * Lengths that break the rules above zero all T rows (FD_DEV_BAD_LENGTHS).
 */
fd_status fd_attn_draft_verify_blocks(fd_ctx* ctx, int batch, int total_q_rows,
                                      const void* q, const void* kv_cache, int num_pages,
                                      const int32_t* page_table, const int32_t* prefix_lens,
                                      const int32_t* q_lens, const int32_t* n_mask,
                                      const int32_t* n_blocks, void* out, void* stream);

/*
 * Pages for the query blocks of a step, and where each of its rows goes: the counterpart of fd_kv_commit, which
 * releases pages.  (The paper describes no page management; the bookkeeping implemented here mirrors the commit's.)
 * The free list is a stack of page ids, free_pages[0 .. n_free).  First the n_freed ids the last commit released
 * are pushed onto it (freed_pages / n_freed exactly as fd_kv_commit wrote them; both NULL: nothing to push; batch 0:
 * nothing but that, which fd_kv_fork and fd_kv_compact ask for).  Then, for b ascending:
 *
 *     for p = ceil(n_b / P) .. ceil((n_b + Lq_b) / P) - 1 ascending:
 *         page_table[b][p] = the id popped from the top of the free list
 *
 * (what was in those entries is not looked at: after a commit they hold -1), and for row i of sequence b, at
 * logical position j = n_b + i:
 *
 *     slot_map[row0_b + i]  = page_table[b][j / P] * P + j % P
 *     positions[row0_b + i] = j                         for a candidate row (i < C_b)
 *                           = n_b + r + 1 + u           for token u of the mask block of hypothesis r (r = C_b - nb_b + g
 *                                                       for block g, as in fd_attn_draft_verify_blocks): the branch
 *                                                       continues behind the r drafts it presumes accepted
 *
 *   total_q_rows    T; must equal sum_b q_lens[b]
 *   page_table      device, [B, max_pages_per_seq] int32, in/out
 *   prefix_lens, q_lens, n_mask   device, [B] int32;  n_blocks   device, [B] int32 or NULL (one block each).  A block without
 *                   mask tokens (a prompt) may be longer than max_q_len
 *   freed_pages     device, int32, read only;  n_freed   device, [1] int32
 *   free_pages      device, [num_pages] int32, in/out
 *   n_free          device, [1] int32: ids on the free list before the call
 *   n_free_out      device, [1] int32: ids on it after the call; may be n_free itself
 *   num_pages       size of the page pool, num_pages * P < 2^31
 *   slot_map, positions   device, [T] int32, overwritten
 *
 * Fewer ids on the list than pages needed: nothing is popped and the table stays as it is, every slot is -1, the
 * positions are written (FD_DEV_NO_PAGES; the pushed ids are on the list).  Inconsistent lengths, or a list longer
 * than the pool: nothing is pushed or popped, every slot and position is -1, n_free_out = n_free
 * (FD_DEV_BAD_LENGTHS).  A page id outside the pool: its entry becomes -1 if it was popped, and the slots that need
 * it are -1 (FD_DEV_BAD_PAGE).  n_freed ids are pushed once per call: pass a commit's output to one call only.
 */
fd_status fd_kv_reserve(fd_ctx* ctx, int batch, int total_q_rows, int32_t* page_table, const int32_t* prefix_lens,
                        const int32_t* q_lens, const int32_t* n_mask, const int32_t* n_blocks,
                        const int32_t* freed_pages, const int32_t* n_freed, int32_t* free_pages,
                        const int32_t* n_free, int32_t* n_free_out, int num_pages, int32_t* slot_map,
                        int32_t* positions, void* stream);

/*
 * From the projection to the cache in one pass (the target model's own step between its QKV projection and
 * fd_attn_draft_verify; the paper's target models norm each query and key head and rotate it by its position).
 * Row t of qkv holds Hq query heads, then Hkv key heads, then Hkv value heads of d elements.  For a head x of q or k:
 *
 *     y = x / sqrt(mean_i x_i^2 + eps) * weight                          (weight NULL: y = x)
 *     for each pair (a, b) of FD_ROPE_* among the first R = rot_dim elements, pair number i, with c = cos_sin[pos][i],
 *     s = cos_sin[pos][R / 2 + i]:        y_a, y_b = y_a c - y_b s,  y_b c + y_a s
 *
 * with pos = positions[t].  q goes to q_out[t]; k and v go to the cache slot slot_map[t] (page slot / P, token slot % P).
 *
 *   total_q_rows    T >= 0; at most max_batch * max_q_len, any number with FD_KV_ROWS
 *   qkv             device, bf16, 16-byte aligned; row t starts at element t * row_stride (a multiple of 8, at least
 *                   (Hq + 2 Hkv) * d)
 *   q_weight, k_weight   device, [d] bf16, 16-byte aligned, or NULL: no norm
 *   eps             >= 0
 *   cos_sin         device, [max_positions, rot_dim] fp32, 16-byte aligned: cosines of a row, then its sines
 *   rot_dim         R: a multiple of 16, 0 <= R <= d (0: no rotation, cos_sin and positions may be NULL)
 *   rope_style      FD_ROPE_HALVES or FD_ROPE_ADJACENT
 *   positions, slot_map   device, [T] int32 (fd_kv_reserve writes both)
 *   q_out           device, [T, Hq, d] bf16, 16-byte aligned, does not overlap qkv
 *   kv_cache        device, the cache of kv_format: bf16 pages (128-byte aligned), 4-bit pages or rows (16-byte aligned)
 *   kv_format       FD_KV_BF16, FD_KV_FP4 or FD_KV_ROWS
 *   k_scale, v_scale   FD_KV_FP4: as in fd_kv_append_fp4; otherwise not used
 *
 * A row whose slot is negative is padding: nothing is written for it.  A slot beyond the pool: k and v of the row are
 * not written (FD_DEV_BAD_PAGE).  A position outside [0, max_positions): nothing is written for the row
 * (FD_DEV_BAD_LENGTHS).  Two rows of a call with the same slot leave a mixture of the two there (codes and scales are stored
 * apart): give each row a slot of its own, as fd_kv_reserve does.
 * Arithmetic: fp32 throughout, each result rounded once, to bf16 or to 4 bits.
 */
fd_status fd_qk_norm_rope_append(fd_ctx* ctx, int total_q_rows, const void* qkv, int64_t row_stride,
                                 const void* q_weight, const void* k_weight, float eps, const float* cos_sin,
                                 int max_positions, int rot_dim, int rope_style, const int32_t* positions,
                                 const int32_t* slot_map, void* q_out, void* kv_cache, int num_pages, int kv_format,
                                 float k_scale, float v_scale, void* stream);

/*
 * A KV cache held in 4 bits: attention over it, and the ways into and out of it.  At long context the step is bound by the
 * bytes of the cache; these pages are 9/32 the size of bf16 pages.  (The paper keeps its cache in bf16; this is the
 * library's own.)  Every 16 consecutive elements of a head's row share an e4m3 scale and are held as e2m1 codes
 * (bit 3 the sign; 0..7 stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6); all of K is scaled by k_scale on top, all of V by v_scale
 * (positive, finite; the same numbers in every call on a cache):
 *
 *     value = code * scale * k_scale
 *     scale = the e4m3 number nearest to max_i |x_i / k_scale| / 6, at most 448         (nearest, ties to even)
 *     code  = the e2m1 number whose multiple of the scale is nearest to x / k_scale      (nearest, ties to even; 6 at most)
 *
 * with fp32 quotients, each correctly rounded (where x / k_scale is not exact, what is nearer to a tie than that counts as one).
 * A NaN is held as 0, an infinity as the largest value of its group's scale.  Zero scale: all codes of the group are zeros.
 *
 *   cache layout    [num_pages, Hkv, 2, P * (d / 2 + d / 16)] bytes, 16-byte aligned: for each page and kv-head K then V,
 *                   each as [P][d / 2] bytes of codes (element 2 i in the low half of byte i) followed by [P][d / 16]
 *                   bytes of scales
 *
 * When to choose it: it holds 3.6 times the tokens in the same memory.  Its attention is faster than the bf16 cache's on long
 * prefixes (32k: 330 to 380 us against 400 to 440 for a batch of 16), about as fast for a batch of 64 on 1k to 4k, and slower
 * on small batches (8 sequences: 44 us against 38; one: 14 against 12).
 *
 * fd_kv_append_fp4 is fd_kv_append for it, fd_kv_read_fp4 the reverse: k_out / v_out [T, Hkv, d] bf16 get the values held
 * at positions n_b .. n_b + Lq_b - 1 (any range of the sequence: pass the range's start as prefix_lens), rounded to bf16.
 * A sequence that is skipped, or a slot whose page id is outside the pool, leaves its rows of k_out / v_out as zeros.
 * Arguments and device-detected errors are fd_kv_append's.  Neither call, nor fd_qk_norm_rope_append, overlaps the calls around
 * it: under a pinned plan the attention call behind one starts when it has completed, as behind a kernel of the caller's.
 *
 * fd_attn_draft_verify_fp4 is fd_attn_draft_verify_blocks for it: same arguments (n_blocks may be NULL), same mask, same
 * errors, same forms (FD_TC_*), pinned plans and overlap of consecutive attention calls included.  fd_step_device and fd_step_host
 * work on bf16 caches: a step on this one is put together from the single calls.  Slots no valid token owns may hold
 * any bit pattern.  Arithmetic: the values of the cache enter exactly, q is held in at least as many bits as bf16
 * relative to its row's largest element, the softmax weights in 11 bits down to 2^-21 of the row's largest (below that to
 * within 2^-32 of it), sums in fp32; bf16 output.
 */
fd_status fd_kv_append_fp4(fd_ctx* ctx, int batch, int total_q_rows, const void* k_new, const void* v_new,
                           void* kv_cache, int num_pages, const int32_t* page_table, const int32_t* prefix_lens,
                           const int32_t* q_lens, float k_scale, float v_scale, void* stream);
fd_status fd_kv_read_fp4(fd_ctx* ctx, int batch, int total_q_rows, const void* kv_cache, int num_pages,
                         const int32_t* page_table, const int32_t* prefix_lens, const int32_t* q_lens, float k_scale,
                         float v_scale, void* k_out, void* v_out, void* stream);
fd_status fd_attn_draft_verify_fp4(fd_ctx* ctx, int batch, int total_q_rows, const void* q, const void* kv_cache,
                                   int num_pages, const int32_t* page_table, const int32_t* prefix_lens,
                                   const int32_t* q_lens, const int32_t* n_mask, const int32_t* n_blocks,
                                   float k_scale, float v_scale, void* out, void* stream);

/*
 * A KV cache held in 8 bits: attention over it, and the ways into and out of it.  Half the size of bf16 pages (0.504 of it at
 * d = 128), four significant bits an element where the 4-bit cache has two.  (The paper keeps its cache in bf16; this is the
 * library's own.)  The P tokens of a page share, for each kv-head and for K and V apart, one scale; every element is an e4m3 code:
 *
 *     value = code * scale
 *     scale = the smallest power of two, from 2^-15 to 2^7, for which the largest magnitude among the block's tokens is at most
 *             448 * scale (2^7 where none is: then larger elements, infinities too, are held as 57344)
 *     code  = the e4m3 number nearest to x / scale                                     (nearest, ties to even; a NaN stays one)
 *
 *   cache layout    [num_pages, Hkv, 2, P * d + 16] bytes, 16-byte aligned: for each page and kv-head K then V, each as [P][d]
 *                   codes followed by the scale as a 32-bit float and 12 bytes of zeros
 *
 * The block's tokens are those of its sequence at positions below n_b + Lq_b.  When tokens join a block that is begun, those at
 * positions below n_b keep their values, expressed in the new scale: exactly, unless the scale has grown so far that a code
 * falls among e4m3's subnormals, where it is rounded again (nearest, ties to even).  Bytes of positions no token owns are
 * left as they are, and do not count for the scale.  So what a block holds depends on its tokens and, within those subnormals,
 * on the order in which they came.
 *
 * fd_kv_append_fp8 is fd_kv_append for it, fd_kv_read_fp8 the reverse: k_out / v_out [T, Hkv, d] bf16 get the values held
 * at positions n_b .. n_b + Lq_b - 1 (any range of the sequence: pass the range's start as prefix_lens), exactly.  Lq_b is not
 * bounded by max_q_len in either.  A sequence that is skipped, or a slot whose page id is outside the pool, leaves its rows of
 * k_out / v_out as zeros.  Arguments and device-detected errors are otherwise fd_kv_append's.  A page that two sequences of a call name is
 * written by both: let each append to pages of its own, as fd_kv_reserve and fd_kv_fork hand out.  Neither call overlaps the
 * calls around it: under a pinned plan the attention call behind one starts when it has completed.
 *
 * fd_attn_draft_verify_fp8 is fd_attn_draft_verify_blocks for it: same arguments (n_blocks may be NULL), same mask, same
 * errors, same forms (FD_TC_*), pinned plans and overlap of consecutive attention calls included.  Slots no valid token owns may
 * hold any bit pattern.  Arithmetic: the values of the cache enter exactly, elements of q exactly down to 2^-9 of their row's
 * largest (below that to within 2^-17 of it), the softmax weights as in fd_attn_draft_verify_fp4, sums in fp32; bf16 output.  A row
 * of q that holds a NaN or an infinity becomes NaN.
 * When to choose it: it holds twice the tokens in the same memory at four significant bits.  Its attention is faster than the bf16
 * cache's on long prefixes (32k, batch 16: 319 us against 351 in short runs, 376 against 429 call after call for a second), about as fast for
 * 64 sequences of 1k to 4k (127 against 116, 128 against 135) and slower for few (8 sequences: 43 against 38; one: 12.4 against 10.9).
 */
fd_status fd_kv_append_fp8(fd_ctx* ctx, int batch, int total_q_rows, const void* k_new, const void* v_new,
                           void* kv_cache, int num_pages, const int32_t* page_table, const int32_t* prefix_lens,
                           const int32_t* q_lens, void* stream);
fd_status fd_kv_read_fp8(fd_ctx* ctx, int batch, int total_q_rows, const void* kv_cache, int num_pages,
                         const int32_t* page_table, const int32_t* prefix_lens, const int32_t* q_lens, void* k_out,
                         void* v_out, void* stream);
fd_status fd_attn_draft_verify_fp8(fd_ctx* ctx, int batch, int total_q_rows, const void* q, const void* kv_cache,
                                   int num_pages, const int32_t* page_table, const int32_t* prefix_lens,
                                   const int32_t* q_lens, const int32_t* n_mask, const int32_t* n_blocks, void* out,
                                   void* stream);

/*
 * Attention of whole prompts, or of chunks of them, over their own keys (what a sequence goes through before its first decode
 * step; the paper starts behind it).  Sequences are packed one behind the other, rows [T, Hq, d] of q and [Tk, Hkv, d] of k and v;
 * sequence b has Lq_b query rows and Lk_b keys, and its last row is the position of its last key.  Row i, q-head h:
 *
 *     out[row0_b + i, h, :] = sum_{j <= i + Lk_b - Lq_b} softmax_j( scale * <q[row0_b + i, h], k_b[j, h/G]> ) v_b[j, h/G]
 *
 * A row that sees no key (Lk_b < Lq_b has such rows, in front) becomes zeros.  Lengths are not bounded by max_q_len or by
 * max_pages_per_seq; scale is the context's.
 *
 *   batch           B, 0 <= B <= max_batch (B = 0 is a no-op)
 *   total_q_rows    T; must equal sum_b q_lens[b]          total_kv_rows   Tk; must equal sum_b kv_lens[b]
 *   q, k, v         device, bf16, 16-byte aligned; row t of q starts at element t * q_stride, of k and v at t * kv_stride (multiples
 *                   of 8, at least Hq * d and Hkv * d: slices of one projection's output will do); k and v NULL only with Tk = 0
 *   q_lens          device, [B] int32
 *   kv_lens         device, [B] int32, or NULL: the same as q_lens
 *   out             device, [T, Hq, d] bf16, 16-byte aligned; fully overwritten; shares no bytes with q, k or v
 *
 * Inconsistent lengths zero all T rows (FD_DEV_BAD_LENGTHS).  What a row must not see -- another sequence, a later position --
 * never reaches it, infinities and NaN included.
 *
 * A prompt's way into a cache, whatever max_q_len: fd_kv_reserve, fd_qk_norm_rope_append with FD_KV_ROWS, this call,
 * fd_kv_append_fp8 or fd_kv_append_fp4 (into bf16 pages fd_kv_append, in pieces of max_q_len rows), and fd_kv_commit with
 * accepted_len[b] = Lq_b - 1.  A chunk behind earlier keys takes all of them as rows: fd_kv_read_fp8 and fd_kv_read_fp4 bring them out
 * of pages.  Over pages as they are -- bf16 ones have no such call -- fd_attn_draft_verify and its 4-bit and 8-bit forms are causal
 * attention too where n_mask is 0, for chunks of up to max_q_len rows that have been appended.
 * Arithmetic: bf16 inputs, fp32 scores / softmax / accumulation, softmax weights rounded to bf16 in front of the product with v,
 * bf16 output.
 */
fd_status fd_attn_prompt(fd_ctx* ctx, int batch, int total_q_rows, int total_kv_rows, const void* q, int64_t q_stride,
                         const void* k, const void* v, int64_t kv_stride, const int32_t* q_lens, const int32_t* kv_lens,
                         void* out, void* stream);

/*
 * The pages of sequences that branch (several samples of one prompt), of sequences that end, and of a pool that is to be
 * compacted.  Tables and lists are the same for all layers; each layer's cache then takes the copies (fd_kv_copy_pages).  (The paper
 * describes no page management.)
 *
 *   shared   device, [num_pages] int32: owners of each page beyond its first; 0 for a free page and for one that has never been
 *            forked.  fd_kv_reserve and fd_kv_commit hand out and release only pages behind a sequence's whole prefix pages,
 *            which are never shared, and need not know of it.
 *   page_table, prefix_lens   device, [batch, max_pages_per_seq] and [batch] int32, in/out
 *   free_pages, n_free, n_free_out   the free list, as in fd_kv_reserve (n_free_out may be n_free itself)
 *   num_pages * P < 2^31
 *
 * Call them between steps, behind fd_kv_commit: fork and free do not look at pages reserved for a query block that has not been
 * committed.  The ids that the commit released have to be on the free list by then.  fd_kv_compact takes every id that is not on it
 * for a page in use and gives it another number, so that a commit's ids pushed behind it would be on the list twice and two sequences
 * would write the same page; fd_kv_fork finds pages on the list only.  A reservation for no sequence pushes them (and the next
 * reservation then gets none of them):
 *
 *     fd_kv_reserve(ctx, 0, 0, NULL, NULL, NULL, NULL, NULL, freed_pages, n_freed, free_pages, n_free, n_free, num_pages, NULL, NULL, stream)
 *
 * Whatever else holds ids outside of page_table and the list while fd_kv_compact runs has to replace them by page_map[id].
 *
 * fd_kv_fork: child children[i] becomes a copy of parents[i], for i ascending.  With n = prefix_lens[parent], f = floor(n / P):
 *
 *     page_table[child][p] = page_table[parent][p],  shared[that page] += 1                            for p < f
 *     n % P > 0:  page_table[child][f] = the id popped from the free list;  copy_src[i], copy_dst[i] = page_table[parent][f], that id
 *     otherwise copy_src[i] = copy_dst[i] = -1;  entries of the child's row behind these = -1;  prefix_lens[child] = n
 *
 * (what was in the child's row is not looked at: free it first).  copy_src, copy_dst: device, [n_forks] int32, written.  Too few
 * ids on the list: nothing is done, the copies are -1 (FD_DEV_NO_PAGES).  An index outside [0, batch), a child named twice or named as
 * a parent too, a length that is negative or beyond the table: nothing is done, the copies are -1 (FD_DEV_BAD_LENGTHS).  A page
 * id outside the pool: not shared (its entry in the child's row is -1), or not copied (FD_DEV_BAD_PAGE).
 *
 * fd_kv_free: the sequences seqs[i] give their pages back, for i descending, from the last page of the prefix to the first:
 *
 *     shared[id] > 0:  shared[id] -= 1;      otherwise id is pushed onto the free list
 *
 * and page_table[seq][p] = -1, prefix_lens[seq] = 0.  (Freeing in the order of forking, or of reserving, leaves the list as it
 * was before.)  An index outside [0, batch), a sequence listed twice, a length negative or beyond the table, a sequence of 2^21
 * pages or more, 2^29 of them in all: nothing is done (FD_DEV_BAD_LENGTHS).  An id outside the pool, or held by more sequences than shared says: dropped, or pushed once
 * (FD_DEV_BAD_PAGE).
 *
 * fd_kv_compact: the m = num_pages - n_free pages that are not on the free list move to ids 0 .. m - 1.  Pages below m stay; the
 * i-th page in use at or above m (ascending) moves to the i-th free id below m:  copy_src[i], copy_dst[i].  Then
 *
 *     page_map[id] = where page id is now, -1 for a page that was free;  every id in the table is replaced by its page_map
 *     shared moves with its pages (shared may be NULL);  free_pages[k] = num_pages - 1 - k for k < n_free (m on top)
 *
 *   page_map   device, [num_pages] int32, written          n_copies   device, [1] int32, written: moves
 *   copy_src, copy_dst   device, [max_copies] int32, written, -1 behind the moves;  min(m, n_free) are enough
 *
 * An id listed twice or outside the pool (FD_DEV_BAD_PAGE), a list longer than the pool, more moves than max_copies
 * (FD_DEV_BAD_LENGTHS): tables, list and shared stay, page_map is the identity, n_copies = 0, the copies are -1.
 *
 * fd_kv_copy_pages: page copy_dst[i] of one layer's cache becomes a copy of page copy_src[i], for i < *n_copies (NULL: for
 * i < max_copies).  A pair with a negative id is skipped; one with an id beyond the pool too (FD_DEV_BAD_PAGE).  The copies of a call
 * are made in no particular order: no page may be the target of two of them, or the target of one and the source of another.
 *
 *   kv_cache   device, the cache of kv_format (FD_KV_BF16, FD_KV_FP4, FD_KV_FP8), 16-byte aligned
 */
fd_status fd_kv_fork(fd_ctx* ctx, int n_forks, const int32_t* parents, const int32_t* children, int batch,
                     int32_t* page_table, int32_t* prefix_lens, int32_t* shared, const int32_t* free_pages,
                     const int32_t* n_free, int32_t* n_free_out, int num_pages, int32_t* copy_src, int32_t* copy_dst,
                     void* stream);
fd_status fd_kv_free(fd_ctx* ctx, int n_seqs, const int32_t* seqs, int batch, int32_t* page_table, int32_t* prefix_lens,
                     int32_t* shared, int32_t* free_pages, const int32_t* n_free, int32_t* n_free_out, int num_pages,
                     void* stream);
fd_status fd_kv_compact(fd_ctx* ctx, int batch, int32_t* page_table, int32_t* shared, int32_t* free_pages,
                        const int32_t* n_free, int num_pages, int32_t* page_map, int max_copies, int32_t* copy_src,
                        int32_t* copy_dst, int32_t* n_copies, void* stream);
fd_status fd_kv_copy_pages(fd_ctx* ctx, int max_copies, const int32_t* n_copies, const int32_t* copy_src,
                           const int32_t* copy_dst, void* kv_cache, int num_pages, int kv_format, void* stream);

/*
 * Draft-side tail of the step (Sec. 4.2, Eq. 4; Sec. 4.3 "Selective verification", Eq. 5).  One row of
 * draft logits per mask token, sequence-major.  Calibrated logits l~ = l + bias (the bias is the output of
 * the calibration MLP of Eq. 4, evaluated by the caller; NULL = no calibration); the drafted token of a
 * row is argmax l~ (lowest index on ties, inputs NaN-free), its confidence p = softmax(l~)[token].  Within
 * every next-draft block (nb_b equal blocks per sequence, as in fd_attn_draft_verify_blocks) the cumulative
 * confidence of position i is prod_{r <= i} p_r -- Eq. 5's estimate of P(L_acc >= i) -- and keep_len of the
 * block is the number of leading positions where it is still >= threshold: how many of that branch's
 * drafts the next step should verify (its candidate rows are then 1 + keep_len).
 *
 *   total_mask_rows  Rm; must equal sum_b n_mask[b]
 *   max_blocks       row length of keep_len; every nb_b must be <= max_blocks
 *   draft_logits     device, [Rm, V] fp32            bias   device, [Rm, V] fp32, or NULL
 *   n_mask, n_blocks device, [B] int32 (n_blocks may be NULL)
 *   threshold        >= 0
 *   mask_tokens      device, [Rm] int32, written     mask_probs   device, [Rm] fp32, written
 *   keep_len         device, [B, max_blocks] int32, written (0 where a sequence has fewer blocks)
 *
 * Arithmetic: l + bias, the maxima and the confidences in fp32 (the sum of exponentials is accumulated in a
 * fixed order, so results are run-to-run identical).  Inconsistent lengths: tokens -1, confidences 0,
 * keep_len 0, FD_DEV_BAD_LENGTHS.
 */
fd_status fd_draft_select(fd_ctx* ctx, int batch, int total_mask_rows, int max_blocks,
                          const float* draft_logits, const float* bias,
                          const int32_t* n_mask, const int32_t* n_blocks, float threshold,
                          int32_t* mask_tokens, float* mask_probs, int32_t* keep_len, void* stream);

/*
 * Branch selection (Sec. 3: once verification has fixed r_acc, the branch prepared under that
 * hypothesis is the next draft).  mask_tokens holds one proposed token per mask row, sequence-major
 * ([sum_b M_b] int32, device).  For each sequence the block g = accepted_len[b] - (C_b - nb_b) is copied to
 * next_draft[b, 0:kb] (device, [B, max_block_len] int32, padded with -1) and next_len[b] = kb; when that
 * hypothesis was not prepared (g outside [0, nb_b)), the sequence has no mask rows, or
 * accepted_len[b] < 0, next_len[b] = 0.  A block longer than max_block_len raises FD_DEV_BAD_LENGTHS.
 */
fd_status fd_select_branch(fd_ctx* ctx, int batch, int max_block_len, const int32_t* mask_tokens,
                           const int32_t* q_lens, const int32_t* n_mask, const int32_t* n_blocks,
                           const int32_t* accepted_len, int32_t* next_draft, int32_t* next_len, void* stream);

/*
 * Lossless verification at temperature 0 (Sec. 3: draft tokens are accepted up to the
 * first rejection, the token produced there is the bonus token, committed length
 * L_acc = r_acc + 1).  With am[r] = argmax_v logits[r, v] (larger value wins, equal
 * values: lower index wins; inputs must be NaN-free) and r0_b the first candidate row of
 * sequence b:
 *
 *     accepted_len[b] = number of leading j < k_b with am[r0_b + j] == draft_tokens[r0_b + j + 1]
 *     bonus_token[b]  = am[r0_b + accepted_len[b]]
 *
 * so 0 <= accepted_len[b] <= k_b = C_b - 1 (this is the paper's r_acc).  A sequence with
 * C_b = 0 gets accepted_len = bonus_token = -1.
 *
 *   total_cand_rows  R; must equal sum_b (q_lens[b] - n_mask[b])
 *   logits           device, [R, V] fp32, candidate rows only, sequence-major
 *   draft_tokens     device, [R] int32: the token fed at each candidate row (row 0 of a
 *                    sequence is the previous bonus token and is never compared)
 *   q_lens, n_mask   device, [B] int32
 *   accepted_len, bonus_token   device, [B] int32, overwritten
 *
 * Inconsistent lengths: every accepted_len / bonus_token is set to -1 (FD_DEV_BAD_LENGTHS).
 * Right behind an attention call of the same context (fd_calls_back_to_back) the sweep over the logits starts while that
 * call is still finishing (neither reads what the other writes); the results are written after it has completed.
 */
fd_status fd_verify_accept(fd_ctx* ctx, int batch, int total_cand_rows,
                           const float* logits, const int32_t* draft_tokens,
                           const int32_t* q_lens, const int32_t* n_mask,
                           int32_t* accepted_len, int32_t* bonus_token, void* stream);

/*
 * Verification at temperature > 0 by speculative sampling (Sec. 3: whether a draft is kept depends on how
 * the target's probability p of the drafted token compares with the drafter's q; where the first draft is
 * dropped, the bonus token is drawn from what is left of p once q is taken out; committed length = accepted + 1).
 * Rows and draft_tokens as in fd_verify_accept.  With p_j = softmax(logits[row j] / T) and q_j =
 * softmax(draft_logits[row j] / T), draft j + 1 = x is accepted iff u_accept[row j] < min(1, p_j(x) / q_j(x));
 * rejected at j: bonus ~ max(0, p_j - q_j) normalised; all k accepted: bonus ~ p_k.  A token is drawn from
 * weights w by inverting their cumulative sum in index order at u_bonus[b] * sum(w).
 *
 *   logits        device, [R, V] fp32: target logits of the candidate rows
 *   draft_logits  device, [R, V] fp32 or NULL: row r holds the (calibrated) draft logits the token fed at row
 *                 r + 1 was proposed from; NULL = the drafter put all its mass on the proposed token
 *   temperature   > 0
 *   u_accept      device, [R] fp32 in [0, 1): one uniform per candidate row (a sequence's last row: unused)
 *   u_bonus       device, [B] fp32 in [0, 1)
 *   accepted_len, bonus_token   device, [B] int32, out; -1 for a sequence without candidate rows
 *
 * Probabilities are formed in fp32; a decision whose two sides differ by less than fp32 rounding may fall
 * either way.  Lengths that do not add up to R raise FD_DEV_BAD_LENGTHS.
 */
fd_status fd_verify_accept_sample(fd_ctx* ctx, int batch, int total_cand_rows, const float* logits,
                                  const float* draft_logits, const int32_t* draft_tokens, const int32_t* q_lens,
                                  const int32_t* n_mask, float temperature, const float* u_accept,
                                  const float* u_bonus, int32_t* accepted_len, int32_t* bonus_token, void* stream);

/*
 * KV commit / rollback.  The paper implies it (the clean-prefix KV cache is reused by
 * every later step, Sec. 4.1 "Inference" and Sec. 4.3 "Decoupled execution"; mask tokens
 * are invisible to clean tokens) without spelling it out; the reading implemented: the
 * bonus row and the accepted drafts stay, every later position of the block (rejected
 * drafts, mask tokens) is dropped by truncating the length and releasing the pages that
 * no kept token lives in.  For b ascending, with new_len = n_b + accepted_len[b] + 1:
 *
 *     for p = ceil(new_len / P) .. ceil((n_b + Lq_b) / P) - 1 ascending:
 *         append page_table[b][p] to freed_pages; page_table[b][p] = -1
 *     prefix_lens[b] = new_len
 *
 * KV bytes are not touched.  Sequences with accepted_len[b] < 0 are left unchanged; one with
 * accepted_len[b] >= q_lens[b] is left unchanged and raises FD_DEV_BAD_ACCEPT.
 *
 *   page_table    device, [B, max_pages_per_seq] int32, in/out
 *   prefix_lens   device, [B] int32, in/out
 *   q_lens, accepted_len   device, [B] int32
 *   freed_pages   device, int32, packed output; capacity >= B * (ceil(max_q_len / P) + 1), or, where a block is longer than
 *                 max_q_len, sum_b (ceil(Lq_b / P) + 1)
 *   n_freed       device, [1] int32, output
 */
fd_status fd_kv_commit(fd_ctx* ctx, int batch, int32_t* page_table, int32_t* prefix_lens,
                       const int32_t* q_lens, const int32_t* accepted_len,
                       int32_t* freed_pages, int32_t* n_freed, void* stream);

/*
 * One whole decode step from HOST buffers: the attention of n_layers layers, the verification
 * and the commit (the three calls above, in the order of Sec. 4.1 "Inference"), with every
 * per-step input copied up and every result copied back by the library.  The KV caches are
 * decode state and stay on the device; all other pointers are host pointers (pinned memory
 * makes the copies asynchronous and lets them overlap the kernels; pageable memory works but
 * serialises).  Copies run on two internal streams so that q of layer l+1 goes up and out of
 * layer l-1 comes back while layer l computes; one cudaMemcpyAsync per buffer.
 *
 * fd_host_reserve(ctx, max_total_q_rows, max_total_cand_rows) allocates the device staging
 * (2 x q, 2 x out, 2 x the block's K and V, logits, small arrays) and the copy streams once; it is the only part that
 * allocates and must precede fd_step_host.  A second call with sizes within the first is a
 * no-op; larger sizes return FD_ERR_INVALID_ARG.
 *
 *   kv_caches         host array of n_layers device pointers, each [num_pages, 2, Hkv, P, d] bf16
 *   q_host            [n_layers][T, Hq, d] bf16          out_host   [n_layers][T, Hq, d] bf16, written
 *   logits_host       [R, V] fp32                        draft_tokens_host [R] int32
 *   page_table_host   [B, max_pages_per_seq] int32, in/out (the commit's edits come back)
 *   prefix_lens_host  [B] int32, in/out                  q_lens_host, n_mask_host [B] int32
 *   n_blocks_host     [B] int32 mask blocks per sequence (see fd_attn_draft_verify_blocks), or NULL
 *   accepted_len_host, bonus_token_host [B] int32, written
 *   freed_pages_host  capacity B * (ceil(max_q_len / P) + 1) int32, written; n_freed_host [1]
 *
 * The call returns after enqueueing; `stream` has finished the step, results on the host
 * included, once everything enqueued on it has completed.  The host buffers must stay valid
 * and untouched until then.  Steps on one context must not overlap.
 */
fd_status fd_host_reserve(fd_ctx* ctx, int max_total_q_rows, int max_total_cand_rows);
fd_status fd_step_host(fd_ctx* ctx, int batch, int total_q_rows, int total_cand_rows, int n_layers,
                       const void* const* kv_caches, int num_pages, const void* q_host, void* out_host,
                       const float* logits_host, const int32_t* draft_tokens_host,
                       int32_t* page_table_host, int32_t* prefix_lens_host,
                       const int32_t* q_lens_host, const int32_t* n_mask_host,
                       const int32_t* n_blocks_host,
                       int32_t* accepted_len_host, int32_t* bonus_token_host,
                       int32_t* freed_pages_host, int32_t* n_freed_host, void* stream);

/*
 * The same step with the KV append inside (Sec. 4.1 "Inference": the K/V that the target's own forward pass
 * computes for the query block go into the cache, where this step's attention and every later step find them).
 * Per layer the block's K/V go up with its q, fd_kv_append writes them into the layer's pages, and the attention
 * call follows on the same stream under programmatic dependent launch (its set-up overlaps the append's tail).
 *
 *   k_new_host, v_new_host   [n_layers][T, Hkv, d] bf16, rows sequence-major as q; both NULL = fd_step_host
 *   kv_caches                as above, but written: positions n_b .. n_b + Lq_b - 1 of every sequence
 */
fd_status fd_step_host_append(fd_ctx* ctx, int batch, int total_q_rows, int total_cand_rows, int n_layers,
                              void* const* kv_caches, int num_pages, const void* q_host, const void* k_new_host,
                              const void* v_new_host, void* out_host, const float* logits_host,
                              const int32_t* draft_tokens_host, int32_t* page_table_host, int32_t* prefix_lens_host,
                              const int32_t* q_lens_host, const int32_t* n_mask_host, const int32_t* n_blocks_host,
                              int32_t* accepted_len_host, int32_t* bonus_token_host, int32_t* freed_pages_host,
                              int32_t* n_freed_host, void* stream);

/*
 * fd_verify_accept without any allocation.  (The paper has no counterpart; this entry point
 * exists for the callers described here.)
 *
 * Who needs it: code that must not call cudaMalloc -- a plugin running inside a serving
 * process whose memory pool owns every byte of the device, a step that runs while a CUDA
 * graph is being captured elsewhere in the process, a late-initialised worker that finds the
 * device already full.  fd_create() is closed to such callers because it allocates the
 * context's scratch memory.  This call needs no context: the (value, index) maxima of the
 * vocabulary sweep and the finished-CTA counter live in a fixed array compiled into the
 * library (FD_STATIC_MAX_ROWS * 8 bytes + 64 bytes = 32.06 KB of device memory on every GPU
 * that loads the library, held until the process exits).
 *
 * Semantics, argument layout and results are those of fd_verify_accept, with these changes:
 *   vocab           V, passed per call (there is no fd_config)
 *   device_status   device pointer to one int32 that receives FD_DEV_* bits (OR-ed in; the
 *                   caller clears it), or NULL to drop them
 * Limits: total_cand_rows <= FD_STATIC_MAX_ROWS and batch <= FD_STATIC_MAX_BATCH, else
 * FD_ERR_STATIC_LIMIT is returned and nothing is launched.
 *
 * The call allocates nothing: no cudaMalloc / cudaFree, no allocating library routine; it
 * enqueues two small cudaMemsetAsync (the part of the array it is about to use keeps the
 * previous call's contents and must start at zero) and one kernel on `stream`.
 * First call on each device: the device address of the array is looked up once
 * (cudaGetSymbolAddress, with that device current) and cached; make that first call outside
 * any stream capture.
 * Every call in the process shares the one array per device.  Calls issued on one stream are
 * safe back to back; calls that can overlap on the GPU (different streams, different threads,
 * different contexts of the same library image) race on it and must be serialised by the caller.
 */
#define FD_STATIC_MAX_ROWS 4096
#define FD_STATIC_MAX_BATCH 4096
fd_status fd_verify_accept_static(int vocab, int batch, int total_cand_rows,
                                  const float* logits, const int32_t* draft_tokens,
                                  const int32_t* q_lens, const int32_t* n_mask,
                                  int32_t* accepted_len, int32_t* bonus_token,
                                  int32_t* device_status, void* stream);

/* Read and clear the sticky device status word (an OR of FD_DEV_* bits) into *code (host
 * pointer).  Synchronises `stream` first. */
fd_status fd_last_device_status(fd_ctx* ctx, int32_t* code, void* stream);

/* Failure-detection self-test (no counterpart in the paper).  Every device-side wait of the
 * attention kernel is bounded: when it runs out, the kernel stops cleanly and raises
 * FD_DEV_TIMEOUT instead of hanging the GPU.  This call exercises exactly that mechanism on a
 * barrier that nothing will ever signal: one warp waits for `limit_ms` (1..1000) milliseconds,
 * gives up, sets FD_DEV_TIMEOUT in the status word and returns.  The context stays usable. */
fd_status fd_selftest_wait_timeout(fd_ctx* ctx, int limit_ms, void* stream);

/* Which attention kernel the context resolved to: FD_ATTN_SIMT or FD_ATTN_TCGEN05. */
int fd_attn_path(const fd_ctx* ctx);

/* FD_TC_* of the context's most recent tensor-core attention call, -1 before the first one. */
int fd_attn_last_mode(const fd_ctx* ctx);

/* Number of CUDA kernels this library has launched through `ctx` since fd_create. */
int64_t fd_launch_count(const fd_ctx* ctx);

/* Static string for a status code. */
const char* fd_status_string(fd_status s);

#ifdef __cplusplus
}
#endif
#endif /* FLEXDRAFT_H */
