"""GPU tests of the 4-bit cache: consecutive and captured attention calls, rows of a tile that no query owns, head counts far
above the usual ones."""
import numpy as np
import pytest
import torch

import fp4_ref as ref
import paper_2605_20022_b200 as fd
from helpers import Ctx
from paper_2605_20022_b200 import workload as wl
from test_gpu_parity import PATHS, _random_step
from test_gpu_serving import attn_ref, check

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.view(torch.int16)


# ---------------------------------------------------------------------------------------------- consecutive calls under a pin
def _chain(ctx, step, n_blocks, layers, q0, pools, kv_pool, k_new, v_new, table, wait_between):
    """Attention calls under one pinned plan.  A layer is (format, query, append): on 4-bit ("4") or bf16 ("b") pages, from q0 (0)
    or the output k layers back (k), behind an append to the bf16 pool or not."""
    T = step.total_q_rows
    ints = [table, step.prefix_lens.cuda(), step.q_lens.cuda()]
    nm, nb = step.n_mask.cuda(), n_blocks.cuda()
    outs = [torch.full(q0.shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in layers]
    kv_pool = kv_pool.clone()
    torch.cuda.synchronize()
    fd.fd_plan_pin(ctx.h, step.batch, T, ints[1], ints[2], nm, nb)
    for l, (fmt, back, append) in enumerate(layers):
        x = outs[l - back] if back else q0
        if append:
            fd.fd_kv_append(ctx.h, step.batch, T, k_new, v_new, kv_pool, step.num_pages, *ints)
        if fmt == "4":
            fd.fd_attn_draft_verify_fp4(ctx.h, step.batch, T, x, pools[l % len(pools)], step.num_pages, *ints, nm, nb, 1.0, 1.0, outs[l])
        else:
            fd.fd_attn_draft_verify_blocks(ctx.h, step.batch, T, x, kv_pool, step.num_pages, *ints, nm, nb, outs[l])
        if wait_between:
            torch.cuda.synchronize()
    fd.fd_plan_unpin(ctx.h)
    return outs, fd.fd_last_device_status(ctx.h)


# every start that a 4-bit call can make: behind a call that does not write its query (reading ahead), behind one that does, behind
# an append to the other cache, behind a bf16 call; in runs, so that several calls may be under way at once
LAYERS = [("4", 0, False), ("4", 0, False), ("4", 1, False), ("4", 0, False), ("4", 2, False), ("4", 0, True), ("4", 1, True),
          ("b", 0, True), ("4", 0, False), ("4", 1, False), ("b", 1, False), ("4", 0, True)]


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("seed", list(range(400, 412)))
def test_chain_of_attention_calls_under_a_pinned_plan(seed, path):
    """With the promise that lets consecutive calls overlap, without it, and with the device idle between any two calls: the same
    bits; and the 4-bit layers match the 64-bit reference on the queries they were given."""
    step, nb = _random_step(seed)
    if step.total_q_rows == 0:
        pytest.skip("all blocks empty")
    s, T = step.shape, step.total_q_rows
    g = torch.Generator().manual_seed(seed)
    q0 = wl.make_q(step).cuda()
    caches = [ref.make_cache(wl.make_kv(step, l), rng_seed=seed) for l in range(2)]
    pools = [torch.from_numpy(c).cuda() for c in caches]
    kv_pool = wl.make_kv(step, 2).cuda()
    k_new, v_new = (torch.randn((T, s.n_kv_heads, s.head_dim), generator=g).bfloat16().cuda() for _ in range(2))
    args = (step, nb, LAYERS, q0, pools, kv_pool, k_new, v_new, step.page_table.cuda())
    with Ctx(step, path) as ctx:
        alone, status = _chain(ctx, *args, wait_between=True)
        assert status == 0
        for l, (fmt, back, _) in enumerate(LAYERS):
            if fmt == "4":
                fed = alone[l - back].cpu() if back else q0.cpu()
                check(alone[l].double().cpu().numpy(), attn_ref(step, fed, caches[l % 2], nb), f"layer {l}")
        for promise in (False, True):
            fd.fd_calls_back_to_back(ctx.h, promise)
            for _ in range(4):
                outs, status = _chain(ctx, *args, wait_between=False)
                assert status == 0
                for l in range(len(LAYERS)):
                    assert torch.equal(_bits(outs[l]), _bits(alone[l])), f"layer {l}, promise {promise}"


@pytest.mark.parametrize("path", PATHS)
def test_chain_with_page_ids_outside_the_pool(path):
    """The sequences that need such a page get zeros in every layer, the others what they get without it."""
    step = wl.make_step("bad", wl.Shape(8, 2, 128, 10), [700, 40, 2000, 300, 9], [8, 16, 9, 1, 30], [4, 0, 3, 0, 16], seed=8)
    nb = torch.ones_like(step.n_mask)
    s, T = step.shape, step.total_q_rows
    g = torch.Generator().manual_seed(8)
    pools = [torch.from_numpy(ref.make_cache(wl.make_kv(step, l))).cuda() for l in range(2)]
    k_new, v_new = (torch.randn((T, s.n_kv_heads, s.head_dim), generator=g).bfloat16().cuda() for _ in range(2))
    layers = [layer for layer in LAYERS if not layer[2]]  # (an append would find the bad ids too)
    args = (step, nb, layers, wl.make_q(step).cuda(), pools, wl.make_kv(step, 2).cuda(), k_new, v_new)
    table = step.page_table.clone()
    table[1, 0], table[2, 100], table[2, 3] = step.num_pages, -1, 2 ** 31 - 1
    row0 = np.concatenate([[0], np.cumsum(step.q_lens.numpy())])
    with Ctx(step, path) as ctx:
        good, status = _chain(ctx, *args, step.page_table.cuda(), wait_between=True)
        assert status == 0
        for promise in (False, True):
            fd.fd_calls_back_to_back(ctx.h, promise)
            for _ in range(3):
                outs, status = _chain(ctx, *args, table.cuda(), wait_between=False)
                assert status == fd.FD_DEV_BAD_PAGE
                for l, out in enumerate(outs):
                    for b in range(step.batch):
                        rows = slice(int(row0[b]), int(row0[b + 1]))
                        assert (out[rows] == 0).all() if b in (1, 2) else torch.equal(_bits(out[rows]), _bits(good[l][rows])), (l, b)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("Hq,Hkv,d,fp4", [(8, 4, 128, True), (8, 4, 64, True), (8, 4, 128, False), (8, 4, 64, False)])
def test_page_ids_outside_the_pool_in_some_of_many_short_sequences(Hq, Hkv, d, fp4, path):
    """Forty pieces of a tile for every CTA, a bad page in some: zeros in exactly those sequences."""
    B = 1600
    step = wl.make_step("many", wl.Shape(Hq, Hkv, d, 10), [(37 * b) % 50 for b in range(B)], [1 + b % 3 for b in range(B)], [0] * B, seed=3)
    T, q, kv = step.total_q_rows, wl.make_q(step).cuda(), wl.make_kv(step)
    cache = torch.from_numpy(ref.make_cache(kv)).cuda() if fp4 else kv.cuda()
    ints = [step.prefix_lens.cuda(), step.q_lens.cuda(), step.n_mask.cuda()]
    good = step.page_table.cuda()
    seq = torch.repeat_interleave(torch.arange(B), step.q_lens).cuda()
    with Ctx(step, path) as ctx:
        def attend(table):
            out = torch.full_like(q, float("nan"))
            if fp4:
                fd.fd_attn_draft_verify_fp4(ctx.h, B, T, q, cache, step.num_pages, table, *ints, None, 1.0, 1.0, out)
            else:
                fd.fd_attn_draft_verify(ctx.h, B, T, q, cache, step.num_pages, table, *ints, out)
            return out, fd.fd_last_device_status(ctx.h)

        want, status = attend(good)
        assert status == 0 and torch.isfinite(want.float()).all()
        for k in range(6):
            bad = torch.rand(B, generator=torch.Generator().manual_seed(k)) < (0.01, 0.3, 0.9)[k % 3]
            table = good.clone()
            table[bad.cuda(), 0] = -5
            out, status = attend(table)
            hit = bad.cuda()[seq]
            assert status == fd.FD_DEV_BAD_PAGE and (out[hit] == 0).all() and torch.equal(_bits(out[~hit]), _bits(want[~hit]))


def test_chain_whose_cache_is_the_output_before():
    """The pages of every second call are the bytes that the call before it writes: nothing of them may be read ahead."""
    step = wl.make_step("alias", wl.Shape(32, 1, 128, 10), [60, 10, 130], [9, 9, 9], [0, 0, 0], seed=12)
    s, T = step.shape, step.total_q_rows
    size = step.num_pages * 2 * ref.page_bytes(128)
    q = wl.make_q(step).cuda()
    assert size <= q.numel() * 2
    pool = torch.from_numpy(ref.make_cache(wl.make_kv(step))).cuda()
    ints = [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda(), step.n_mask.cuda()]
    with Ctx(step, fd.FD_ATTN_TCGEN05_PLANNED, max_q_len=9) as ctx:
        def run(wait):
            outs = [torch.zeros_like(q) for _ in range(8)]
            torch.cuda.synchronize()
            fd.fd_plan_pin(ctx.h, step.batch, T, *ints[1:])
            for l, out in enumerate(outs):
                cache = outs[l - 1].view(torch.uint8).view(-1)[:size] if l % 2 else pool
                fd.fd_attn_draft_verify_fp4(ctx.h, step.batch, T, q, cache, step.num_pages, *ints, None, 1.0, 1.0, out)
                if wait:
                    torch.cuda.synchronize()
            fd.fd_plan_unpin(ctx.h)
            assert fd.fd_last_device_status(ctx.h) == 0
            return outs

        alone = run(True)
        assert any((o[T - 1] != 0).any() for o in alone[1::2])
        fd.fd_calls_back_to_back(ctx.h, True)
        for _ in range(10):
            assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(run(False), alone))


# ---------------------------------------------------------------------------------------------- captured calls
@pytest.mark.parametrize("pin", [False, True])
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("fp4", [True, False])
def test_captured_call_forgets_the_bad_page_of_an_earlier_replay(fp4, path, pin):
    """Two calls in a graph, replayed with page ids outside the pool in some sequences, then in others, then in none: zeros where this
    replay met one, and nowhere else."""
    step = wl.make_step("replay", wl.Shape(8, 2, 128, 10), [700, 40, 2000, 300], [8, 16, 9, 1], [4, 0, 3, 0], seed=9)
    T, q = step.total_q_rows, wl.make_q(step).cuda()
    kv = wl.make_kv(step)
    cache = torch.from_numpy(ref.make_cache(kv)).cuda() if fp4 else kv.cuda()
    good = step.page_table.cuda()
    ints = [good.clone(), step.prefix_lens.cuda(), step.q_lens.cuda(), step.n_mask.cuda()]
    outs = [torch.zeros_like(q) for _ in range(2)]
    row0 = np.concatenate([[0], np.cumsum(step.q_lens.numpy())])
    with Ctx(step, path) as ctx:
        def body():
            if pin:
                fd.fd_plan_pin(ctx.h, step.batch, T, *ints[1:])
            for out in outs:
                if fp4:
                    fd.fd_attn_draft_verify_fp4(ctx.h, step.batch, T, q, cache, step.num_pages, *ints, None, 1.0, 1.0, out)
                else:
                    fd.fd_attn_draft_verify(ctx.h, step.batch, T, q, cache, step.num_pages, *ints, out)
            if pin:
                fd.fd_plan_unpin(ctx.h)

        body()
        torch.cuda.synchronize()
        want = outs[0].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            body()
        for bad in ((1,), (), (0, 2), (3,), (), (1, 2, 3), ()):
            ints[0].copy_(good)
            for b in bad:
                ints[0][b, 1 if b < 3 else 18] = step.num_pages + b
            for out in outs:
                out.fill_(float("nan"))
            graph.replay()
            assert fd.fd_last_device_status(ctx.h) == (fd.FD_DEV_BAD_PAGE if bad else 0)
            for out in outs:
                for b in range(step.batch):
                    rows = slice(int(row0[b]), int(row0[b + 1]))
                    assert (out[rows] == 0).all() if b in bad else torch.equal(_bits(out[rows]), _bits(want[rows])), (bad, b)


# ---------------------------------------------------------------------------------------------- rows that no query owns
@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (40, 8), (48, 8), (8, 8), (16, 8)])
def test_time_and_result_do_not_depend_on_rows_that_no_query_owns(Hq, Hkv):
    """A tile has 128 query rows; one block row of one sequence fills Hq / Hkv of them.  The others hold rows of the sequences behind
    it, or what the call before left in shared memory.  Whatever is in those, the one real row has to come out the same, in the same
    time: a row whose scores keep rising, or are NaN, sends the 32 rows of its warp over the scores of a tile twice."""
    d, G = 128, Hq // Hkv
    step = wl.make_step("rows", wl.Shape(Hq, Hkv, d, 10), [60_000, 0, 0, 0], [1, 1, 1, 1], [0] * 4, seed=5)
    full = 128 // G
    table = torch.cat([step.page_table[:1], torch.full((1, full // 16 + 1), int(step.page_table[0, 0]), dtype=torch.int32)], 1)
    wide = wl.make_step("wide", wl.Shape(Hq, Hkv, d, 10), [60_000 - full], [full], [0], seed=5)
    g = torch.Generator(device="cuda").manual_seed(1)
    pages = torch.randint(0, 256, (step.num_pages, Hkv, 2, ref.page_bytes(d)), generator=g, dtype=torch.uint8, device="cuda")
    pages[..., 16 * d // 2:] = 0x30 + pages[..., 16 * d // 2:] % 8  # (scales from 0.5 to 0.94)
    q = torch.randn((4, Hq, d), generator=g, device="cuda").bfloat16()
    q_wide = torch.randn((full, Hq, d), generator=g, device="cuda").bfloat16()
    ints = [x.cuda() for x in (step.page_table, step.prefix_lens, step.q_lens, step.n_mask)]
    wide_ints = [x.cuda() for x in (table, wide.prefix_lens, wide.q_lens, wide.n_mask)]
    around = {"zeros": lambda t: t.zero_(), "numbers": lambda t: t, "nan": lambda t: t.fill_(float("nan"))}
    times, outs = {kind: [] for kind in around}, {}
    with Ctx(step, fd.FD_ATTN_TCGEN05_PLANNED, max_q_len=full) as ctx, Ctx(wide, fd.FD_ATTN_TCGEN05_PLANNED, max_q_len=full) as before:
        wide_ints[0] = wide_ints[0][:, :wide.max_pages_per_seq].contiguous()
        for k in range(14):
            for kind, fill in around.items():
                x, xw = q.clone(), fill(q_wide.clone())
                fill(x[1:])
                out, out_wide = torch.zeros_like(x), torch.zeros_like(xw)
                fd.fd_attn_draft_verify_fp4(before.h, 1, full, xw, pages, step.num_pages, *wide_ints, None, 1.0, 1.0, out_wide)
                start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                torch.cuda.synchronize()
                start.record()
                fd.fd_attn_draft_verify_fp4(ctx.h, 4, 4, x, pages, step.num_pages, *ints, None, 1.0, 1.0, out)
                end.record()
                torch.cuda.synchronize()
                if k >= 2:
                    times[kind].append(1e3 * start.elapsed_time(end))
                    outs[kind] = out[0].clone()
        assert fd.fd_last_device_status(ctx.h) == 0 and fd.fd_last_device_status(before.h) == 0
    assert torch.isfinite(outs["zeros"].float()).all() and (outs["zeros"] != 0).any()
    assert all(torch.equal(_bits(o), _bits(outs["zeros"])) for o in outs.values())
    us = {kind: float(np.median(t)) for kind, t in times.items()}
    print(f"Hq {Hq} Hkv {Hkv}: us with the other rows", us)
    assert max(us.values()) < 1.1 * us["zeros"], us


# ---------------------------------------------------------------------------------------------- many kv-heads
@pytest.mark.parametrize("Hkv,d,rows", [(545, 128, 40), (546, 128, 1300), (2961, 128, 600), (2961, 128, 3), (4097, 128, 2), (4170, 128, 1),
                                        (1071, 64, 1250), (5883, 64, 600), (8317, 64, 2)])
def test_append_and_read_of_very_long_rows(Hkv, d, rows):
    """A thread finds its row by a product with a reciprocal, exact for so many scale groups only; with more of them a CTA works on
    fewer rows at a time.  The values are multiples of their group's scale, largest 6: held exactly, so what is read back is what was
    appended; and nothing else in the pool changes."""
    step = wl.make_step("long", wl.Shape(Hkv, Hkv, d, 10), [7, 0], [rows - rows // 3, rows // 3], [0, 0], seed=2)
    T = step.total_q_rows
    g = torch.Generator(device="cuda").manual_seed(Hkv)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    def values():
        x = grid[torch.randint(0, 8, (T, Hkv, d), generator=g, device="cuda")] * (1 - 2 * torch.randint(0, 2, (T, Hkv, d), generator=g, device="cuda"))
        x.view(-1, 16)[:, 5] = 6.0
        x.view(-1, 16).mul_(2.0 ** torch.randint(-4, 5, (T * Hkv * d // 16, 1), generator=g, device="cuda"))
        return x.bfloat16()
    k, v = values(), values()
    cache = torch.full((step.num_pages, Hkv, 2, ref.page_bytes(d)), 0xA5, dtype=torch.uint8, device="cuda")
    ints = [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda()]
    ko, vo = (torch.full_like(k, float("nan")) for _ in range(2))
    with Ctx(step, max_q_len=rows) as ctx:
        fd.fd_kv_append_fp4(ctx.h, 2, T, k, v, cache, step.num_pages, *ints)
        fd.fd_kv_read_fp4(ctx.h, 2, T, cache, step.num_pages, *ints, 1.0, 1.0, ko, vo)
        assert fd.fd_last_device_status(ctx.h) == 0
    assert torch.equal(ko, k) and torch.equal(vo, v)
    owned = torch.zeros((step.num_pages, 16), dtype=torch.bool)
    for b, _, j in ref.rows_of(step):
        owned[int(step.page_table[b, j // 16]), j % 16] = True
    free = ~owned.cuda()
    codes = cache[..., :8 * d].view(step.num_pages, Hkv, 2, 16, d // 2).permute(0, 3, 1, 2, 4)
    scales = cache[..., 8 * d:].view(step.num_pages, Hkv, 2, 16, d // 16).permute(0, 3, 1, 2, 4)
    assert (codes[free] == 0xA5).all() and (scales[free] == 0xA5).all()
