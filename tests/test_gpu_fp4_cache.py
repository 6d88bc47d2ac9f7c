"""GPU tests of the 4-bit cache: rows of a tile that no query owns, head counts far above the usual ones."""
import numpy as np
import pytest
import torch

import fp4_ref as ref
import paper_2605_20022_b200 as fd
from helpers import Ctx
from paper_2605_20022_b200 import workload as wl

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.view(torch.int16)


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
