"""GPU tests of the 4-bit cache: head counts far above the usual ones."""
import pytest
import torch

import fp4_ref as ref
import paper_2605_20022_b200 as fd
from helpers import Ctx
from paper_2605_20022_b200 import workload as wl

pytestmark = pytest.mark.gpu


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
