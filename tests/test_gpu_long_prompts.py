"""GPU tests of prompts longer than a context's max_q_len: the calls on their way from the projection to the cache."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_20022_b200 as fd
from paper_2605_20022_b200 import workload as wl

pytestmark = pytest.mark.gpu

I32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731


@pytest.mark.parametrize("max_q_len,longest", [(1, 2), (5, 6), (5, 9), (30, 31), (300, 1001)])
def test_append_of_blocks_longer_than_max_q_len(max_q_len, longest):
    """fd_kv_append leaves such a sequence out and says so, and writes the others: the oracle's bytes, all of the pool.  In pieces it
    takes the rows that it has left out."""
    lens = [longest, 1, 0, max_q_len, longest + 7]
    step = wl.make_step("long", wl.Shape(2, 2, 64, 10), [5, 0, 100, 40, 16], lens, [0] * 5, seed=3)
    T, kv = step.total_q_rows, wl.make_kv(step)
    k, v = (torch.randn((T, 2, 64), generator=torch.Generator().manual_seed(i)).bfloat16() for i in (1, 2))
    want = oracle.kv_append(k, v, kv, step.page_table, step.prefix_lens, step.q_lens)
    short = want.copy()
    for b in (0, 4):
        n = int(step.prefix_lens[b])
        for j in range(n, n + lens[b]):
            page = int(step.page_table[b, j // 16])
            short[page, :, :, j % 16] = kv.view(torch.int16).numpy().view(np.uint16)[page, :, :, j % 16]
    ctx = fd.fd_create(2, 2, 64, 10, 5, max_q_len, step.max_pages_per_seq)
    bits = lambda x: x.cpu().view(torch.int16).numpy().view(np.uint16)  # noqa: E731
    try:
        dev, table = kv.cuda(), step.page_table.cuda()
        fd.fd_kv_append(ctx, 5, T, k.cuda(), v.cuda(), dev, step.num_pages, table, step.prefix_lens.cuda(), step.q_lens.cuda())
        assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_LENGTHS
        np.testing.assert_array_equal(bits(dev), short)
        row = 0
        for b, n_rows in enumerate(lens):
            for at in range(0, n_rows if n_rows > max_q_len else 0, max_q_len):
                some = slice(row + at, row + min(at + max_q_len, n_rows))
                fd.fd_kv_append(ctx, 1, some.stop - some.start, k[some].cuda(), v[some].cuda(), dev, step.num_pages, table[b:b + 1].contiguous(),
                                I32([int(step.prefix_lens[b]) + at]), I32([some.stop - some.start]))
            row += n_rows
        assert fd.fd_last_device_status(ctx) == 0
        np.testing.assert_array_equal(bits(dev), want)
    finally:
        fd.fd_destroy(ctx)
