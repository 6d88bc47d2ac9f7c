"""GPU tests of prompts longer than a context's max_q_len: the calls on their way from the projection to the cache."""
import numpy as np
import pytest
import torch

import fp8_ref as ref
import oracle
import paper_2605_20022_b200 as fd
from fp4_ref import rows_of
from paper_2605_20022_b200 import workload as wl
from test_gpu_fp8_cache import attn_ref
from test_gpu_prompt import _check as check_prompt
from test_gpu_serving import check

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


@pytest.mark.parametrize("Hq,Hkv,d,prompts,max_q_len", [(8, 2, 128, [1500, 5, 2600, 33], 8), (16, 2, 64, [40, 4500], 32)])
def test_prompts_longer_than_max_q_len_into_the_8_bit_cache(Hq, Hkv, d, prompts, max_q_len):
    """reserve -> norm and rotation to rows -> prompt attention -> append -> commit, in a context made for short blocks; then a decode
    step over what is held.  Rows and cache against the definitions."""
    B, T = len(prompts), sum(prompts)
    width = -(-(max(prompts) + max_q_len) // 16)
    pool = sum(-(-(n + max_q_len) // 16) for n in prompts) + 3
    g = torch.Generator().manual_seed(d)
    bf = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    qkv, w = bf(T, (Hq + 2 * Hkv) * d), torch.ones(d, dtype=torch.bfloat16, device="cuda")
    angle = np.arange(max(prompts))[:, None] * 100.0 ** (-np.arange(d // 2) * 2.0 / d)[None]
    cos_sin = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda()
    cap = -(-T // 16)
    q, rows, out = z(T, Hq, d), z(2, cap * 16, Hkv, d), z(T, Hq, d)
    table, prefix, lens, none = I32(np.full((B, width), -1)), I32([0] * B), I32(prompts), I32([0] * B)
    free, n, slots, pos = I32(np.random.default_rng(d).permutation(pool)), I32([pool]), I32([0] * T), I32([0] * T)
    freed, n_freed = I32([-1] * (pool + B)), I32([7])
    cache = torch.randint(0, 256, (pool, Hkv, 2, ref.block_bytes(d)), generator=g, dtype=torch.uint8).cuda()
    before = cache.cpu().numpy()
    ctx = fd.fd_create(Hq, Hkv, d, 10, B, max_q_len, width)
    try:
        fd.fd_kv_reserve(ctx, B, T, table, prefix, lens, none, None, None, None, free, n, n, pool, slots, pos)
        assert fd.fd_last_device_status(ctx) == 0
        assert pos.tolist() == [j for L in prompts for j in range(L)] and int(n) == pool - sum(-(-L // 16) for L in prompts)
        assert slots.tolist() == [int(table[b, j // 16]) * 16 + j % 16 for b, L in enumerate(prompts) for j in range(L)]
        fd.fd_qk_norm_rope_append(ctx, T, qkv, qkv.stride(0), w, w, 1e-6, cos_sin, cos_sin.shape[0], d, fd.FD_ROPE_HALVES, pos, I32(np.arange(T)), q, rows,
                                  cap, fd.FD_KV_ROWS)
        k, v = rows[0, :T], rows[1, :T]
        fd.fd_attn_prompt(ctx, B, T, T, q, Hq * d, k, v, Hkv * d, lens, None, out)
        fd.fd_kv_append_fp8(ctx, B, T, k, v, cache, pool, table, prefix, lens)
        step = wl.Step("prompts", wl.Shape(Hq, Hkv, d, 10), 0, 0.0, prefix.cpu(), lens.cpu(), none.cpu(), table.cpu(), pool)
        fd.fd_kv_commit(ctx, B, table, prefix, lens, I32([L - 1 for L in prompts]), freed, n_freed)
        assert fd.fd_last_device_status(ctx) == 0 and prefix.tolist() == prompts and int(n_freed) == 0
        assert torch.equal(v, qkv.view(T, Hq + 2 * Hkv, d)[:, Hq + Hkv:])
        check_prompt(out, q, k, v, prompts, prompts, "prompt")
        want = ref.values(*ref.split(ref.append(before, d, step, k.cpu(), v.cpu()), d))
        held = ref.values(*ref.split(cache.cpu().numpy(), d))
        at = [(int(step.page_table[b, j // 16]), j % 16) for b, _, j in rows_of(step)]
        page, tok = (np.array(x) for x in zip(*at))
        np.testing.assert_array_equal(held[page, :, :, tok], want[page, :, :, tok])
        # a step of all of them
        T2 = B * max_q_len
        q2, k2, v2, out2, lens2 = bf(T2, Hq, d), bf(T2, Hkv, d), bf(T2, Hkv, d), z(T2, Hq, d), I32([max_q_len] * B)
        fd.fd_kv_reserve(ctx, B, T2, table, prefix, lens2, none, None, freed, n_freed, free, n, n, pool, slots, pos)
        fd.fd_kv_append_fp8(ctx, B, T2, k2, v2, cache, pool, table, prefix, lens2)
        fd.fd_attn_draft_verify_fp8(ctx, B, T2, q2, cache, pool, table, prefix, lens2, none, None, out2)
        assert fd.fd_last_device_status(ctx) == 0
        step = wl.Step("step", step.shape, 0, 0.0, prefix.cpu(), lens2.cpu(), none.cpu(), table.cpu(), pool)
        check(out2.double().cpu().numpy(), attn_ref(step, q2.cpu(), cache.cpu().numpy()), "decode")
    finally:
        fd.fd_destroy(ctx)


def test_long_blocks_that_are_still_refused():
    """A block with mask tokens beyond max_q_len; rows beyond max_batch * max_q_len into pages."""
    ctx = fd.fd_create(4, 1, 64, 10, 2, 32, 8)
    try:
        table, free, n, slots, pos = I32(np.full((2, 8), -1)), I32(range(20)), I32([20]), I32([9] * 50), I32([9] * 50)
        call = lambda lens, masks: fd.fd_kv_reserve(ctx, 2, 50, table, I32([0, 0]), I32(lens), I32(masks), None, None, None, free, n, n, 20, slots, pos)  # noqa: E731
        call([40, 10], [3, 3])
        assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_LENGTHS and (slots == -1).all() and (table == -1).all() and int(n) == 20
        call([40, 10], [0, 3])
        assert fd.fd_last_device_status(ctx) == 0 and int(n) == 16
        q, kv = torch.zeros((65, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 80, 1, 64), dtype=torch.bfloat16, device="cuda")
        qkv, slot = torch.zeros((65, 6 * 64), dtype=torch.bfloat16, device="cuda"), I32(range(65))
        rope = lambda T, fmt: fd.fd_qk_norm_rope_append(ctx, T, qkv, 384, None, None, 1e-6, None, 0, 0, fd.FD_ROPE_HALVES, None, slot, q, kv, 5, fmt, 1.0, 1.0,  # noqa: E731
                                                        raise_on_error=False)
        assert rope(65, fd.FD_KV_BF16) == rope(65, fd.FD_KV_FP4) == fd.FD_ERR_INVALID_ARG
        assert rope(65, fd.FD_KV_ROWS) == rope(64, fd.FD_KV_BF16) == fd.FD_OK and fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)
