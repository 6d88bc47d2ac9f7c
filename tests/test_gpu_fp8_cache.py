"""GPU tests of the 8-bit cache: append and read byte for byte against the 64-bit reference, attention against the oracle.

Attention tolerance: as for the 4-bit cache (test_gpu_serving.py).  The values of the cache enter exactly, and the queries but for
elements below 2^-9 of their row's largest, which are off by at most 2^-17 of it (here less than 2^-12 of a weight); the softmax weights are held in at least 11 bits (relative 2^-11) before the product with V, exponentials and fp32 sums add relative
2^-14, the output is rounded to bf16 (2^-8, half a step), and weights below fp16's steps are off by at most 2^-32 of the row's
largest: |err| <= 2^-8 |ref| + 2^-10 sum_j p_j |v_j| + 2^-32 keys max |v|."""
import zlib

import numpy as np
import pytest
import torch

import fp8_ref as ref
import oracle
import paper_2605_20022_b200 as fd
from fp4_ref import rows_of
from helpers import Ctx
from paper_2605_20022_b200 import workload as wl
from test_gpu_parity import BLOCK_CASES, EDGE, PATHS, _random_step
from test_gpu_serving import ROWS, check

pytestmark = pytest.mark.gpu


def attn_ref(step, q, cache, n_blocks=None, scale=None):
    """(reference, tolerance) of the attention over an 8-bit cache."""
    d = step.shape.head_dim
    kv = ref.as_bf16_cache(cache, d)
    nb = torch.ones_like(step.n_mask) if n_blocks is None else n_blocks
    args = (step.page_table, step.prefix_lens, step.q_lens, step.n_mask, nb)
    scale = scale or 1 / np.sqrt(d)
    out = oracle.attn_blocks(q, kv, *args, scale=scale)
    kv[:, 1] = kv[:, 1].abs()
    size = oracle.attn_blocks(q, kv, *args, scale=scale)
    owned = torch.zeros((kv.shape[0], 16), dtype=torch.bool)
    for b in range(step.batch):
        for j in range(int(step.kv_lens[b])):
            owned[int(step.page_table[b, j // 16]), j % 16] = True
    largest = float(kv[:, 1].transpose(1, 2)[owned].double().max()) if owned.any() else 0.0
    return out, 2.0 ** -8 * np.abs(out) + 2.0 ** -10 * size + 2.0 ** -32 * int(step.kv_lens.max()) * largest


def attn_gpu(ctx, step, q, cache, n_blocks=None, lens=None, page_table=None):
    pl, ql, nm = lens if lens is not None else (step.prefix_lens, step.q_lens, step.n_mask)
    pt = step.page_table if page_table is None else page_table
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    c = torch.from_numpy(cache).cuda() if isinstance(cache, np.ndarray) else cache
    fd.fd_attn_draft_verify_fp8(ctx.h, step.batch, step.total_q_rows, q.cuda(), c, step.num_pages, pt.cuda(), pl.cuda(), ql.cuda(),
                                nm.cuda(), None if n_blocks is None else n_blocks.cuda(), out)
    return out.double().cpu().numpy(), fd.fd_last_device_status(ctx.h)


# ---------------------------------------------------------------------------------------------- append and read
def _rows(T, Hkv, d, seed):
    """Rows over many magnitudes, ties of the codes, zeros, infinities, NaN, the largest and smallest numbers."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, Hkv, d), generator=g) * 2.0 ** torch.randint(-12, 8, (T, Hkv, 1), generator=g)
    flat = x.view(T * Hkv, d)
    flat[::5, :8] = torch.tensor([448.0, 464.0, 17.0, 19.0, -1.0625, 0.0, -0.0, 2.0 ** -9])
    for k, v in enumerate((float("inf"), float("nan"), 3.0e38, 1e-38, -float("inf"), 57344.0, 60000.0)):
        if T * Hkv > 3 + 11 * k:
            flat[3 + 11 * k, k + 9] = v
    return x.bfloat16()


def _pool(step, Hkv, d, seed):
    """A pool whose blocks hold codes and scales of every kind, and whose other bytes are random."""
    r = np.random.default_rng(seed)
    codes = r.integers(0, 256, (step.num_pages, Hkv, 2, 16, d)).astype(np.uint8)
    return ref.join(codes, r.choice(ref.POWERS, (step.num_pages, Hkv, 2)))


@pytest.mark.parametrize("name", sorted(ROWS))
def test_append_and_read_match_the_definition(name):
    """Every byte of the pool, untouched ones included (a NaN's sign aside); then the rows back out of it, exactly."""
    Hkv, d, pl, ql = ROWS[name]
    step = wl.make_step(name, wl.Shape(Hkv, Hkv, d, 10), pl, ql, [0] * len(pl), seed=3, extra_table_cols=1)
    T = step.total_q_rows
    k, v, cache = _rows(T, Hkv, d, 5), _rows(T, Hkv, d, 6), _pool(step, Hkv, d, 7)
    want = ref.append(cache, d, step, k, v)
    with Ctx(step, max_q_len=max(ql)) as ctx:
        dev = torch.from_numpy(cache).cuda()
        tail = [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda()]
        for _ in range(2):  # (a second time: the same)
            fd.fd_kv_append_fp8(ctx.h, step.batch, T, k.cuda(), v.cuda(), dev, step.num_pages, *tail)
            assert fd.fd_last_device_status(ctx.h) == 0
            got = dev.cpu().numpy()
            nan = (got[..., :16 * d] & 127 == 127) & (want[..., :16 * d] & 127 == 127)
            np.testing.assert_array_equal(np.where(nan, 127, got[..., :16 * d]), np.where(nan, 127, want[..., :16 * d]))
            np.testing.assert_array_equal(got[..., 16 * d:], want[..., 16 * d:])
        ko, vo = (torch.full((T + 1, Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        fd.fd_kv_read_fp8(ctx.h, step.batch, T, dev, step.num_pages, *tail, ko, vo)
        assert fd.fd_last_device_status(ctx.h) == 0
        assert (ko[T] == 7).all() and (vo[T] == 7).all()
    held = ref.values(*ref.split(want, d))
    for got, which in ((ko, 0), (vo, 1)):
        exp = np.stack([held[int(step.page_table[b, j // 16]), :, which, j % 16] for b, _, j in rows_of(step)])
        np.testing.assert_array_equal(got[:T].double().cpu().numpy(), exp)


def test_tokens_join_a_block_one_by_one():
    """Louder and quieter tokens in turn: values above the subnormals of the loudest stay what they were when they came; a rejected
    loud one (rolled back, overwritten) gives its range back."""
    d, Hkv = 64, 2
    step = wl.make_step("join", wl.Shape(Hkv, Hkv, d, 10), [0], [40], [0], seed=1)
    cache = np.random.default_rng(3).integers(0, 256, (step.num_pages, Hkv, 2, ref.block_bytes(d)), dtype=np.uint8)
    dev = torch.from_numpy(cache).cuda()
    g = torch.Generator().manual_seed(2)
    n = 0
    with Ctx(step, max_q_len=40) as ctx:
        for count, loud in ((1, 1.0), (1, 64.0), (2, 0.01), (5, 2000.0), (1, 1.0), (9, 1.0), (17, 30.0)):
            k, v = (torch.randn((count, Hkv, d), generator=g).mul(loud).bfloat16() for _ in range(2))
            here = wl.Step("join", step.shape, 0, 0.0, torch.tensor([n], dtype=torch.int32), torch.tensor([count], dtype=torch.int32),
                           torch.zeros(1, dtype=torch.int32), step.page_table, step.num_pages)
            cache = ref.append(cache, d, here, k, v)
            fd.fd_kv_append_fp8(ctx.h, 1, count, k.cuda(), v.cuda(), dev, step.num_pages, step.page_table.cuda(), here.prefix_lens.cuda(), here.q_lens.cuda())
            np.testing.assert_array_equal(dev.cpu().numpy(), cache)
            n += count if loud != 2000.0 else 0
        assert fd.fd_last_device_status(ctx.h) == 0


def test_append_and_read_errors():
    step = wl.make_step("err", wl.Shape(2, 2, 64, 10), [10, 20, 40], [8, 8, 8], [0, 0, 0], seed=4)
    k = torch.randn((24, 2, 64)).bfloat16()
    cache = _pool(step, 2, 64, 1)
    table, pl, ql = step.page_table, step.prefix_lens, step.q_lens
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    with Ctx(step) as ctx:
        def both(total=24, table=table, pl=pl, ql=ql, clean=()):
            """What is written and read, and that everything of the sequences in `clean` is as it would be."""
            dev = torch.from_numpy(cache).cuda()
            ko, vo = (torch.full((24, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            ints = [table.cuda(), pl.cuda(), ql.cuda()]
            fd.fd_kv_append_fp8(ctx.h, 3, total, k.cuda(), k.cuda(), dev, step.num_pages, *ints)
            one = fd.fd_last_device_status(ctx.h)
            fd.fd_kv_read_fp8(ctx.h, 3, total, dev, step.num_pages, *ints, ko, vo)
            two = fd.fd_last_device_status(ctx.h)
            assert one == two
            want = ref.append(cache, 64, step, k, k, skip=set(range(3)) - set(clean))
            np.testing.assert_array_equal(dev.cpu().numpy(), want)
            return one, ko.float().cpu(), vo.float().cpu()

        for page in (step.num_pages, -1, 2 ** 31 - 1, -2 ** 31):
            bad = table.clone()
            bad[1, 1] = page                                   # positions 16..31 of sequence 1: all of its rows
            status, ko, vo = both(table=bad, clean=(0, 2))
            assert status == fd.FD_DEV_BAD_PAGE and (ko[8:16] == 0).all() and (vo[8:16] == 0).all() and (ko[:8] != 0).any()
        for lens in ((i32(10, -1, 40), ql), (i32(10, 10 ** 6, 40), ql), (i32(10, 2 ** 31 - 1, 40), ql)):
            status, ko, _ = both(pl=lens[0], ql=lens[1], clean=(0, 2))
            assert status == fd.FD_DEV_BAD_LENGTHS and (ko[8:16] == 0).all() and (ko[16:] != 0).any()
        status, ko, _ = both(total=20, clean=(0, 1))           # the last sequence's rows pass the call's
        assert status == fd.FD_DEV_BAD_LENGTHS and (ko[16:20] == 0).all() and (ko[20:] == 7).all()
        n, c, dk = fd.fd_launch_count(ctx.h), torch.from_numpy(cache).cuda(), k.cuda()
        ints = [table.cuda(), pl.cuda(), ql.cuda()]
        for args in ([3, 24, None, dk, c, step.num_pages, *ints], [3, 24, dk, dk, None, step.num_pages, *ints], [4, 24, dk, dk, c, step.num_pages, *ints],
                     [3, -1, dk, dk, c, step.num_pages, *ints], [3, 24, dk, dk, c, -1, *ints], [3, 24, dk, dk.data_ptr() + 2, c, step.num_pages, *ints],
                     [3, 24, dk, dk, c.data_ptr() + 8, step.num_pages, *ints], [3, 24, dk, dk, c, step.num_pages, None, ints[1], ints[2]],
                     [0, 24, dk, dk, c, step.num_pages, *ints]):
            assert fd.fd_kv_append_fp8(ctx.h, *args, raise_on_error=False) == fd.FD_ERR_INVALID_ARG
            B, T, a, b, cc, pages, *i = args
            assert fd.fd_kv_read_fp8(ctx.h, B, T, cc, pages, *i, a, b, raise_on_error=False) == fd.FD_ERR_INVALID_ARG
        assert fd.fd_launch_count(ctx.h) == n
        assert fd.fd_kv_append_fp8(ctx.h, 0, 0, None, None, None, 0, None, None, None) == fd.FD_OK


# ---------------------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("name", sorted(EDGE))
def test_attention_edge_cases(name, path):
    Hq, Hkv, d, pl, ql, nm = EDGE[name]
    step = wl.make_step(name, wl.Shape(Hq, Hkv, d, 1000), pl, ql, nm, seed=zlib.crc32(name.encode()) % 10000, extra_table_cols=2)
    q, cache = wl.make_q(step), ref.make_cache(wl.make_kv(step), rng_seed=9)
    with Ctx(step, path, max_batch=len(pl)) as ctx:
        got, status = attn_gpu(ctx, step, q, cache)
        again, _ = attn_gpu(ctx, step, q, cache)
    assert status == 0
    check(got, attn_ref(step, q, cache), name)
    assert np.array_equal(got, again), "two runs on the same inputs differ bitwise"


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("name", sorted(BLOCK_CASES))
def test_attention_mask_blocks(name, path):
    Hq, Hkv, d, pl, C, M, nb = BLOCK_CASES[name]
    step = wl.make_step(name, wl.Shape(Hq, Hkv, d, 1000), pl, [c + m for c, m in zip(C, M)], M, seed=zlib.crc32(name.encode()) % 10000)
    q, cache = wl.make_q(step), ref.make_cache(wl.make_kv(step), rng_seed=10)
    n_blocks = torch.tensor(nb, dtype=torch.int32)
    with Ctx(step, path, max_q_len=max(int(step.q_lens.max()), 1)) as ctx:
        got, status = attn_gpu(ctx, step, q, cache, n_blocks)
        assert status == 0
        check(got, attn_ref(step, q, cache, n_blocks), name)


@pytest.mark.parametrize("seed", list(range(500, 520)))
def test_attention_random_shapes(seed):
    step, n_blocks = _random_step(seed)
    if step.total_q_rows == 0:
        pytest.skip("all blocks empty")
    q, cache = wl.make_q(step), ref.make_cache(wl.make_kv(step), rng_seed=seed)
    want = attn_ref(step, q, cache, n_blocks)
    for path in PATHS:
        with Ctx(step, path) as ctx:
            got, status = attn_gpu(ctx, step, q, cache, n_blocks)
        assert status == 0
        check(got, want, f"{step.name} path {path}")


@pytest.mark.parametrize("Hq,Hkv,d,batch,longest", [(32, 8, 128, 330, 120), (16, 2, 64, 700, 100)])
def test_attention_many_short_sequences(Hq, Hkv, d, batch, longest):
    """A CTA works through a dozen segments of one to three tiles: the roles run pieces ahead of one another."""
    rng = np.random.default_rng(batch)
    pl = rng.integers(0, longest + 1, batch)
    nm = rng.integers(0, 3, batch) * (rng.random(batch) < 0.5)
    ql = rng.integers(0, 6, batch) + nm + (rng.random(batch) < 0.9)
    step = wl.make_step("short sequences", wl.Shape(Hq, Hkv, d, 1000), pl.tolist(), ql.tolist(), nm.tolist(), seed=batch)
    q, cache = wl.make_q(step), ref.make_cache(wl.make_kv(step), rng_seed=batch)
    with Ctx(step, 0, max_batch=batch) as ctx:
        first, status = attn_gpu(ctx, step, q, cache)
        assert status == 0
        check(first, attn_ref(step, q, cache), "short sequences")
        c = torch.from_numpy(cache).cuda()
        for _ in range(60):
            got, status = attn_gpu(ctx, step, q, c)
            assert status == 0 and np.array_equal(got, first), "two runs on the same inputs differ bitwise"


@pytest.mark.parametrize("path", PATHS)
def test_attention_every_scale_of_a_block(path):
    """Blocks of every power from 2^-15 to 2^7 side by side, every code but NaN: values from 2^-24 to 57344 in one cache."""
    step = wl.make_step("bytes", wl.Shape(8, 2, 64, 1000), [500, 33], [9, 32], [4, 16], seed=13)
    r = np.random.default_rng(2)
    codes = r.integers(0, 256, (step.num_pages, 2, 2, 16, 64)).astype(np.uint8)
    codes[codes & 127 == 127] = 0
    scales = r.choice(ref.POWERS, (step.num_pages, 2, 2))
    scales[:, :, 0] = r.choice(ref.POWERS[4:9], (step.num_pages, 2))  # keys: small enough for scores that are not one-hot
    cache = ref.join(codes, scales)
    q = wl.make_q(step)
    with Ctx(step, path) as ctx:
        got, status = attn_gpu(ctx, step, q, cache)
    assert status == 0
    check(got, attn_ref(step, q, cache), "bytes")


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("Hq,Hkv,d,by", [(32, 8, 128, 4.0), (16, 2, 64, 12.0)])
def test_attention_scores_that_rise_and_fall_along_the_sequence(Hq, Hkv, d, by, path):
    pl, ql, nm = [5000, 2100, 700, 90, 1], [32, 17, 32, 5, 1], [16, 0, 16, 0, 0]
    step = wl.make_step("drift", wl.Shape(Hq, Hkv, d, 1000), pl, ql, nm, seed=int(by) + d)
    kv = wl.make_kv(step)
    for b in range(len(pl)):
        for page in range(-(-(pl[b] + ql[b]) // 16)):
            kv[step.page_table[b, page], 0] += by * (page // 8)
    q, cache = wl.make_q(step), ref.make_cache(kv, rng_seed=5)
    with Ctx(step, path, max_q_len=32) as ctx:
        got, status = attn_gpu(ctx, step, q, cache)
        assert status == 0
        check(got, attn_ref(step, q, cache), "drift")
        for _ in range(10):
            again, _ = attn_gpu(ctx, step, q, cache)
            assert np.array_equal(got, again), "two runs on the same inputs differ bitwise"


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("size,scale", [(3.0e5, 1e-7), (1e-6, 1e4), (8.0, 0.0), (1e30, 1e-32)])
def test_attention_queries_of_any_size(path, size, scale):
    """Queries far outside and far inside an 8-bit type's range: rows of one call differ by factors of a thousand, elements within a row by
    a hundred."""
    step = wl.make_step("sizes", wl.Shape(8, 2, 128, 1000), [300, 40, 1000], [12, 32, 5], [4, 16, 0], seed=12)
    g = torch.Generator().manual_seed(1)
    q = wl.make_q(step).float() * 10.0 ** torch.randint(-1, 2, (1, 1, 128), generator=g)
    q = q * size
    q[3] *= 1e-3
    q[7, 2] = 0.0
    q = q.bfloat16()
    cache = ref.make_cache(wl.make_kv(step))
    with Ctx(step, path, scale=scale) as ctx:
        got, status = attn_gpu(ctx, step, q, cache)
    assert status == 0
    check(got, attn_ref(step, q, cache, scale=scale or None), "sizes")


def _quick_cache(kv):
    """ref.make_cache of large caches: the same bytes, by torch's conversion."""
    x = kv.cuda().float().permute(0, 2, 1, 3, 4)
    live = (x.abs() < 1e20).all(-1, keepdim=True)
    x = torch.where(live, x, 0.0)
    amax = x.abs().amax((-1, -2))
    m, e = torch.frexp(amax / 448)
    e = torch.where(amax > 0, e - (m == 0.5).int(), -15).clamp(-15, 7)
    power = lambda n: ((n + 127) << 23).int().view(torch.float32)  # noqa: E731
    codes = (x * power(-e)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    scale = power(e)[..., None]
    tail = torch.cat([scale, torch.zeros(scale.shape[:-1] + (3,), device="cuda")], -1).view(torch.uint8)
    return torch.cat([codes.flatten(-2), tail], -1)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (8, 4, 64)])
@pytest.mark.parametrize("pl,ql", [([300, 40], [12, 32]), ([40000], [8]), ([5000] * 40, [6] * 40)])
def test_attention_queries_that_are_not_finite(pl, ql, Hq, Hkv, d, path):
    """A query that is NaN or infinite makes its own row NaN, in sequences that one CTA works on and in those that several share."""
    step = wl.make_step("not finite", wl.Shape(Hq, Hkv, d, 1000), pl, ql, [2] * len(pl), seed=12)
    q, kv = wl.make_q(step), wl.make_kv(step)
    cache = _quick_cache(kv)
    if len(pl) == 2:
        assert torch.equal(cache, torch.from_numpy(ref.make_cache(kv)).cuda())
    gone = torch.zeros(q.shape[:2], dtype=torch.bool)
    gone[3, 1] = gone[5, 2] = gone[7, 0] = True
    with Ctx(step, path) as ctx:
        clean, _ = attn_gpu(ctx, step, q, cache)
        q[3, 1, 7], q[5, 2], q[7, 0, 3] = float("nan"), float("nan"), -float("inf")
        got, status = attn_gpu(ctx, step, q, cache)
    assert status == 0 and np.isnan(got[gone.numpy()]).all()
    np.testing.assert_array_equal(got[~gone.numpy()], clean[~gone.numpy()])


@pytest.mark.parametrize("pin", [False, True])
@pytest.mark.parametrize("path", PATHS)
def test_captured_call_forgets_the_bad_page_of_an_earlier_replay(path, pin):
    """A page id outside the pool zeroes its sequence in that replay and in no other."""
    step = wl.make_step("replay", wl.Shape(8, 2, 128, 1000), [300, 700, 40], [8, 8, 8], [4, 4, 4], seed=8)
    q, cache = wl.make_q(step).cuda(), ref.make_cache(wl.make_kv(step))
    c, table = torch.from_numpy(cache).cuda(), step.page_table.cuda()
    ints, nm, out = [table, step.prefix_lens.cuda(), step.q_lens.cuda()], step.n_mask.cuda(), torch.zeros_like(q)
    with Ctx(step, path) as ctx:
        call = lambda: fd.fd_attn_draft_verify_fp8(ctx.h, 3, 24, q, c, step.num_pages, *ints, nm, None, out)  # noqa: E731
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            if pin:
                fd.fd_plan_pin(ctx.h, 3, 24, ints[1], ints[2], nm)
            call()
        for bad in (False, True, False, True, False):
            table.copy_(step.page_table)
            if bad:
                table[1, 20] = step.num_pages
            graph.replay()
            torch.cuda.synchronize()
            got = out.double().cpu().numpy()
            assert fd.fd_last_device_status(ctx.h) == (fd.FD_DEV_BAD_PAGE if bad else 0)
            exp, tol = attn_ref(step, q.cpu(), cache)
            if bad:
                assert (got[8:16] == 0).all()
                got, exp, tol = np.delete(got, range(8, 16), 0), np.delete(exp, range(8, 16), 0), np.delete(tol, range(8, 16), 0)
            check(got, (exp, tol), "replay")
        if pin:
            fd.fd_plan_unpin(ctx.h)


def test_norm_rope_into_rows():
    """FD_KV_ROWS: the bytes that FD_KV_BF16 puts into pages, as rows; padding and slots beyond the rows; the 8-bit format is refused."""
    Hq, Hkv, d, T, pages = 8, 2, 128, 37, 4
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((T, (Hq + 2 * Hkv) * d), generator=g).bfloat16().cuda()
    w = (1 + 0.1 * torch.randn(d, generator=g)).bfloat16().cuda()
    cos_sin = torch.randn((64, d), generator=g).cuda()
    pos = torch.randint(0, 64, (T,), generator=g).int().cuda()
    slot = torch.randperm(pages * 16, generator=g)[:T].int()
    slot[5] = -1
    ctx = fd.fd_create(Hq, Hkv, d, 10, 1, 64, 8)
    try:
        for style, rot in ((fd.FD_ROPE_HALVES, d), (fd.FD_ROPE_ADJACENT, d), (fd.FD_ROPE_HALVES, 64), (fd.FD_ROPE_HALVES, 0)):
            q1, q2 = (torch.zeros((T, Hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            paged, rows = torch.zeros((pages, 2, Hkv, 16, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, pages * 16, Hkv, d), dtype=torch.bfloat16, device="cuda")
            args = [ctx, T, qkv, qkv.stride(0), w, w, 1e-6, cos_sin[:, :max(rot, 1)].contiguous(), 64, rot, style, pos, slot.cuda()]
            fd.fd_qk_norm_rope_append(*args, q1, paged, pages, fd.FD_KV_BF16)
            fd.fd_qk_norm_rope_append(*args, q2, rows, pages, fd.FD_KV_ROWS)
            assert fd.fd_last_device_status(ctx) == 0
            assert torch.equal(q1, q2) and torch.equal(paged.permute(1, 0, 3, 2, 4).reshape(2, pages * 16, Hkv, d), rows) and (rows != 0).any()
        beyond = slot.clone()
        beyond[7] = pages * 16
        fd.fd_qk_norm_rope_append(*args[:-1], beyond.cuda(), q2, rows, pages, fd.FD_KV_ROWS)
        assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_PAGE
        for fmt in (fd.FD_KV_FP8, 4, -1):
            assert fd.fd_qk_norm_rope_append(*args, q2, rows, pages, fmt, raise_on_error=False) == fd.FD_ERR_INVALID_ARG
    finally:
        fd.fd_destroy(ctx)


@pytest.mark.parametrize("Hkv,d,rows", [(546, 128, 300), (2961, 64, 40), (4097, 128, 2)])
def test_append_and_read_of_very_long_rows(Hkv, d, rows):
    step = wl.make_step("long rows", wl.Shape(Hkv, Hkv, d, 10), [5], [rows], [0], seed=2)
    k, v = (torch.randn((rows, Hkv, d), generator=torch.Generator().manual_seed(i)).bfloat16() for i in (1, 2))
    cache = _pool(step, Hkv, d, 3)
    with Ctx(step, max_q_len=rows) as ctx:
        dev, tail = torch.from_numpy(cache).cuda(), [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda()]
        fd.fd_kv_append_fp8(ctx.h, 1, rows, k.cuda(), v.cuda(), dev, step.num_pages, *tail)
        ko, vo = torch.full_like(k, float("nan")).cuda(), torch.full_like(v, float("nan")).cuda()
        fd.fd_kv_read_fp8(ctx.h, 1, rows, dev, step.num_pages, *tail, ko, vo)
        assert fd.fd_last_device_status(ctx.h) == 0
    # the prefix's rows are the pool's, of any scale, and set the first block's: what is held is the definition's, exactly
    held = ref.values(*ref.split(ref.append(cache, d, step, k, v), d))
    for got, which in ((ko, 0), (vo, 1)):
        exp = np.stack([held[int(step.page_table[b, j // 16]), :, which, j % 16] for b, _, j in rows_of(step)])
        np.testing.assert_array_equal(got.double().cpu().numpy(), exp)


@pytest.mark.parametrize("path", PATHS)
def test_attention_device_detected_errors(path):
    step = wl.make_step("err", wl.Shape(8, 2, 128, 1000), [100, 200, 50], [8, 8, 8], [4, 4, 4], seed=6)
    q, cache = wl.make_q(step), ref.make_cache(wl.make_kv(step))
    exp, tol = attn_ref(step, q, cache)
    with Ctx(step, path) as ctx:
        for page in (step.num_pages, -1, 2 ** 31 - 1, -2 ** 31):
            bad = step.page_table.clone()
            bad[1, 3] = page
            got, status = attn_gpu(ctx, step, q, cache, page_table=bad)
            assert status == fd.FD_DEV_BAD_PAGE and (got[8:16] == 0).all()
            check(got[:8], (exp[:8], tol[:8])); check(got[16:], (exp[16:], tol[16:]))
        for lens in [(step.prefix_lens, torch.tensor([8, 9, 8], dtype=torch.int32), step.n_mask),
                     (torch.tensor([100, 10 ** 6, 50], dtype=torch.int32), step.q_lens, step.n_mask)]:
            got, status = attn_gpu(ctx, step, q, cache, lens=lens)
            assert status == fd.FD_DEV_BAD_LENGTHS and (got == 0).all()
        got, status = attn_gpu(ctx, step, q, cache)
        assert status == 0
        check(got, (exp, tol), "after errors")
        n, dq, c = fd.fd_launch_count(ctx.h), q.cuda(), torch.from_numpy(cache).cuda()
        ints = [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda(), step.n_mask.cuda()]
        for args in ([3, 24, dq, None, step.num_pages, *ints, None, dq], [3, 24, dq, c.data_ptr() + 8, step.num_pages, *ints, None, dq],
                     [3, 24, dq, c, 0, *ints, None, dq], [3, 24, None, c, step.num_pages, *ints, None, dq], [4, 24, dq, c, step.num_pages, *ints, None, dq]):
            assert fd.fd_attn_draft_verify_fp8(ctx.h, *args, raise_on_error=False) == fd.FD_ERR_INVALID_ARG
        assert fd.fd_launch_count(ctx.h) == n


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("seed", list(range(600, 608)))
def test_chain_of_attention_calls_under_a_pinned_plan(seed, path):
    """8-bit, 4-bit and bf16 layers under one pinned plan, right behind one another, a call's query sometimes an output before it: the
    bits of the same calls with a wait behind each; the 8-bit ones against the oracle."""
    import fp4_ref

    step, n_blocks = _random_step(seed)
    if step.total_q_rows == 0:
        pytest.skip("all blocks empty")
    s, T = step.shape, step.total_q_rows
    kv = wl.make_kv(step)
    c8, c4 = ref.make_cache(kv, rng_seed=seed), fp4_ref.make_cache(kv, rng_seed=seed)
    pools = {"8": torch.from_numpy(c8).cuda(), "4": torch.from_numpy(c4).cuda(), "b": kv.cuda()}
    k_new, v_new = (torch.randn((T, s.n_kv_heads, s.head_dim), generator=torch.Generator().manual_seed(seed + i)).bfloat16().cuda() for i in (1, 2))
    layers = [("8", 0), ("8", 0), ("8", 1), ("4", 0), ("8", 2), ("b", 0), ("8", 1), ("8", 0), ("a", 0), ("8", 0), ("8", 0)]
    q0 = wl.make_q(step).cuda()
    results = []
    with Ctx(step, path) as ctx:
        for wait in (True, False):
            fd.fd_calls_back_to_back(ctx.h, not wait)
            pools["8"].copy_(torch.from_numpy(c8))
            ints = [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda()]
            nm, nb, outs = step.n_mask.cuda(), n_blocks.cuda(), []
            torch.cuda.synchronize()
            fd.fd_plan_pin(ctx.h, step.batch, T, ints[1], ints[2], nm, nb)
            for fmt, back in layers:
                x = outs[-back] if back else q0
                if fmt == "a":
                    fd.fd_kv_append_fp8(ctx.h, step.batch, T, k_new, v_new, pools["8"], step.num_pages, *ints)
                else:
                    outs.append(torch.full_like(q0, float("nan")))
                    args = [ctx.h, step.batch, T, x, pools[fmt], step.num_pages, *ints, nm, nb]
                    if fmt == "8":
                        fd.fd_attn_draft_verify_fp8(*args, outs[-1])
                    elif fmt == "4":
                        fd.fd_attn_draft_verify_fp4(*args, 1.0, 1.0, outs[-1])
                    else:
                        fd.fd_attn_draft_verify_blocks(*args, outs[-1])
                if wait:
                    torch.cuda.synchronize()
            fd.fd_plan_unpin(ctx.h)
            assert fd.fd_last_device_status(ctx.h) == 0
            results.append(outs)
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    check(results[0][0].double().cpu().numpy(), attn_ref(step, q0.cpu(), c8, n_blocks), "first")
    after = ref.append(c8, s.head_dim, step, k_new.cpu(), v_new.cpu())
    check(results[0][-1].double().cpu().numpy(), attn_ref(step, q0.cpu(), after, n_blocks), "behind the append")
