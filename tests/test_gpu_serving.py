"""GPU parity of the operators around the 4-bit cache and of page reservation, through the C ABI, against the 64-bit
references of fp4_ref.py and the CPU oracle.

Attention tolerance.  The values of the 4-bit cache and the queries enter exactly; what rounds is the softmax weight (held
in at least 11 bits before the product with V: relative 2^-11 each), the exponential and the fp32 sums (relative 2^-14 at
these sizes), and the output (bf16: 2^-8, half a step).  So |err| <= 2^-8 |ref| + 2^-10 sum_j p_j |v_j|, the last factor
from the oracle on the magnitudes of V -- and, where all keys of weight have a V of zero, what the smallest weights lose:
fp16 ends at steps of 2^-24, the largest weight of a row is held as 2^7 or more, so a weight is off by at most
2^-25 / 2^7 = 2^-32 of the largest, which is at most the row's sum: + 2^-32 sum_j |v_j| <= 2^-32 keys max |v|."""
import zlib

import numpy as np
import pytest
import torch

import fp4_ref as ref
import oracle
import paper_2605_20022_b200 as fd
from helpers import Ctx
from paper_2605_20022_b200 import workload as wl
from test_gpu_parity import BLOCK_CASES, EDGE, PATHS, _random_step

pytestmark = pytest.mark.gpu

ONE = wl.Shape(4, 1, 64, 10)


def attn_ref(step, q, cache, n_blocks=None, k_scale=1.0, v_scale=1.0, scale=None):
    """(reference, tolerance) of the attention over a 4-bit cache."""
    d = step.shape.head_dim
    kv = ref.as_bf16_cache(cache, d)
    nb = torch.ones_like(step.n_mask) if n_blocks is None else n_blocks
    scale = (scale or 1 / np.sqrt(d)) * k_scale
    args = (step.page_table, step.prefix_lens, step.q_lens, step.n_mask, nb)
    out = oracle.attn_blocks(q, kv, *args, scale=scale) * v_scale
    kv[:, 1] = kv[:, 1].abs()
    size = oracle.attn_blocks(q, kv, *args, scale=scale) * v_scale
    largest = float(kv[:, 1].double().nan_to_num(0.0).max()) * v_scale
    return out, 2.0 ** -8 * np.abs(out) + 2.0 ** -10 * size + 2.0 ** -32 * int(step.kv_lens.max()) * largest


def attn_gpu(ctx, step, q, cache, n_blocks=None, k_scale=1.0, v_scale=1.0, lens=None, page_table=None, out=None):
    pl, ql, nm = lens if lens is not None else (step.prefix_lens, step.q_lens, step.n_mask)
    pt = step.page_table if page_table is None else page_table
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    c = torch.from_numpy(cache).cuda() if isinstance(cache, np.ndarray) else cache
    fd.fd_attn_draft_verify_fp4(ctx.h, step.batch, step.total_q_rows, q.cuda(), c, step.num_pages, pt.cuda(), pl.cuda(), ql.cuda(),
                                nm.cuda(), None if n_blocks is None else n_blocks.cuda(), k_scale, v_scale, out)
    return out.double().cpu().numpy(), fd.fd_last_device_status(ctx.h)


def check(got, want, what=""):
    exp, tol = want
    assert np.isfinite(got).all(), f"{what}: not finite"
    worst = float((np.abs(got - exp) / tol).max()) if got.size else 0.0
    assert worst <= 1, f"{what}: {worst:.3f} of the tolerance, max |err| {np.abs(got - exp).max():.4g}"


# ---------------------------------------------------------------------------------------------- append and read
ROWS = {
    # name: (Hkv, d, prefix_lens, q_lens)
    "one_token": (1, 64, [0], [1]),
    "page_ends": (2, 128, [0, 15, 16, 31, 700], [32, 3, 17, 1, 20]),
    "empty_between": (8, 64, [5, 9, 100, 33], [0, 16, 0, 7]),
    "many": (3, 128, [(7 * b) % 41 for b in range(300)], [(5 * b) % 9 for b in range(300)]),
    "prompts": (8, 128, [0, 3], [517, 1000]),
}


def _values(shape, seed):
    """N(0, 1) over many magnitudes; exact ties of the codes; zeros, infinities, NaN, the largest and smallest numbers."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    x = x * 10.0 ** torch.randint(-3, 3, shape[:-1] + (1,), generator=g)
    flat = x.view(-1, 16)
    n = flat.shape[0]
    flat[:: 7] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 0.0]) * \
        2.0 ** torch.randint(-5, 6, (len(flat[:: 7]), 1), generator=g)
    for k, v in enumerate((0.0, float("inf"), float("nan"), 3.0e38, 1e-38, -float("inf"))):
        if n > 3 + 11 * k:
            flat[3 + 11 * k, k:] = v
    return x.bfloat16()


@pytest.mark.parametrize("scales", [(1.0, 1.0), (0.75, 1.3)])
@pytest.mark.parametrize("name", sorted(ROWS))
def test_append_and_read_match_the_definition(name, scales):
    """Every byte of the pool against the reference, untouched slots included; then the rows back out of it.  With scales of 1
    (and powers of two) the kernel's arithmetic is exact; x / 0.75 is rounded to 32 bits in both (true division)."""
    Hkv, d, pl, ql = ROWS[name]
    step = wl.make_step(name, wl.Shape(Hkv, Hkv, d, 10), pl, ql, [0] * len(pl), seed=3, extra_table_cols=1)
    T, (ks, vs) = step.total_q_rows, scales
    k, v = _values((T, Hkv, d), 5), _values((T, Hkv, d), 6)
    cache = np.random.default_rng(7).integers(0, 256, (step.num_pages, Hkv, 2, ref.page_bytes(d)), dtype=np.uint8)
    rk, rv = (x if s == 1 else (x.float() / s) for x, s in ((k, ks), (v, vs)))
    want = ref.append(cache, d, step, rk, rv, 1.0, 1.0)
    with Ctx(step, max_q_len=max(ql)) as ctx:
        dev = torch.from_numpy(cache).cuda()
        tail = [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda()]
        fd.fd_kv_append_fp4(ctx.h, step.batch, T, k.cuda(), v.cuda(), dev, step.num_pages, *tail, ks, vs)
        assert fd.fd_last_device_status(ctx.h) == 0
        np.testing.assert_array_equal(dev.cpu().numpy(), want)
        ko, vo = (torch.full((T, Hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        fd.fd_kv_read_fp4(ctx.h, step.batch, T, dev, step.num_pages, *tail, ks, vs, ko, vo)
        assert fd.fd_last_device_status(ctx.h) == 0
    held = ref.values(*ref.split(want, d))
    for got, which, by in ((ko, 0, ks), (vo, 1, vs)):
        exp = np.stack([held[int(step.page_table[b, j // 16]), :, which, j % 16] for b, _, j in ref.rows_of(step)])
        exp = torch.from_numpy((exp * np.float32(by)).astype(np.float32)).to(torch.bfloat16)
        assert torch.equal(got.cpu(), exp)


def test_append_and_read_errors():
    step = wl.make_step("err", wl.Shape(2, 2, 64, 10), [10, 20, 40], [8, 8, 8], [0, 0, 0], seed=4)
    k = torch.randn((24, 2, 64)).bfloat16().cuda()
    cache = torch.full((step.num_pages, 2, 2, ref.page_bytes(64)), 0x77, dtype=torch.uint8, device="cuda")
    table, pl, ql = step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda()
    with Ctx(step) as ctx:
        def both(total=24, table=table, pl=pl, ql=ql):
            c = cache.clone()
            fd.fd_kv_append_fp4(ctx.h, 3, total, k, k, c, step.num_pages, table, pl, ql)
            s1 = fd.fd_last_device_status(ctx.h)
            out = torch.full_like(k, 7.0)
            fd.fd_kv_read_fp4(ctx.h, 3, total, cache, step.num_pages, table, pl, ql, 1.0, 1.0, out, out.clone())
            assert fd.fd_last_device_status(ctx.h) == s1
            return c, out.cpu(), s1

        bad = table.clone(); bad[1, 1] = step.num_pages
        c, out, st = both(table=bad)
        assert st == fd.FD_DEV_BAD_PAGE
        on_page = torch.tensor([(20 + i) // 16 == 1 for i in range(8)])
        assert (out[8:16][on_page] == 0).all() and (out[:8] != 0).any() and (out[16:] != 0).any()
        for i in range(8):                                       # the other sequences' rows are in
            page, tok = int(table[0, (10 + i) // 16]), (10 + i) % 16
            assert not torch.equal(c[page, :, 0, tok * 32:tok * 32 + 32], cache[page, :, 0, tok * 32:tok * 32 + 32])
        c, out, st = both(total=20)                              # the last sequence passes the end
        assert st == fd.FD_DEV_BAD_LENGTHS and (out[16:20] == 0).all() and (out[20:] == 7).all() and (out[:16] != 0).any()
        c, out, st = both(pl=torch.tensor([-1, 20, 40], dtype=torch.int32).cuda())
        assert st == fd.FD_DEV_BAD_LENGTHS and (out[:8] == 0).all() and (out[8:] != 0).any()
        c, out, st = both(pl=torch.tensor([10, 2 ** 31 - 4, 40], dtype=torch.int32).cuda())
        assert st == fd.FD_DEV_BAD_LENGTHS and (out[8:16] == 0).all()
        c, out, st = both(ql=torch.tensor([2 ** 31 - 1, 2 ** 31 - 1, 8], dtype=torch.int32).cuda())
        assert st == fd.FD_DEV_BAD_LENGTHS and torch.equal(c, cache) and (out == 0).all()
        c, out, st = both(ql=torch.tensor([-5, 8, 8], dtype=torch.int32).cuda(), total=24)  # rows behind the last sequence stay
        assert st == 0 and (out[16:] == 7).all()
        n = fd.fd_launch_count(ctx.h)
        t4 = [table, pl, ql]
        for args in ([4, 24, k, k, cache, step.num_pages, *t4], [3, -1, k, k, cache, step.num_pages, *t4],
                     [3, 24, None, k, cache, step.num_pages, *t4], [3, 24, k, k, None, step.num_pages, *t4],
                     [3, 24, k, k, cache.data_ptr() + 8, step.num_pages, *t4], [3, 24, k.data_ptr() + 2, k, cache, step.num_pages, *t4],
                     [3, 24, k, k, cache, step.num_pages, *t4, 0.0, 1.0], [3, 24, k, k, cache, step.num_pages, *t4, 1.0, float("nan")],
                     [3, 24, k, k, cache, step.num_pages, *t4, float("inf"), 1.0], [0, 1, k, k, cache, step.num_pages, *t4]):
            assert fd.fd_kv_append_fp4(ctx.h, *args, raise_on_error=False) == fd.FD_ERR_INVALID_ARG
        assert fd.fd_kv_append_fp4(ctx.h, 0, 0, None, None, None, 0, None, None, None) == fd.FD_OK
        assert fd.fd_kv_read_fp4(ctx.h, 3, 24, cache, step.num_pages, *t4, 1.0, 1.0, None, k, raise_on_error=False) == fd.FD_ERR_INVALID_ARG
        assert fd.fd_launch_count(ctx.h) == n


# ---------------------------------------------------------------------------------------------- reservation
class Pages:
    """A reservation's operands on the device."""

    def __init__(self, table, prefix, q_lens, n_mask, n_blocks, freed, free, pool, with_freed=True):
        t = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
        self.pool, self.batch, self.total = pool, len(prefix), int(np.maximum(q_lens, 0).sum()) if len(q_lens) else 0
        self.table, self.prefix, self.q_lens, self.n_mask = t(table), t(prefix), t(q_lens), t(n_mask)
        self.n_blocks = None if n_blocks is None else t(n_blocks)
        self.free = t(list(free) + [-9] * (pool - len(free)))
        self.n_free = t([len(free)])
        self.freed, self.n_freed = (t(list(freed) + [-8]), t([len(freed)])) if with_freed else (None, None)
        self.slots = torch.full((max(self.total, 1),), -99, dtype=torch.int32, device="cuda")
        self.pos = torch.full((max(self.total, 1),), -99, dtype=torch.int32, device="cuda")

    def call(self, ctx, out=None, total=None, **kw):
        self.n_out = self.n_free if out is None else out
        return fd.fd_kv_reserve(ctx, self.batch, self.total if total is None else total, self.table, self.prefix, self.q_lens, self.n_mask,
                                self.n_blocks, self.freed, self.n_freed, self.free, self.n_free, self.n_out, self.pool, self.slots, self.pos, **kw)

    def check(self, want):
        table, stack, slots, pos, _ = want
        np.testing.assert_array_equal(self.table.cpu().numpy(), table)
        n = int(self.n_out)
        assert n == len(stack)
        np.testing.assert_array_equal(self.free[:n].cpu().numpy(), stack)
        np.testing.assert_array_equal(self.slots[:self.total].cpu().numpy(), slots)
        np.testing.assert_array_equal(self.pos[:self.total].cpu().numpy(), pos)


def _reserve_case(seed, B, most):
    r = np.random.default_rng(seed)
    prefix = np.where(r.random(B) < 0.3, 16 * r.integers(0, 20, B), r.integers(0, 300, B))
    blocks, each = r.integers(1, 4, B), r.integers(0, 5, B)
    cand = np.where(r.random(B) < 0.1, 0, r.integers(1, most, B))
    blocks = np.where(blocks > cand, 1, blocks)
    mask = blocks * each
    rows = cand + mask
    width = int((-(-(prefix + rows) // 16)).max()) + 1
    pool = int((-(-(prefix + rows) // 16)).sum()) + 40
    ids = list(r.permutation(pool))
    table = np.full((B, width), -1)
    for b in range(B):
        for p in range(-(-int(prefix[b]) // 16)):
            table[b, p] = ids.pop()
    k = int(r.integers(0, len(ids)))
    return table, prefix, rows, mask, blocks, ids[:k], ids[k:], pool


def _ctx(case):
    table, _, rows = case[:3]
    return fd.fd_create(4, 1, 64, 10, max(len(rows), 1), max(int(rows.max()), 1), table.shape[1])


@pytest.mark.parametrize("seed,B,most", [(1, 1, 2), (2, 1, 40), (3, 7, 20), (4, 64, 17), (5, 255, 9), (6, 256, 3), (7, 257, 12), (8, 700, 8),
                                         (9, 4096, 3), (10, 3, 4000), (11, 40, 900)])
def test_reserve_matches_the_definition(seed, B, most):
    case = _reserve_case(seed, B, most)
    ctx = _ctx(case)
    try:
        s = Pages(*case)
        keep = s.n_free.clone()
        s.call(ctx, out=torch.full((1,), -5, dtype=torch.int32, device="cuda"))  # the count before the call is left alone
        assert fd.fd_last_device_status(ctx) == 0 and torch.equal(s.n_free, keep)
        s.check(ref.reserve(*case))
        s = Pages(*case)
        s.call(ctx)                                                              # ... or replaced
        s.check(ref.reserve(*case))
        case = case[:5] + ([],) + case[6:]
        s = Pages(*case, with_freed=False)
        if ref.reserve(*case)[4]:
            s.call(ctx)
            assert fd.fd_last_device_status(ctx) == fd.FD_DEV_NO_PAGES
        else:
            s.call(ctx)
            assert fd.fd_last_device_status(ctx) == 0
        s.check(ref.reserve(*case))
        case = case[:4] + (None,) + case[5:]
        if (case[3] <= case[2] - 1).all():
            s = Pages(*case)
            s.call(ctx)
            s.check(ref.reserve(*case))
    finally:
        fd.fd_destroy(ctx)


def test_reserve_takes_pages_until_there_are_none():
    """Exactly enough, then one too few: nothing is handed out, released ids are on the list all the same."""
    table, prefix = np.full((2, 4), -1), [0, 16]
    table[1, 0] = 5
    ctx = fd.fd_create(4, 1, 64, 10, 2, 64, 4)
    try:
        for free, freed in (([1, 2], [3, 4]), ([1, 2], [3]), ([], [1, 2, 3]), ([0, 1, 2], [])):
            case = (table, prefix, [33, 1], [0, 0], None, freed, free, 8)
            s = Pages(*case)
            s.call(ctx)
            want = ref.reserve(*case)
            assert fd.fd_last_device_status(ctx) == (fd.FD_DEV_NO_PAGES if want[4] else 0)
            s.check(want)
            if want[4]:
                assert (s.slots == -1).all() and int(s.pos[0]) == 0
    finally:
        fd.fd_destroy(ctx)


def test_reserve_errors():
    case = (np.full((2, 4), -1), [0, 16], [20, 7], [0, 3], [1, 1], [9], [1, 2, 3, 4, 5], 12)
    case[0][1, 0] = 6
    ctx = fd.fd_create(4, 1, 64, 10, 2, 32, 4)
    try:
        for change in (dict(prefix=[-1, 16]), dict(prefix=[0, 60]), dict(q_lens=[20, -7]), dict(q_lens=[40, 7]), dict(n_mask=[0, 8]),
                       dict(n_mask=[-1, 3]), dict(n_blocks=[1, 2]), dict(n_blocks=[-1, 1]), dict(total=26), dict(n_free=[12]), dict(n_free=[-1]),
                       dict(n_freed=[-1])):
            s = Pages(*case)
            for key, value in change.items():
                if key != "total":
                    setattr(s, key, torch.tensor(value, dtype=torch.int32, device="cuda"))
            before = s.table.clone(), s.free.clone(), int(s.n_free)
            s.call(ctx, total=change.get("total"))
            assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_LENGTHS, change
            n = change.get("total", 27)
            assert (s.slots[:n] == -1).all() and (s.pos[:n] == -1).all() and (s.slots[n:27] == -99).all()
            assert torch.equal(s.table, before[0]) and torch.equal(s.free, before[1]) and int(s.n_free) == before[2]
        for free in ([1, 2, 3, 4, 12], [1, 2, 3, 4, -1]):         # an id outside the pool on the list; the pushed one is fine
            c = case[:5] + ([],) + (free,) + case[7:]
            s = Pages(*c)
            s.call(ctx)
            assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_PAGE
            s.check(ref.reserve(*c))
        c = (case[0].copy(),) + case[1:]                          # ... or where the prefix ends inside a page
        c[0][1, 0] = 77
        c = c[:1] + ([0, 12],) + c[2:]
        s = Pages(*c)
        s.call(ctx)
        assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_PAGE
        table, stack, slots, pos, _ = ref.reserve(*c)
        assert (s.slots.cpu().numpy() == slots).all() and int(s.table[1, 0]) == 77
        s = Pages(*case)
        n = fd.fd_launch_count(ctx)
        for kw in (dict(batch=3), dict(total=-1), dict(pool=0), dict(free=None), dict(n_free=None), dict(freed=None), dict(slots=None), dict(table=None),
                   dict(batch=0)):
            t = Pages(*case)
            for key, value in kw.items():
                setattr(t, key, value)
            assert t.call(ctx, raise_on_error=False) == fd.FD_ERR_INVALID_ARG, kw
        s.pool = 2 ** 28
        assert s.call(ctx, raise_on_error=False) == fd.FD_ERR_UNSUPPORTED
        assert fd.fd_launch_count(ctx) == n
        s = Pages(np.zeros((0, 4)), [], [], [], None, [7, 8], [1], 12)  # no sequence: the released ids go onto the list
        s.call(ctx)
        assert fd.fd_last_device_status(ctx) == 0 and int(s.n_free) == 3 and s.free[:3].tolist() == [1, 7, 8]
    finally:
        fd.fd_destroy(ctx)


# ---------------------------------------------------------------------------------------------- norm, rotation, append
ROPE = {
    # name: (Hq, Hkv, d, rows, rot, adjacent, norm, extra stride)
    "one_row": (4, 1, 64, 1, 64, False, True, 0),
    "block": (32, 8, 128, 32, 128, False, True, 0),
    "adjacent": (8, 2, 128, 37, 128, True, True, 8),
    "half_rotated": (5, 1, 64, 19, 32, False, True, 0),
    "sixteen_rotated_adjacent": (12, 2, 128, 23, 16, True, True, 64),
    "sixteen_rotated": (7, 7, 64, 23, 16, False, True, 8),
    "no_rotation": (16, 2, 64, 40, 0, False, True, 0),
    "no_norm": (8, 4, 128, 11, 128, False, False, 0),
    "copy_only": (4, 4, 64, 9, 0, False, False, 0),
    "many_rows": (16, 1, 128, 2500, 64, False, True, 0),
}


def _rope_state(name, seed=11):
    Hq, Hkv, d, T, rot, adjacent, norm, extra = ROPE[name]
    g = torch.Generator().manual_seed(seed)
    stride = (Hq + 2 * Hkv) * d + extra
    buf = torch.randn((T, stride), generator=g) * 10.0 ** torch.randint(-2, 3, (T, 1), generator=g)
    buf[:, (Hq + 2 * Hkv) * d:] = float("nan")
    pool = T // 16 + 5
    slots = torch.randperm(pool * 16, generator=g)[:T].to(torch.int32)
    slots[T // 2] = -1 if T > 1 else slots[0]                      # a padding row
    pos = torch.randint(0, 70000, (T,), generator=g).to(torch.int32)
    pos[0], pos[-1] = 0, 69999
    angle = np.arange(70000)[:, None] * 1e6 ** (-np.arange(rot // 2) * 2.0 / max(rot, 1))[None]
    table = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().contiguous()
    w = [(1 + 0.2 * torch.randn(d, generator=g)).bfloat16() if norm else None for _ in range(2)]
    return dict(Hq=Hq, Hkv=Hkv, d=d, T=T, rot=rot, adjacent=adjacent, stride=stride, qkv=buf.bfloat16(), pool=pool, slots=slots, pos=pos,
                table=table, wq=w[0], wk=w[1], eps=1e-6)


def _rope_call(ctx, s, q_out, cache, fmt, ks=1.0, vs=1.0, **kw):
    a = dict(s, **kw)
    cuda = lambda t: t.cuda() if isinstance(t, torch.Tensor) else t  # noqa: E731
    return fd.fd_qk_norm_rope_append(ctx, a["T"], cuda(a["qkv"]), a["stride"], cuda(a["wq"]), cuda(a["wk"]), a["eps"], cuda(a["table"]) if a["rot"] else None,
                                     a.get("max_positions", 70000), a["rot"], fd.FD_ROPE_ADJACENT if a["adjacent"] else fd.FD_ROPE_HALVES,
                                     cuda(a["pos"]) if a["rot"] else None, cuda(a["slots"]), q_out, cache, a["pool"], fmt, ks, vs,
                                     raise_on_error=kw.get("raise_on_error", True))


def _rope_ref(s):
    """q, k in 64 bits with the size of their terms, v."""
    x = s["qkv"][:, :(s["Hq"] + 2 * s["Hkv"]) * s["d"]].double().numpy().reshape(s["T"], -1, s["d"])
    out = []
    for lo, n, w in ((0, s["Hq"], s["wq"]), (s["Hq"], s["Hkv"], s["wk"])):
        out.append(ref.norm_rope(x[:, lo:lo + n], None if w is None else w.double().numpy(), s["eps"], s["table"].numpy(), s["pos"].numpy(),
                                 s["rot"], s["adjacent"]))
    return out[0], out[1], x[:, s["Hq"] + s["Hkv"]:]


def _rope_ctx(s):
    return fd.fd_create(s["Hq"], s["Hkv"], s["d"], 10, 4, max(4, -(-s["T"] // 4)), 8)


@pytest.mark.parametrize("name", sorted(ROPE))
def test_norm_rope_append_bf16(name):
    """|err| <= 2^-8 |y| (bf16, half a step) + 2^-18 (|first term| + |second term|): the fp32 sum of at most 128 squares, a square
    root, a division and four products, each 2^-24, add up to less than 2^-18 of the terms' size."""
    s = _rope_state(name)
    (q, qs), (k, ks), v = _rope_ref(s)
    ctx = _rope_ctx(s)
    try:
        q_out = torch.full((s["T"], s["Hq"], s["d"]), 77.0, dtype=torch.bfloat16, device="cuda")
        cache = torch.full((s["pool"], 2, s["Hkv"], 16, s["d"]), 55.0, dtype=torch.bfloat16, device="cuda")
        _rope_call(ctx, s, q_out, cache, fd.FD_KV_BF16)
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)
    got, cache, slots = q_out.double().cpu().numpy(), cache.double().cpu().numpy(), s["slots"].numpy()
    live = slots >= 0
    assert (np.abs(got - q) <= 2.0 ** -8 * np.abs(q) + 2.0 ** -18 * qs)[live].all()
    assert (got[~live] == 77).all()
    kg, vg = cache[slots[live] // 16, 0, :, slots[live] % 16], cache[slots[live] // 16, 1, :, slots[live] % 16]
    assert (np.abs(kg - k[live]) <= 2.0 ** -8 * np.abs(k[live]) + 2.0 ** -18 * ks[live]).all()
    np.testing.assert_array_equal(vg, v[live])
    untouched = np.ones((s["pool"] * 16,), bool)
    untouched[slots[live]] = False
    assert (cache.transpose(0, 3, 1, 2, 4).reshape(s["pool"] * 16, -1)[untouched] == 55).all()


@pytest.mark.parametrize("scales", [(1.0, 1.0), (0.8, 3.0)])
@pytest.mark.parametrize("name", sorted(ROPE))
def test_norm_rope_append_fp4(name, scales):
    """V bit for bit; K within what 32-bit arithmetic leaves open: the scale is a nearest one of a value within 2^-18 of the group's
    exact amax / 6, every held value a nearest multiple of it to a value within 2^-18 of the terms' size."""
    s = _rope_state(name)
    (q, qs), (k, kt), v = _rope_ref(s)
    d, by = s["d"], [np.float64(np.float32(x)) for x in scales]
    ctx = _rope_ctx(s)
    try:
        q_out = torch.full((s["T"], s["Hq"], d), 77.0, dtype=torch.bfloat16, device="cuda")
        cache = torch.full((s["pool"], s["Hkv"], 2, ref.page_bytes(d)), 0x5a, dtype=torch.uint8, device="cuda")
        _rope_call(ctx, s, q_out, cache, fd.FD_KV_FP4, *scales)
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)
    slots = s["slots"].numpy()
    live = slots >= 0
    assert (np.abs(q_out.double().cpu().numpy() - q) <= 2.0 ** -8 * np.abs(q) + 2.0 ** -18 * qs)[live].all()
    codes, sc = ref.split(cache.cpu().numpy(), d)
    page, tok = slots[live] // 16, slots[live] % 16
    wc, ws = ref.quantise((v[live].astype(np.float32) / np.float32(scales[1])).astype(np.float64))
    np.testing.assert_array_equal(sc[page, :, 1, tok], ws)
    np.testing.assert_array_equal(codes[page, :, 1, tok], wc)
    x, off = k[live] / by[0], 2.0 ** -18 * kt[live] / by[0]
    groups = x.shape[:2] + (d // 16, 16)
    amax, slack = np.abs(x.reshape(groups)).max(-1) / 6, off.reshape(groups).max(-1) / 6
    held_s = ref.E4M3[sc[page, :, 0, tok]]
    best = np.abs(amax[..., None] - ref.E4M3).min(-1)
    assert (np.abs(np.minimum(amax, 448) - held_s) <= best + 2 * slack + 1e-12).all()
    held = ref.values(codes[page, :, 0, tok], sc[page, :, 0, tok])
    every = np.concatenate([-ref.E2M1, ref.E2M1])
    near = np.abs(x.reshape(groups)[..., None] - every * held_s[..., None, None]).min(-1).reshape(x.shape)
    assert (np.abs(held - x) <= near + 2 * off + 1e-12).all()
    untouched = np.ones((s["pool"] * 16,), bool)
    untouched[slots[live]] = False
    assert (codes.transpose(0, 3, 1, 2, 4).reshape(s["pool"] * 16, -1)[untouched] == np.tile([0xa, 5], codes[0, :, :, 0].size // 2)).all()


def test_norm_rope_append_errors():
    s = _rope_state("adjacent")
    ctx = _rope_ctx(s)
    try:
        new = lambda: (torch.full((s["T"], s["Hq"], s["d"]), 77.0, dtype=torch.bfloat16, device="cuda"),  # noqa: E731
                       torch.full((s["pool"], 2, s["Hkv"], 16, s["d"]), 55.0, dtype=torch.bfloat16, device="cuda"))
        ref_q, ref_c = new()
        _rope_call(ctx, s, ref_q, ref_c, fd.FD_KV_BF16)
        assert fd.fd_last_device_status(ctx) == 0
        for where, value in ((5, 70000), (5, -1), (5, -2 ** 31)):  # a position outside the table: the row is left alone
            q, c = new()
            pos = s["pos"].clone(); pos[where] = value
            _rope_call(ctx, s, q, c, fd.FD_KV_BF16, pos=pos)
            assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_LENGTHS and (q[where] == 77).all()
            q[where] = ref_q[where]
            assert torch.equal(q, ref_q)
        for value in (s["pool"] * 16, 2 ** 31 - 1):                # a slot beyond the pool: q is written, the cache is not
            q, c = new()
            slots = s["slots"].clone(); slots[5] = value
            _rope_call(ctx, s, q, c, fd.FD_KV_BF16, slots=slots)
            assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_PAGE and torch.equal(q, ref_q)
            at = int(s["slots"][5])
            assert (c[at // 16, :, :, at % 16] == 55).all()
        q, c = new()
        n = fd.fd_launch_count(ctx)
        bad = dict(raise_on_error=False)
        for kw in (dict(T=-1), dict(T=10 ** 6), dict(stride=s["stride"] - 16), dict(stride=s["stride"] + 1), dict(rot=8), dict(rot=144), dict(rot=-16),
                   dict(eps=-1.0), dict(eps=float("nan")), dict(qkv=None), dict(slots=None), dict(pos=None), dict(table=None), dict(max_positions=0),
                   dict(qkv=s["qkv"].cuda().data_ptr() + 2), dict(wq=s["table"].cuda().data_ptr() + 4), dict(pool=-1)):
            assert _rope_call(ctx, s, q, c, fd.FD_KV_BF16, **kw, **bad) == fd.FD_ERR_INVALID_ARG, kw
        assert _rope_call(ctx, s, q, c, 2, **bad) == fd.FD_ERR_INVALID_ARG
        assert _rope_call(ctx, s, q, c, fd.FD_KV_FP4, 0.0, 1.0, **bad) == fd.FD_ERR_INVALID_ARG
        assert _rope_call(ctx, s, q, c, fd.FD_KV_FP4, 1.0, -1.0, **bad) == fd.FD_ERR_INVALID_ARG
        assert _rope_call(ctx, s, None, c, fd.FD_KV_BF16, **bad) == fd.FD_ERR_INVALID_ARG
        x = s["qkv"].cuda()
        assert _rope_call(ctx, s, x, c, fd.FD_KV_BF16, qkv=x, **bad) == fd.FD_ERR_INVALID_ARG   # q onto its own source
        assert _rope_call(ctx, s, q, c, fd.FD_KV_BF16, pool=2 ** 28, **bad) == fd.FD_ERR_UNSUPPORTED
        assert _rope_call(ctx, s, None, None, fd.FD_KV_BF16, T=0, **bad) == fd.FD_OK
        assert fd.fd_launch_count(ctx) == n and fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)


# ---------------------------------------------------------------------------------------------- attention
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("name", sorted(EDGE))
def test_attention_edge_cases(name, path):
    Hq, Hkv, d, pl, ql, nm = EDGE[name]
    step = wl.make_step(name, wl.Shape(Hq, Hkv, d, 1000), pl, ql, nm, seed=zlib.crc32(name.encode()) % 10000, extra_table_cols=2)
    q, cache = wl.make_q(step), ref.make_cache(wl.make_kv(step), rng_seed=9)
    with Ctx(step, path, max_batch=len(pl)) as ctx:
        got, status = attn_gpu(ctx, step, q, cache, k_scale=0.5, v_scale=2.5)
        again, _ = attn_gpu(ctx, step, q, cache, k_scale=0.5, v_scale=2.5)
    assert status == 0
    check(got, attn_ref(step, q, cache, k_scale=0.5, v_scale=2.5), name)
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


@pytest.mark.parametrize("seed", list(range(200, 230)))
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


@pytest.mark.parametrize("Hq,Hkv,d,batch,longest", [(32, 8, 128, 330, 120), (16, 2, 64, 700, 100), (8, 8, 128, 290, 300)])
def test_attention_many_short_sequences(Hq, Hkv, d, batch, longest):
    """A CTA works through a dozen segments of one to three tiles: the roles run pieces ahead of one another."""
    rng = np.random.default_rng(batch)
    pl = rng.integers(0, longest + 1, batch)
    nm = rng.integers(0, 3, batch) * (rng.random(batch) < 0.5)
    ql = rng.integers(0, 6, batch) + nm + (rng.random(batch) < 0.9)
    step = wl.make_step("short sequences", wl.Shape(Hq, Hkv, d, 1000), pl.tolist(), ql.tolist(), nm.tolist(), seed=batch)
    q, cache = wl.make_q(step), ref.make_cache(wl.make_kv(step), rng_seed=batch)
    want = attn_ref(step, q, cache)
    with Ctx(step, 0, max_batch=batch) as ctx:
        first, status = attn_gpu(ctx, step, q, cache)
        assert status == 0
        check(first, want, "short sequences")
        c = torch.from_numpy(cache).cuda()
        for _ in range(60):
            got, status = attn_gpu(ctx, step, q, c)
            assert status == 0 and np.array_equal(got, first), "two runs on the same inputs differ bitwise"


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("Hq,Hkv,d,by", [(32, 8, 128, 4.0), (16, 2, 64, 4.0), (32, 8, 128, 12.0)])
def test_attention_scores_that_rise_and_fall_along_the_sequence(Hq, Hkv, d, by, path):
    """K drifts from tile to tile, so that half of the rows meet a new maximum in every tile (what was summed so far is
    rescaled, again and again) and the other half never after the first."""
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
        for _ in range(20):
            again, _ = attn_gpu(ctx, step, q, cache)
            assert np.array_equal(got, again), "two runs on the same inputs differ bitwise"


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("size,scale", [(3.0e5, 1e-7), (1e-6, 1e4), (8.0, 0.0), (1e30, 1e-32)])
def test_attention_queries_of_any_size(path, size, scale):
    """Queries far outside and far inside fp16's range (the kernels may hold them in 16 bits, but not lose them): rows of one
    call differ by factors of a million, elements within a row by a thousand."""
    step = wl.make_step("sizes", wl.Shape(8, 2, 128, 1000), [300, 40, 1000], [12, 32, 5], [4, 16, 0], seed=12)
    g = torch.Generator().manual_seed(1)
    q = wl.make_q(step).float() * 10.0 ** torch.randint(-2, 2, (1, 1, 128), generator=g)
    q = q * size
    q[3] *= 1e-3
    q[7, 2] = 0.0
    q = q.bfloat16()
    cache = ref.make_cache(wl.make_kv(step))
    with Ctx(step, path, scale=scale) as ctx:
        got, status = attn_gpu(ctx, step, q, cache)
    assert status == 0
    check(got, attn_ref(step, q, cache, scale=scale or None), "sizes")


@pytest.mark.parametrize("path", PATHS)
def test_attention_extreme_scales_of_the_cache(path):
    """Every scale byte from the smallest to the largest: values from 2^-10 to 2688 in one cache."""
    step = wl.make_step("bytes", wl.Shape(8, 2, 64, 1000), [500, 33], [9, 32], [4, 16], seed=13)
    r = np.random.default_rng(2)
    codes = r.integers(0, 16, (step.num_pages, 2, 2, 16, 64)).astype(np.uint8)
    scales = r.integers(0, 127, (step.num_pages, 2, 2, 16, 4)).astype(np.uint8)
    scales[:, :, 0] = r.integers(0, 40, scales[:, :, 0].shape)   # keys: small enough for scores that are not one-hot
    cache = ref.join(codes, scales)
    q = wl.make_q(step)
    with Ctx(step, path) as ctx:
        got, status = attn_gpu(ctx, step, q, cache)
    assert status == 0
    check(got, attn_ref(step, q, cache), "bytes")


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
                     (step.prefix_lens, step.q_lens, torch.tensor([4, 9, 4], dtype=torch.int32)),
                     (torch.tensor([100, -1, 50], dtype=torch.int32), step.q_lens, step.n_mask),
                     (torch.tensor([100, 10 ** 6, 50], dtype=torch.int32), step.q_lens, step.n_mask)]:
            got, status = attn_gpu(ctx, step, q, cache, lens=lens)
            assert status == fd.FD_DEV_BAD_LENGTHS and (got == 0).all()
        got, status = attn_gpu(ctx, step, q, cache)
        assert status == 0
        check(got, (exp, tol), "after errors")
        n, dq, c = fd.fd_launch_count(ctx.h), q.cuda(), torch.from_numpy(cache).cuda()
        ints = [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda(), step.n_mask.cuda()]
        for args in ([3, 24, dq, None, step.num_pages, *ints, None, 1.0, 1.0, dq], [3, 24, dq, c.data_ptr() + 8, step.num_pages, *ints, None, 1.0, 1.0, dq],
                     [3, 24, dq, c, 0, *ints, None, 1.0, 1.0, dq], [3, 24, dq, c, step.num_pages, *ints, None, 0.0, 1.0, dq],
                     [3, 24, dq, c, step.num_pages, *ints, None, 1.0, float("inf"), dq], [3, 24, None, c, step.num_pages, *ints, None, 1.0, 1.0, dq],
                     [4, 24, dq, c, step.num_pages, *ints, None, 1.0, 1.0, dq], [3, -1, dq, c, step.num_pages, *ints, None, 1.0, 1.0, dq]):
            assert fd.fd_attn_draft_verify_fp4(ctx.h, *args, raise_on_error=False) == fd.FD_ERR_INVALID_ARG
        assert fd.fd_launch_count(ctx.h) == n
        assert fd.fd_attn_draft_verify_fp4(ctx.h, 0, 0, None, None, 0, None, None, None, None, None, 1.0, 1.0, None) == fd.FD_OK


@pytest.mark.parametrize("seed", list(range(300, 316)))
def test_chains_of_appends_and_attention_on_both_caches(seed):
    """Layers under one pinned plan, 4-bit and bf16 caches in turn, each call's query sometimes the call before's output, with and
    without the promise that lets consecutive calls overlap."""
    step, _ = _random_step(seed)
    if step.total_q_rows == 0:
        pytest.skip("all blocks empty")
    s, T, L = step.shape, step.total_q_rows, 4
    g = torch.Generator().manual_seed(seed)
    kn = [torch.randn((T, s.n_kv_heads, s.head_dim), generator=g).bfloat16() for _ in range(L)]
    vn = [torch.randn((T, s.n_kv_heads, s.head_dim), generator=g).bfloat16() for _ in range(L)]
    kvs = [wl.make_kv(step, l) for l in range(L)]
    caches = [ref.make_cache(kv) for kv in kvs]
    q0 = wl.make_q(step)
    with Ctx(step) as ctx:
        fd.fd_calls_back_to_back(ctx.h, bool(seed % 2))
        ints = [step.page_table.cuda(), step.prefix_lens.cuda(), step.q_lens.cuda()]
        nm, dq = step.n_mask.cuda(), q0.cuda()
        for rep in range(2):
            pools = [torch.from_numpy(c).cuda() if l != 2 else kvs[2].cuda() for l, c in enumerate(caches)]
            outs = [torch.full(q0.shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(L)]
            fd.fd_plan_pin(ctx.h, step.batch, T, ints[1], ints[2], nm)
            for l in range(L):
                x = outs[l - 1] if l % 2 else dq
                if l == 2:
                    fd.fd_kv_append(ctx.h, step.batch, T, kn[l].cuda(), vn[l].cuda(), pools[l], step.num_pages, *ints)
                    fd.fd_attn_draft_verify(ctx.h, step.batch, T, x, pools[l], step.num_pages, *ints, nm, outs[l])
                else:
                    fd.fd_kv_append_fp4(ctx.h, step.batch, T, kn[l].cuda(), vn[l].cuda(), pools[l], step.num_pages, *ints)
                    fd.fd_attn_draft_verify_fp4(ctx.h, step.batch, T, x, pools[l], step.num_pages, *ints, nm, None, 1.0, 1.0, outs[l])
            fd.fd_plan_unpin(ctx.h)
            assert fd.fd_last_device_status(ctx.h) == 0
            for l in (0, 1, 3):
                c = ref.append(caches[l], s.head_dim, step, kn[l], vn[l], 1.0, 1.0)
                np.testing.assert_array_equal(pools[l].cpu().numpy(), c)
                fed = outs[l - 1].cpu() if l % 2 else q0
                check(outs[l].double().cpu().numpy(), attn_ref(step, fed, c), f"layer {l} rep {rep}")


# ---------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("fp4", [False, True])
def test_decode_loop_reserve_project_attend_accept_commit(fp4):
    """Eight steps as they are used: pages out of the free list, norm + rotation + append, attention, greedy verification, commit --
    each step's page bookkeeping against the reference, each attention against the oracle on what the cache then holds, no page
    lost or handed out twice, every append read back."""
    Hq, Hkv, d, V, B, pool = 8, 2, 64, 50, 5, 60
    r = np.random.default_rng(5)
    g = torch.Generator().manual_seed(5)
    ctx = fd.fd_create(Hq, Hkv, d, V, B, 32, 12)
    t32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
    angle = np.arange(300)[:, None] * 100.0 ** (-np.arange(d // 2) * 2.0 / d)[None]
    cos_sin = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda()
    try:
        table, prefix = t32(np.full((B, 12), -1)), t32(np.zeros(B))
        free, n_free = t32(list(r.permutation(pool))), t32([pool])
        freed, n_freed = torch.zeros(B * 4, dtype=torch.int32, device="cuda"), t32([0])
        cache = torch.randint(0, 256, (pool, Hkv, 2, ref.page_bytes(d)), generator=g, dtype=torch.uint8).cuda() if fp4 else \
            torch.full((pool, 2, Hkv, 16, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        for _ in range(8):
            C = r.integers(1, 9, B)
            M = r.choice([0, 4, 6], B)
            nb = np.where((C >= 2) & (M > 0), 2, 1)
            L = C + M
            T = int(L.sum())
            ql, nm, dnb = t32(L), t32(M), t32(nb)
            want = ref.reserve(table.cpu().numpy(), prefix.cpu().numpy(), L, M, nb, freed[:int(n_freed)].tolist(), free[:int(n_free)].tolist(), pool)
            slots, pos = torch.empty(T, dtype=torch.int32, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda")
            fd.fd_kv_reserve(ctx, B, T, table, prefix, ql, nm, dnb, freed, n_freed, free, n_free, n_free, pool, slots, pos)
            np.testing.assert_array_equal(table.cpu().numpy(), want[0])
            np.testing.assert_array_equal(free[:int(n_free)].cpu().numpy(), want[1])
            held = [p for p in table.flatten().tolist() if p >= 0]
            assert sorted(held + free[:int(n_free)].tolist()) == list(range(pool))
            qkv = torch.randn((T, (Hq + 2 * Hkv) * d), generator=g).bfloat16().cuda()
            w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
            q = torch.empty((T, Hq, d), dtype=torch.bfloat16, device="cuda")
            fd.fd_qk_norm_rope_append(ctx, T, qkv, qkv.stride(0), w, w, 1e-6, cos_sin, 300, d, fd.FD_ROPE_HALVES, pos, slots, q, cache, pool,
                                      fd.FD_KV_FP4 if fp4 else fd.FD_KV_BF16, 0.5, 2.0)
            out = torch.full_like(q, float("nan"))
            if fp4:
                fd.fd_attn_draft_verify_fp4(ctx, B, T, q, cache, pool, table, prefix, ql, nm, dnb, 0.5, 2.0, out)
            else:
                fd.fd_attn_draft_verify_blocks(ctx, B, T, q, cache, pool, table, prefix, ql, nm, dnb, out)
            step = wl.Step("loop", wl.Shape(Hq, Hkv, d, V), 0, 0.0, prefix.cpu().clone(), ql.cpu(), nm.cpu(), table.cpu().clone(), pool)
            R = int(C.sum())
            logits = torch.randn((R, V), generator=g)
            drafts = torch.randint(0, 3, (R,), generator=g).to(torch.int32)
            logits[:, :3] += 2
            acc, bonus = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
            fd.fd_verify_accept(ctx, B, R, logits.cuda(), drafts.cuda(), ql, nm, acc, bonus)
            if fp4:
                ko, vo = torch.empty((T, Hkv, d), dtype=torch.bfloat16, device="cuda"), torch.empty((T, Hkv, d), dtype=torch.bfloat16, device="cuda")
                fd.fd_kv_read_fp4(ctx, B, T, cache, pool, table, prefix, ql, 0.5, 2.0, ko, vo)
                v = qkv[:, (Hq + Hkv) * d:].view(T, Hkv, d)
                assert (vo.float() - v.float()).abs().max() < 0.2 * v.float().abs().max()  # a step of e2m1 at its top is 2 of 6
                check(out.double().cpu().numpy(), attn_ref(step, q.cpu(), cache.cpu().numpy(), dnb.cpu(), 0.5, 2.0), "loop")
            else:
                exp = oracle.attn_blocks(q.cpu(), cache.cpu(), step.page_table, step.prefix_lens, step.q_lens, step.n_mask, dnb.cpu())
                assert (np.abs(out.double().cpu().numpy() - exp) <= 2e-2 + 2e-2 * np.abs(exp)).all()
            fd.fd_kv_commit(ctx, B, table, prefix, ql, acc, freed, n_freed)
            assert fd.fd_last_device_status(ctx) == 0
            wt, wp, wf = oracle.commit(step.page_table, step.prefix_lens, step.q_lens, acc.cpu())
            assert (table.cpu().numpy() == wt).all() and freed[:int(n_freed)].tolist() == wf.tolist()
    finally:
        fd.fd_destroy(ctx)


def test_captured_step_replays_and_other_streams():
    """Reserve, append, read and attention captured in a CUDA graph on a stream of its own and replayed with other inputs in the same
    buffers: the results of eager calls on the default stream."""
    step = wl.make_step("graph", wl.Shape(8, 2, 128, 10), [100, 3, 700], [9, 32, 17], [4, 16, 0], seed=21)
    s, T = step.shape, step.total_q_rows
    held = [-(-int(n) // 16) for n in step.prefix_lens]
    table = step.page_table.clone()
    for b, n in enumerate(held):
        table[b, n:] = -1
    free = [p for p in range(step.num_pages) if p not in set(table.flatten().tolist())]
    with Ctx(step) as ctx:
        st = Pages(table.numpy(), step.prefix_lens.numpy(), step.q_lens.numpy(), step.n_mask.numpy(), None, [], free, step.num_pages)
        n_out = torch.zeros(1, dtype=torch.int32, device="cuda")
        pt0 = st.table.clone()
        q, k, v = (torch.zeros((T, h, 128), dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))
        out, ko, vo = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        cache = torch.from_numpy(ref.make_cache(wl.make_kv(step))).cuda()

        def body():
            st.table.copy_(pt0)
            st.call(ctx.h, out=n_out)
            fd.fd_kv_append_fp4(ctx.h, 3, T, k, v, cache, step.num_pages, st.table, st.prefix, st.q_lens)
            fd.fd_attn_draft_verify_fp4(ctx.h, 3, T, q, cache, step.num_pages, st.table, st.prefix, st.q_lens, st.n_mask, None, 1.0, 1.0, out)
            fd.fd_kv_read_fp4(ctx.h, 3, T, cache, step.num_pages, st.table, st.prefix, st.q_lens, 1.0, 1.0, ko, vo)

        body()                                                   # tensor maps and the like exist before the capture
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            body()
        for seed in range(3):
            g = torch.Generator().manual_seed(seed)
            for t in (q, k, v):
                t.copy_(torch.randn(t.shape, generator=g))
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (out, ko, vo, st.table, st.slots, n_out)]
            for t in (out, ko, vo, st.slots, n_out):
                t.zero_()
            body()
            torch.cuda.synchronize()
            for a, b in zip(got, (out, ko, vo, st.table, st.slots, n_out)):
                assert torch.equal(a, b)
            here = wl.Step("graph", s, 0, 0.0, step.prefix_lens, step.q_lens, step.n_mask, st.table.cpu(), step.num_pages)
            check(out.double().cpu().numpy(), attn_ref(here, q.cpu(), cache.cpu().numpy()), "graph")
        assert fd.fd_last_device_status(ctx.h) == 0
