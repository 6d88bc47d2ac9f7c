"""GPU tests of forking, freeing, compacting and copying pages, against the definitions, and of a run of them with the operators
they stand beside."""
import numpy as np
import pytest
import torch

import fp8_ref as ref
import paper_2605_20022_b200 as fd
from fp4_ref import page_bytes
from paper_2605_20022_b200 import workload as wl
from test_gpu_fp8_cache import attn_ref
from test_gpu_prompt import _check as check_prompt
from test_gpu_serving import check

pytestmark = pytest.mark.gpu

I32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731


class Pool:
    """Host copies of a pool's books, and the calls on the device's."""

    def __init__(self, B, width, pool, seed, lens):
        r = np.random.default_rng(seed)
        self.pool, self.B = pool, B
        ids = list(r.permutation(pool))
        self.table, self.prefix, self.shared = np.full((B, width), -1), np.array(lens), np.zeros(pool, int)
        for b, n in enumerate(lens):
            for p in range(-(-n // 16)):
                self.table[b, p] = ids.pop()
        self.free = [int(x) for x in ids]
        self.up()
        self.ctx = fd.fd_create(2, 1, 64, 10, B, 64, width)

    def up(self):
        self.d_table, self.d_prefix, self.d_shared = I32(self.table), I32(self.prefix), I32(self.shared)
        self.d_free = I32(self.free + [-5] * (self.pool - len(self.free)))
        self.d_n = I32([len(self.free)])

    def same(self, n_free=None):
        n = int(self.d_n if n_free is None else n_free)
        assert n == len(self.free)
        np.testing.assert_array_equal(self.d_table.cpu().numpy(), self.table)
        np.testing.assert_array_equal(self.d_prefix.cpu().numpy(), self.prefix)
        np.testing.assert_array_equal(self.d_shared.cpu().numpy(), self.shared)
        np.testing.assert_array_equal(self.d_free[:n].cpu().numpy(), self.free)

    def fork(self, parents, children, out=None, n=None):
        n = len(parents) if n is None else n
        src, dst = I32(np.full(max(n, 1), -9)), I32(np.full(max(n, 1), -9))
        fd.fd_kv_fork(self.ctx, n, I32(parents), I32(children), self.B, self.d_table, self.d_prefix, self.d_shared, self.d_free, self.d_n,
                      self.d_n if out is None else out, self.pool, src, dst)
        return fd.fd_last_device_status(self.ctx), src.tolist()[:n], dst.tolist()[:n]

    def give_back(self, seqs, out=None):
        fd.fd_kv_free(self.ctx, len(seqs), I32(seqs), self.B, self.d_table, self.d_prefix, self.d_shared, self.d_free, self.d_n,
                      self.d_n if out is None else out, self.pool)
        return fd.fd_last_device_status(self.ctx)

    def compact(self, most, with_shared=True):
        pm, src, dst, n = I32(np.full(self.pool, -9)), I32(np.full(max(most, 1), -9)), I32(np.full(max(most, 1), -9)), I32([-9])
        fd.fd_kv_compact(self.ctx, self.B, self.d_table, self.d_shared if with_shared else None, self.d_free, self.d_n, self.pool, pm, most, src, dst, n)
        return fd.fd_last_device_status(self.ctx), pm.cpu().numpy(), src.tolist()[:most], dst.tolist()[:most], int(n)

    def check_owners(self):
        """Every page is free or owned, and shared counts its owners beyond the first."""
        owners = np.zeros(self.pool, int)
        for b in range(self.B):
            for p in range(-(-int(self.prefix[b]) // 16)):
                owners[self.table[b, p]] += 1
        for i in self.free:
            assert owners[i] == 0
            owners[i] = 1
        assert (owners >= 1).all()
        np.testing.assert_array_equal(self.shared, owners - 1)


@pytest.fixture
def pools():
    made = []

    def make(*a):
        made.append(Pool(*a))
        return made[-1]

    yield make
    for p in made:
        fd.fd_destroy(p.ctx)


@pytest.mark.parametrize("seed,B,longest,width", [(1, 2, 40, 4), (2, 3, 16, 1), (3, 40, 300, 30), (4, 300, 100, 9), (5, 20, 20000, 1300), (6, 4096, 30, 2),
                                                  (7, 600, 900, 70)])
def test_fork_free_compact_match_the_definition(pools, seed, B, longest, width):
    """Rounds of forks, of sequences that end (prompts before their samples, too) and of compactions; in place and into another count."""
    r = np.random.default_rng(seed)
    lens = np.zeros(B, int)
    lens[: max(1, B // 4)] = r.integers(0, longest + 1, max(1, B // 4))
    lens[0] = longest
    pages = int((-(-lens // 16)).sum())
    s = pools(B, width, pages + B + 40 if seed != 5 else 9000, seed, lens)
    for turn in range(4):
        alive, idle = np.flatnonzero(s.prefix > 0), np.flatnonzero(s.prefix == 0)
        n = int(r.integers(1, len(idle) + 1)) if len(idle) else 0
        children = r.permutation(idle)[:n]
        parents = r.choice(alive, n) if len(alive) else np.zeros(0, int)
        need = int((s.prefix[parents] % 16 > 0).sum())
        if len(alive) and need <= len(s.free):
            s.table, s.prefix, s.shared, s.free, copies = ref.fork(parents, children, s.table, s.prefix, s.shared, s.free)
            out = I32([0]) if turn % 2 else None
            status, src, dst = s.fork(parents, children, out)
            assert status == 0 and list(zip(src, dst)) == copies
            if out is not None:
                s.d_n = out
            s.same()
            s.check_owners()
        gone = r.permutation(B)[: int(r.integers(0, B + 1))]
        s.table, s.prefix, s.shared, s.free = ref.free(gone, s.table, s.prefix, s.shared, s.free)
        assert s.give_back(gone) == 0
        s.same()
        s.check_owners()
        most = min(len(s.free), s.pool - len(s.free))
        s.table, s.shared, s.free, pm, moves = ref.compact(s.table, s.shared, s.free, s.pool)
        status, got_map, src, dst, count = s.compact(most + turn)
        assert status == 0 and count == len(moves) and list(zip(src, dst))[:count] == moves and set(src[count:] + dst[count:]) <= {-1}
        np.testing.assert_array_equal(got_map, pm)
        s.same()
        s.check_owners()
        if not (s.prefix > 0).any():
            break


def test_freeing_in_the_order_of_forking_undoes_it(pools):
    s = pools(30, 20, 400, 9, [100 + 7 * b for b in range(6)] + [0] * 24)
    parents, children = [b % 6 for b in range(24)], list(range(6, 30))
    assert s.fork(parents, children)[0] == 0
    assert int(s.d_n) < len(s.free)
    assert s.give_back(children) == 0
    s.same()


def test_page_errors_leave_everything_as_it_was(pools):
    s = pools(6, 8, 60, 3, [100, 50, 32, 0, 0, 0])
    B, P = fd.FD_DEV_BAD_LENGTHS, fd.FD_DEV_BAD_PAGE
    for parents, children in (([0, 1], [3, 3]), ([0, 3], [3, 4]), ([0], [0]), ([6], [3]), ([-1], [3]), ([0], [6]), ([0], [-1]), ([2 ** 31 - 1], [3])):
        status, src, dst = s.fork(parents, children)
        assert status == B and set(src + dst) == {-1}
        s.same()
    for seqs in ([0, 0], [6], [-1], [1, 2, 1], [-2 ** 31]):
        assert s.give_back(seqs) == B
        s.same()
    for bad in (-1, 129, 2 ** 31 - 1):
        s.d_prefix[1] = bad
        assert s.fork([0, 1], [3, 4])[0] == B and s.give_back([0, 1]) == B
        s.up()
        s.same()
    for n in (-1, 61, 2 ** 31 - 1):
        s.d_n = I32([n])
        assert s.fork([0], [3])[0] == B and s.give_back([0]) == B and int(s.d_n) == n
        status, pm, _, _, count = s.compact(30)
        assert status == B and count == 0 and (pm == np.arange(60)).all()
        s.d_n = I32([len(s.free)])
        s.same()
    # too few pages
    full, s.free = s.free, []
    s.up()
    status, src, dst = s.fork([0, 1], [3, 4])
    assert status == fd.FD_DEV_NO_PAGES and set(src + dst) == {-1}
    s.same()
    status, src, dst = s.fork([2], [3])                        # (a length of whole pages needs none)
    assert status == 0 and src == dst == [-1]
    s.free = full
    s.up()
    # a free list with an id twice or outside the pool
    for bad in (s.free[1], 60, -1):
        s.d_free[0] = bad
        status, pm, _, _, count = s.compact(60)
        assert status == P and count == 0 and (pm == np.arange(60)).all()
        s.up()
    moves = ref.compact(s.table, s.shared, s.free, s.pool)[4]
    assert len(moves) > 1
    status, pm, _, _, count = s.compact(len(moves) - 1)
    assert status == B and count == 0
    s.same()


def test_page_ids_outside_the_pool(pools):
    s = pools(5, 8, 60, 4, [100, 50, 0, 0, 0])
    s.d_table[0, 2] = 60                                       # a whole page of the first, the begun one of the second
    s.d_table[1, 3] = -7
    n = len(s.free)
    status, src, dst = s.fork([0, 1], [2, 3])
    assert status == fd.FD_DEV_BAD_PAGE and src == [int(s.table[0, 6]), -1] and dst == [s.free[-1], -1] and int(s.d_n) == n - 2
    assert s.d_table[2].tolist() == [int(s.table[0, p]) if p != 2 else -1 for p in range(6)] + [s.free[-1], -1]
    assert s.d_table[3, 3] == s.free[-2]
    assert s.give_back([2, 3]) == fd.FD_DEV_BAD_PAGE
    assert int(s.d_n) == n and s.d_free[:n].tolist() == s.free and int(s.d_shared.abs().sum()) == 0


def test_a_page_held_more_often_than_counted_is_pushed_once(pools):
    s = pools(4, 8, 40, 5, [64, 64, 0, 0])
    s.d_table[1] = s.d_table[0]
    n = len(s.free)
    assert s.give_back([0, 1]) == fd.FD_DEV_BAD_PAGE
    assert int(s.d_n) == n + 4 and sorted(s.d_free[n:n + 4].tolist()) == sorted(s.table[0, :4].tolist()) and int(s.d_shared.abs().sum()) == 0


@pytest.mark.parametrize("Hkv,d,pages,copies", [(1, 64, 9, 4), (8, 128, 300, 140), (3, 64, 70, 30), (37, 128, 12, 5), (8, 128, 2000, 900)])
@pytest.mark.parametrize("fmt", [fd.FD_KV_BF16, fd.FD_KV_FP4, fd.FD_KV_FP8])
def test_copies(fmt, Hkv, d, pages, copies):
    block = {fd.FD_KV_BF16: 32 * d, fd.FD_KV_FP4: page_bytes(d), fd.FD_KV_FP8: ref.block_bytes(d)}[fmt]
    g = torch.Generator(device="cuda").manual_seed(1)
    cache = torch.randint(0, 256, (pages, 2 * Hkv * block), generator=g, dtype=torch.uint8, device="cuda")
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(2))
    dst, src = ids[:copies], ids[copies:][torch.arange(copies) % max(1, pages - 2 * copies + 1)]  # (a source may be copied often)
    want = cache.clone()
    live = torch.arange(copies) % 7 != 3
    want[dst[live].cuda()] = cache[src[live].cuda()]
    a, b = I32(torch.where(live, src, -1)), I32(dst)
    b[~live.cuda()] = torch.where(torch.arange(int((~live).sum()), device="cuda") % 2 == 0, -1, b[~live.cuda()]).int()
    ctx = fd.fd_create(Hkv, Hkv, d, 10, 1, 1, 4)
    try:
        for n in (None, copies, copies // 2, 0, -3, copies + 5):
            dev = cache.clone()
            fd.fd_kv_copy_pages(ctx, copies, None if n is None else I32([n]), a, b, dev, pages, fmt)
            assert fd.fd_last_device_status(ctx) == 0
            exp = want
            if n is not None and n < copies:
                exp = cache.clone()
                sel = live & (torch.arange(copies) < n)
                exp[dst[sel].cuda()] = cache[src[sel].cuda()]
            assert torch.equal(dev, exp)
        dev = cache.clone()
        a[0], b[0] = pages, 0
        a[1], b[1] = 0, 2 ** 31 - 1
        fd.fd_kv_copy_pages(ctx, 2, None, a, b, dev, pages, fmt)
        assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_PAGE and torch.equal(dev, cache)
        n = fd.fd_launch_count(ctx)
        for args in ([-1, None, a, b, dev, pages, fmt], [1, None, None, b, dev, pages, fmt], [1, None, a, b, None, pages, fmt], [1, None, a, b, dev, pages, 3],
                     [1, None, a, b, dev.data_ptr() + 8, pages, fmt], [1, None, a, b, dev, -1, fmt]):
            assert fd.fd_kv_copy_pages(ctx, *args, raise_on_error=False) == fd.FD_ERR_INVALID_ARG
        assert fd.fd_kv_copy_pages(ctx, 0, None, None, None, None, 0, fmt) == fd.FD_OK and fd.fd_launch_count(ctx) == n
    finally:
        fd.fd_destroy(ctx)


def test_refusals(pools):
    s = pools(3, 4, 20, 1, [10, 0, 0])
    i, n = I32([0, 1, 2]), fd.fd_launch_count(s.ctx)
    good = [1, i, i, 3, s.d_table, s.d_prefix, s.d_shared, s.d_free, s.d_n, s.d_n, 20, i, i]
    for at, v in ((0, -1), (0, 4), (1, None), (2, None), (3, 4), (3, -1), (3, 0), (4, None), (5, None), (6, None), (7, None), (8, None), (9, None), (10, 0),
                  (11, None), (12, None)):
        assert fd.fd_kv_fork(s.ctx, *(good[:at] + [v] + good[at + 1:]), raise_on_error=False) == fd.FD_ERR_INVALID_ARG, at
    good = [1, i, 3, s.d_table, s.d_prefix, s.d_shared, s.d_free, s.d_n, s.d_n, 20]
    for at, v in ((0, -1), (0, 4), (1, None), (2, 4), (3, None), (4, None), (5, None), (6, None), (7, None), (8, None), (9, 0)):
        assert fd.fd_kv_free(s.ctx, *(good[:at] + [v] + good[at + 1:]), raise_on_error=False) == fd.FD_ERR_INVALID_ARG, at
    good = [3, s.d_table, s.d_shared, s.d_free, s.d_n, 20, s.d_free, 3, i, i, s.d_n]
    for at, v in ((0, -1), (0, 4), (1, None), (3, None), (4, None), (5, 0), (6, None), (7, -1), (8, None), (9, None), (10, None)):
        assert fd.fd_kv_compact(s.ctx, *(good[:at] + [v] + good[at + 1:]), raise_on_error=False) == fd.FD_ERR_INVALID_ARG, at
    for call, args in ((fd.fd_kv_fork, [1, i, i, 3, s.d_table, s.d_prefix, s.d_shared, s.d_free, s.d_n, s.d_n, 2 ** 27, i, i]),
                       (fd.fd_kv_free, [1, i, 3, s.d_table, s.d_prefix, s.d_shared, s.d_free, s.d_n, s.d_n, 2 ** 27]),
                       (fd.fd_kv_compact, [3, s.d_table, s.d_shared, s.d_free, s.d_n, 2 ** 27, s.d_free, 3, i, i, s.d_n])):
        assert call(s.ctx, *args, raise_on_error=False) == fd.FD_ERR_UNSUPPORTED
    assert fd.fd_launch_count(s.ctx) == n
    assert s.fork([], [])[0] == 0 and s.give_back([]) == 0
    s.same()


# ---------------------------------------------------------------------------------------------- together
def _prompts_to_samples(ctx, st, Hq, Hkv, d, prompts, samples):
    """Prompts in (norm and rotation to rows, attention, append in 8 bits), samples branch off, one decode step of all of them."""
    B, T = len(prompts) * (1 + samples), sum(prompts)
    fd.fd_kv_reserve(ctx, len(prompts), T, st["table"], st["prefix"], st["q_lens"], st["none"], None, None, None, st["free"], st["n_free"], st["n_free"],
                     st["pool"], st["slots"], st["pos"])
    fd.fd_qk_norm_rope_append(ctx, T, st["qkv"], st["qkv"].stride(0), st["w"], st["w"], 1e-6, st["cos_sin"], st["cos_sin"].shape[0], d, fd.FD_ROPE_HALVES,
                              st["pos"], st["row"], st["q"], st["rows"], st["cap"], fd.FD_KV_ROWS)
    k, v = st["rows"][0], st["rows"][1]
    fd.fd_attn_prompt(ctx, len(prompts), T, T, st["q"], Hq * d, k, v, Hkv * d, st["q_lens"], None, st["out"])
    fd.fd_kv_append_fp8(ctx, len(prompts), T, k, v, st["cache"], st["pool"], st["table"], st["prefix"], st["q_lens"])
    st["prefix"][: len(prompts)] += st["q_lens"]
    n = len(prompts) * samples
    fd.fd_kv_fork(ctx, n, st["parents"], st["children"], B, st["table"], st["prefix"], st["shared"], st["free"], st["n_free"], st["n_free"], st["pool"],
                  st["src"], st["dst"])
    fd.fd_kv_copy_pages(ctx, n, None, st["src"], st["dst"], st["cache"], st["pool"], fd.FD_KV_FP8)
    T2 = 3 * B
    fd.fd_kv_reserve(ctx, B, T2, st["table"], st["prefix"], st["q_lens2"], st["none"], None, None, None, st["free"], st["n_free"], st["n_free"], st["pool"],
                     st["slots2"], st["pos2"])
    fd.fd_kv_append_fp8(ctx, B, T2, st["k2"], st["v2"], st["cache"], st["pool"], st["table"], st["prefix"], st["q_lens2"])
    fd.fd_attn_draft_verify_fp8(ctx, B, T2, st["q2"], st["cache"], st["pool"], st["table"], st["prefix"], st["q_lens2"], st["none"], None, st["out2"])


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (16, 2, 64)])
def test_prompts_to_samples_to_a_compacted_pool(Hq, Hkv, d):
    """The operators as they are used: prompts attend and enter the 8-bit cache, samples share their pages, decode, end; the pool is
    compacted and decodes on.  Eagerly and replayed from a graph, every stage against its reference."""
    prompts, samples, pool, cap = [33, 160, 5], 3, 120, 13
    T, B = sum(prompts), len(prompts) * (1 + samples)
    g = torch.Generator().manual_seed(d)
    r = np.random.default_rng(d)
    ctx = fd.fd_create(Hq, Hkv, d, 10, B, 256, 14)
    angle = np.arange(400)[:, None] * 100.0 ** (-np.arange(d // 2) * 2.0 / d)[None]
    ids = r.permutation(pool)
    table0, prefix0 = np.full((B, 14), -1), np.zeros(B, int)
    bf = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    st = dict(pool=pool, cap=cap, qkv=bf(T, (Hq + 2 * Hkv) * d), w=torch.ones(d, dtype=torch.bfloat16, device="cuda"),
              cos_sin=torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda(), q=z(T, Hq, d), out=z(T, Hq, d),
              rows=z(2, cap * 16, Hkv, d), row=I32(np.arange(T)), slots=I32(np.zeros(T)), pos=I32(np.zeros(T)), q_lens=I32(prompts), none=I32(np.zeros(B)),
              cache=torch.randint(0, 256, (pool, Hkv, 2, ref.block_bytes(d)), generator=g, dtype=torch.uint8).cuda(), table=I32(table0), prefix=I32(prefix0),
              shared=I32(np.zeros(pool)), free=I32(ids), n_free=I32([pool]), parents=I32(np.arange(9) % 3), children=I32(3 + np.arange(9)),
              src=I32(np.zeros(9)), dst=I32(np.zeros(9)), q_lens2=I32([3] * B), slots2=I32(np.zeros(3 * B)), pos2=I32(np.zeros(3 * B)), k2=bf(3 * B, Hkv, d),
              v2=bf(3 * B, Hkv, d), q2=bf(3 * B, Hq, d), out2=z(3 * B, Hq, d))
    try:
        def reset():
            st["table"].copy_(I32(table0)); st["prefix"].zero_(); st["shared"].zero_(); st["free"].copy_(I32(ids)); st["n_free"].fill_(pool)
            st["out"].fill_(float("nan")); st["out2"].fill_(float("nan"))

        def verify():
            assert fd.fd_last_device_status(ctx) == 0
            k, v = st["rows"][0][:T], st["rows"][1][:T]
            assert torch.equal(v, st["qkv"].view(T, Hq + 2 * Hkv, d)[:, Hq + Hkv:])
            check_prompt(st["out"], st["q"], k, v, prompts, prompts, "prompt")
            parents = [0, 1, 2] + [i % 3 for i in range(9)]
            assert st["prefix"].tolist() == [prompts[p] for p in parents]
            step = wl.Step("run", wl.Shape(Hq, Hkv, d, 10), 0, 0.0, st["prefix"].cpu(), st["q_lens2"].cpu(), st["none"].cpu(), st["table"].cpu(), pool)
            cache = st["cache"].cpu().numpy()
            check(st["out2"].double().cpu().numpy(), attn_ref(step, st["q2"].cpu(), cache), "decode")
            # the prompt's values, through every sample's own table
            held, row = ref.values(*ref.split(cache, d)), 0
            full = {}
            for b, n in enumerate(prompts):
                for h in range(Hkv):
                    for t in range(n // 16 * 16):
                        full[b, t, h] = (k[row + t, h].double().cpu().numpy(), v[row + t, h].double().cpu().numpy())
                row += n
            for i, p in enumerate(parents):
                for t in range(0, prompts[p] // 16 * 16, 5):
                    for h in range(Hkv):
                        for which in (0, 1):
                            x, y = full[p, t, h][which], held[int(step.page_table[i, t // 16]), h, which, t % 16]
                            assert (np.abs(x - y) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * 2.0 ** -4)).all()
            return step

        reset()
        _prompts_to_samples(ctx, st, Hq, Hkv, d, prompts, samples)
        step = verify()
        # sequences end, the pool is compacted, the others decode on: the same values through other pages
        gone = [1, 4, 7, 0]
        st["prefix"] += st["q_lens2"]
        fd.fd_kv_free(ctx, 4, I32(gone), B, st["table"], st["prefix"], st["shared"], st["free"], st["n_free"], st["n_free"], pool)
        stay = [b for b in range(B) if b not in gone]
        pm, src, dst, n = I32(np.zeros(pool)), I32(np.zeros(pool)), I32(np.zeros(pool)), I32([0])
        fd.fd_kv_compact(ctx, B, st["table"], st["shared"], st["free"], st["n_free"], pool, pm, pool, src, dst, n)
        fd.fd_kv_copy_pages(ctx, pool, n, src, dst, st["cache"], pool, fd.FD_KV_FP8)
        out3 = torch.full_like(st["out2"][: 3 * len(stay)], float("nan"))
        st["prefix"] -= st["q_lens2"]
        sel = torch.tensor(stay).cuda()
        rows = (sel[:, None] * 3 + torch.arange(3, device="cuda")).flatten()
        tb, pf, ql = st["table"][sel].contiguous(), st["prefix"][sel].contiguous(), st["q_lens2"][sel].contiguous()
        fd.fd_attn_draft_verify_fp8(ctx, len(stay), 3 * len(stay), st["q2"][rows].contiguous(), st["cache"], pool, tb, pf, ql, st["none"], None, out3)
        assert fd.fd_last_device_status(ctx) == 0 and int(n) > 0
        used = pool - int(st["n_free"])
        assert int(tb.max()) < used and torch.equal(st["free"][: int(st["n_free"])].cpu(), torch.arange(pool - 1, used - 1, -1, dtype=torch.int32))
        here = wl.Step("run", wl.Shape(Hq, Hkv, d, 10), 0, 0.0, pf.cpu(), ql.cpu(), st["none"][: len(stay)].cpu(), tb.cpu(), pool)
        check(out3.double().cpu().numpy(), attn_ref(here, st["q2"][rows].cpu(), st["cache"].cpu().numpy()), "compacted")
        # not bitwise: another batch is cut into other pieces
        assert (out3.double() - st["out2"][rows].double()).abs().max() < 2e-2
        # replayed from a graph
        reset()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _prompts_to_samples(ctx, st, Hq, Hkv, d, prompts, samples)
        for _ in range(2):
            reset()
            graph.replay()
            torch.cuda.synchronize()
            verify()
    finally:
        fd.fd_destroy(ctx)
