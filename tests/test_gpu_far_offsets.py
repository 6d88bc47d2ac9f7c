"""Offsets beyond 32 bits (pools and rows of several GB), and two contexts at work at once: each result is, bit for bit, that of the same call on
small memory, by itself."""
import pytest
import torch

import paper_2605_20022_b200 as fd

pytestmark = pytest.mark.gpu

PAGES, HKV, D = 140_000, 8, 128  # pages of 33 024 bytes in 8 bits: 4.6 GB


def I32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _randn(*shape, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


@pytest.mark.parametrize("path", [fd.FD_ATTN_AUTO, fd.FD_ATTN_SIMT])
def test_8_bit_pages_beyond_32_bits(path):
    n, Lq, Hq = 200, 9, 32
    k, v, q = _randn(n, HKV, D, seed=1), _randn(n, HKV, D, seed=2), _randn(Lq, Hq, D, seed=3)
    last = -(-n // 16)
    results = []
    for pages in (64, PAGES):
        cache = torch.empty((pages, HKV, 2, fd.fd_kv_fp8_block_bytes(D)), dtype=torch.uint8, device="cuda")
        cache[:1].fill_(255)
        cache[pages - 40:].fill_(255)
        table = torch.arange(pages - 1, pages - 1 - last, -1, dtype=torch.int32, device="cuda")[None].contiguous()
        ctx = fd.fd_create(Hq, HKV, D, 10, 1, 64, last, attn_path=path)
        try:
            fd.fd_kv_append_fp8(ctx, 1, n, k, v, cache, pages, table, I32(0), I32(n))
            ko, vo, out = torch.empty_like(k), torch.empty_like(v), torch.empty_like(q)
            fd.fd_kv_read_fp8(ctx, 1, n, cache, pages, table, I32(0), I32(n), ko, vo)
            fd.fd_attn_draft_verify_fp8(ctx, 1, Lq, q, cache, pages, table, I32(n - Lq), I32(Lq), I32(2), None, out)
            fd.fd_kv_copy_pages(ctx, 1, None, I32(pages - 1), I32(pages - 30), cache, pages, fd.FD_KV_FP8)
            assert fd.fd_last_device_status(ctx) == 0
            assert torch.equal(cache[pages - 30], cache[pages - 1]) and (cache[0] == 255).all() and (cache[pages - 29:pages - last] == 255).all()
        finally:
            fd.fd_destroy(ctx)
        results.append((ko, vo, out))
        del cache
    for near, far in zip(*results):
        assert torch.equal(near, far) and torch.isfinite(far).all()
    assert ((results[1][0].float() - k.float()).abs() <= (k.float().abs() * 2.0 ** -4).clamp(min=2.0 ** -12)).all()  # (half a step; blocks below 8)


@pytest.mark.parametrize("path", [fd.FD_ATTN_AUTO, fd.FD_ATTN_SIMT])
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_rows_beyond_32_bits(d, path):
    """Rows of 2^20 elements: the last ones start 4.6 GB in.  A value that is not finite is taken out and put back there too."""
    Hq, Hkv, T, stride = 4, 2, 2200, 1 << 20
    wide = torch.empty((T, stride), dtype=torch.bfloat16, device="cuda")
    ctx = fd.fd_create(Hq, Hkv, d, 10, 2, 1, 4, attn_path=path)
    try:
        q, k, v = (wide[:, at:at + h * d].view(T, h, d) for at, h in ((8, Hq), (1 << 12, Hkv), (1 << 19, Hkv)))
        for i, x in enumerate((q, k, v)):
            x.copy_(_randn(*x.shape, seed=i))
        v[2150, 1, 5] = float("inf")
        outs = []
        for a, b, c in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
            out = torch.full((T, Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
            fd.fd_attn_prompt(ctx, 2, T, T, a, a.stride(0), b, c, b.stride(0), I32(100, 2100), None, out)
            outs.append(out)
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)
    assert torch.equal(outs[0], outs[1])
    assert torch.isfinite(outs[0][:2150]).all() and (outs[0][2150:, 2:, 5] == float("inf")).all()


def test_rows_out_of_the_norm_beyond_32_bits():
    T, Hq = 5, 8
    qkv, w = _randn(T, (Hq + 2 * HKV) * D, seed=4), _randn(D, seed=5)
    cos_sin, pos = torch.randn((16, D), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda"), I32(3, 1, 4, 1, 5)
    ctx = fd.fd_create(Hq, HKV, D, 10, 1, 64, 4)
    try:
        got = []
        for pages in (4, PAGES):
            q, rows = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.empty((2, pages * 16, HKV, D), dtype=torch.bfloat16, device="cuda")
            fd.fd_qk_norm_rope_append(ctx, T, qkv, qkv.stride(0), w, w, 1e-6, cos_sin, 16, D, fd.FD_ROPE_HALVES, pos, I32(*range(pages * 16 - T, pages * 16)), q, rows, pages,
                                      fd.FD_KV_ROWS)
            assert fd.fd_last_device_status(ctx) == 0
            got.append((q, rows[:, -T:].clone()))
            del rows
    finally:
        fd.fd_destroy(ctx)
    for near, far in zip(*got):
        assert torch.equal(near, far)


def test_two_contexts_at_once():
    """Prompt, 8-bit attention and page calls of two contexts on two streams, eagerly and as two graphs replayed side by side."""
    Hq, T = 16, 700
    made = []
    for seed in (1, 2):
        q, k, v = _randn(T, Hq, D, seed=seed), _randn(T, HKV, D, seed=seed + 10), _randn(T, HKV, D, seed=seed + 20)
        pages = 120
        s = dict(ctx=fd.fd_create(Hq, HKV, D, 10, 4, 64, 50), q=q, k=k, v=v, pages=pages, prompt=torch.zeros_like(q), out=torch.zeros_like(q[:40]),
                 cache=torch.zeros((pages, HKV, 2, fd.fd_kv_fp8_block_bytes(D)), dtype=torch.uint8, device="cuda"), stream=torch.cuda.Stream(),
                 table=torch.full((4, 50), -1, dtype=torch.int32, device="cuda"), lens=I32(T - 40, 0, 0, 0), shared=torch.zeros(pages, dtype=torch.int32, device="cuda"),
                 free=torch.arange(pages - 44, dtype=torch.int32, device="cuda"), n_free=I32(pages - 44), src=I32(0, 0), dst=I32(0, 0),
                 one=I32(T), zero=I32(0), n_mask=I32(4), Lq=I32(40), parents=I32(0, 0), children=I32(1, 2))
        s["table"][0, :44] = torch.arange(pages - 1, pages - 45, -1, dtype=torch.int32, device="cuda")
        made.append(s)

    def run(s):
        c, table = s["ctx"], s["table"]
        fd.fd_attn_prompt(c, 1, T, T, s["q"], Hq * D, s["k"], s["v"], HKV * D, s["one"], None, s["prompt"])
        fd.fd_kv_append_fp8(c, 1, T, s["k"], s["v"], s["cache"], s["pages"], table, s["zero"], s["one"])
        fd.fd_attn_draft_verify_fp8(c, 1, 40, s["q"], s["cache"], s["pages"], table, s["lens"], s["Lq"], s["n_mask"], None, s["out"])
        fd.fd_kv_fork(c, 2, s["parents"], s["children"], 4, table, s["lens"], s["shared"], s["free"], s["n_free"], s["n_free"], s["pages"], s["src"], s["dst"])
        fd.fd_kv_copy_pages(c, 2, None, s["src"], s["dst"], s["cache"], s["pages"], fd.FD_KV_FP8)
        fd.fd_kv_free(c, 2, s["children"], 4, table, s["lens"], s["shared"], s["free"], s["n_free"], s["n_free"], s["pages"])

    def state(s):
        torch.cuda.synchronize()
        assert fd.fd_last_device_status(s["ctx"]) == 0
        return [s[x].clone() for x in ("prompt", "out", "table", "lens", "shared", "free", "n_free", "src", "dst")] + [s["cache"][s["table"][0, :44].long()]]

    try:
        want = []
        for s in made:
            run(s)
            want.append(state(s))
        for _ in range(5):
            for s in made:
                with torch.cuda.stream(s["stream"]):
                    s["prompt"].zero_(), s["out"].zero_()
                    run(s)
            for s, w in zip(made, want):
                assert all(torch.equal(a, b) for a, b in zip(state(s), w))
        graphs = []
        for s in made:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s["stream"]):
                run(s)
            graphs.append(g)
        for _ in range(5):
            for s, g in zip(made, graphs):
                with torch.cuda.stream(s["stream"]):
                    s["prompt"].zero_(), s["out"].zero_()
                    g.replay()
            for s, w in zip(made, want):
                assert all(torch.equal(a, b) for a, b in zip(state(s), w))
        del graphs
    finally:
        for s in made:
            fd.fd_destroy(s["ctx"])
