"""GPU tests of the prompt attention against the definition in 64 bits.

Tolerance: inputs enter exactly; scores and sums are fp32 (a score of size s is off by at most about 2^-20 s, which at the sizes
here changes a weight by less than 2^-12 of it, as does the exponential); the weights are rounded to bf16 before the product
with V (2^-8, half a step) while their sum is not; the output is rounded to bf16:
|err| <= 2^-8 |ref| + (2^-8 + 2^-10) sum_j p_j |v_j|."""
import numpy as np
import pytest
import torch

import fp8_ref as ref
import paper_2605_20022_b200 as fd

pytestmark = pytest.mark.gpu

PATHS = [fd.FD_ATTN_SIMT, fd.FD_ATTN_AUTO]
CASES = {
    # name: (Hq, Hkv, d, q_lens, kv_lens or None)
    "one token": (32, 8, 128, [1], None),
    "tile edges": (8, 2, 128, [31, 32, 33, 63, 64, 65, 127, 128, 129, 1, 255, 256, 257], None),
    "empty sequences": (8, 2, 128, [0, 5, 0, 130, 0, 0], None),
    "head_dim 64, 8 to a head": (16, 2, 64, [700, 1, 129, 48], None),
    "one head to a head": (4, 4, 128, [300, 127, 128, 1, 512], None),
    "one head to a head, 64": (3, 3, 64, [257, 1000], None),
    "3 to a head": (6, 2, 128, [42, 43, 84, 85, 400], None),
    "5 to a head": (20, 4, 64, [25, 26, 50, 51, 300], None),
    "6 to a head": (12, 2, 128, [21, 42, 43, 130], None),
    "16 to a head": (16, 1, 128, [8, 16, 17, 200], None),
    "100 to a head": (100, 1, 64, [1, 2, 3, 150], None),
    "128 to a head": (128, 1, 128, [1, 2, 130], None),
    "chunks behind earlier keys": (8, 2, 128, [5, 64, 200, 0, 3, 1], [1000, 64, 333, 17, 700, 1]),
    "chunks behind earlier keys, 64": (16, 4, 64, [130, 1, 70], [131, 4000, 513]),
    "rows without a key": (8, 2, 128, [10, 40, 300, 3, 70], [4, 0, 130, 3, 1]),
    "no key at all": (4, 1, 128, [10, 40], [0, 0]),
    # few items: several CTAs share one along the keys
    "one row behind many keys": (8, 2, 128, [1], [5000]),
    "short chunks behind long prefixes": (32, 8, 128, [64, 3], [9000, 2000]),
    "short chunks behind long prefixes, 64": (16, 2, 64, [17, 1, 0, 40], [3000, 700, 5, 100]),
    "a shared item with rows that see no key": (4, 1, 128, [300, 7], [40, 4000]),
    "a shared item, both tiles, one head": (1, 1, 128, [200], [6400]),
    "a shared item among 40 sequences": (2, 1, 64, [3 if b == 7 else 0 for b in range(40)], [4000 if b == 7 else 5 * (b % 3) for b in range(40)]),
    "as many parts as there may be": (4, 1, 64, [33], [20000]),
    "many short": (8, 2, 64, [(5 * b) % 9 for b in range(300)], None),
    "a long one among short ones": (32, 8, 128, [3, 2500, 17, 1, 900, 40], None),
    "more items than SMs": (32, 8, 128, [2100, 1700], None),
    "4096 sequences": (2, 1, 64, [b % 3 for b in range(4096)], None),
}


def _inputs(name, strided, seed=0):
    Hq, Hkv, d, ql, kl = CASES[name]
    kl_ = ql if kl is None else kl
    g = torch.Generator(device="cuda").manual_seed(seed + len(name))
    randn = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    T, Tk = sum(ql), sum(kl_)
    if strided:  # slices of wider rows
        q = randn(max(T, 1), Hq + 3, d)[:T, 1: Hq + 1]
        kv = randn(max(Tk, 1), 2 * Hkv + 1, d)[:Tk]
        k, v = kv[:, :Hkv], kv[:, Hkv + 1:]
    else:
        q, k, v = randn(T, Hq, d), randn(Tk, Hkv, d), randn(Tk, Hkv, d)
    return q, k, v, ql, kl_


def _ctx(Hq, Hkv, d, B, path=fd.FD_ATTN_AUTO, scale=0.0):
    return fd.fd_create(Hq, Hkv, d, 10, B, 1, 4, softmax_scale=scale, attn_path=path)


def _call(ctx, q, k, v, ql, kl, out=None, **kw):
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    fd.fd_attn_prompt(ctx, len(ql), q.shape[0], k.shape[0], q, q.stride(0), k, v, k.stride(0), i32(ql), i32(kl), out, **kw)
    return out


def _check(got, q, k, v, ql, kl, what, scale=None, rows=slice(None)):
    exp, size = ref.prompt(q, k, v, ql, kl, scale)
    got, exp, size = got.double()[rows], exp[rows], size[rows]
    assert torch.isfinite(got).all(), f"{what}: not finite"
    if got.numel():
        worst = ((got - exp).abs() - (2.0 ** -8 * exp.abs() + (2.0 ** -8 + 2.0 ** -10) * size)).max()
        assert worst <= 0, f"{what}: {float(worst):.3g} beyond the tolerance, max |err| {float((got - exp).abs().max()):.3g}"


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("name", sorted(CASES))
def test_prompt_attention_matches_the_definition(name, strided, path):
    q, k, v, ql, kl = _inputs(name, strided)
    Hq, Hkv, d, _, given = CASES[name]
    ctx = _ctx(Hq, Hkv, d, len(ql), path)
    try:
        got = _call(ctx, q, k, v, ql, given)
        again = _call(ctx, q, k, v, ql, kl)
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)
    _check(got, q, k, v, ql, kl, name)
    assert torch.equal(got.view(torch.int16), again.view(torch.int16)), "two runs on the same inputs differ bitwise"


@pytest.mark.parametrize("seed", list(range(24)))
def test_prompt_attention_random_shapes(seed):
    r = np.random.default_rng(seed)
    Hkv = int(r.choice([1, 2, 4, 8]))
    G, d = int(r.choice([1, 2, 3, 4, 5, 7, 8, 16])), int(r.choice([64, 128]))
    B = int(r.integers(1, 9))
    ql = [int(r.choice([0, 1, r.integers(1, 40), r.integers(1, 700)])) for _ in range(B)]
    kl = ql if seed % 2 else [max(0, n + int(r.choice([0, 0, r.integers(0, 300), -1, -r.integers(0, 140)]))) for n in ql]
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((sum(ql), Hkv * G, d), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((sum(kl), Hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    for path in PATHS:
        ctx = _ctx(Hkv * G, Hkv, d, B + seed % 3, path)
        try:
            got = _call(ctx, q, k, v, ql, kl)
            assert fd.fd_last_device_status(ctx) == 0
        finally:
            fd.fd_destroy(ctx)
        _check(got, q, k, v, ql, kl, f"seed {seed} path {path}")


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("Hq,Hkv,d,by", [(8, 2, 128, 3.0), (8, 1, 64, 3.0), (4, 4, 128, -2.0)])
def test_prompt_attention_scores_that_rise_and_fall(Hq, Hkv, d, by, path):
    """K drifts from tile to tile: half of the rows meet a new maximum in every tile and rescale what they have summed."""
    ql = [1500, 130, 700]
    g = torch.Generator(device="cuda").manual_seed(7)
    q = torch.randn((sum(ql), Hq, d), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((sum(ql), Hkv, d), generator=g, device="cuda") for _ in range(2))
    k += by * (torch.arange(sum(ql), device="cuda") // 128)[:, None, None]
    k, v = k.bfloat16(), v.bfloat16()
    ctx = _ctx(Hq, Hkv, d, 3, path)
    try:
        got = _call(ctx, q, k, v, ql, None)
        for _ in range(10):
            assert torch.equal(got, _call(ctx, q, k, v, ql, None)), "two runs on the same inputs differ bitwise"
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)
    _check(got, q, k, v, ql, ql, "drift")


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_sequence_must_not_see(d, path):
    """Neighbours full of infinities and NaN (queries, keys and values) leave a sequence's bits alone; so does a key that is not
    finite in a place the mask hides, for the rows in front of it."""
    ql, Hq, Hkv = [70, 133, 50, 300, 20], 8, 2
    g = torch.Generator(device="cuda").manual_seed(d)
    q = torch.randn((sum(ql), Hq, d), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((sum(ql), Hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    ctx = _ctx(Hq, Hkv, d, 5, path)
    try:
        clean = _call(ctx, q, k, v, ql, None)
        q2, k2, v2 = q.clone(), k.clone(), v.clone()
        for lo, hi in ((0, 70), (203, 253), (553, 573)):
            for i, x in enumerate((q2, k2, v2)):
                x[lo:hi] = torch.tensor([float("nan"), float("inf"), -float("inf")])[i]
                x[lo:hi, :, ::2] = float("nan")
        got = _call(ctx, q2, k2, v2, ql, None)
        for lo, hi in ((70, 203), (253, 553)):
            assert torch.equal(got[lo:hi].view(torch.int16), clean[lo:hi].view(torch.int16))
        k3 = k.clone()
        k3[253 + 200:253 + 300] = float("nan")                  # keys of the fourth sequence from 200 on
        got = _call(ctx, q, k3, v, ql, None)
        assert torch.equal(got[253:453].view(torch.int16), clean[253:453].view(torch.int16))
        for at, value in ((0, float("inf")), (77, float("nan")), (130, -float("inf")), (200, float("inf")), (299, float("nan"))):
            v3 = v.clone()                                      # a value of the fourth sequence, kv-head 1: the rows in front, and the other head
            v3[253 + at, 1, 3:d:7] = value
            got = _call(ctx, q, k, v3, ql, None)
            assert torch.equal(got[:253 + at].view(torch.int16), clean[:253 + at].view(torch.int16))
            assert torch.equal(got[:, :4].view(torch.int16), clean[:, :4].view(torch.int16))
            behind, kept = got[253 + at:553, 4:].float(), torch.ones(d, dtype=torch.bool)
            kept[3:d:7] = False
            assert torch.equal(behind[..., kept], clean[253 + at:553, 4:].float()[..., kept])
            assert torch.isnan(behind[..., 3:d:7]).all() if value != value else (behind[..., 3:d:7] == value).all()
        v3 = v.clone()
        v3[253 + 160, 1, 0], v3[253 + 170, 1, 0] = float("inf"), -float("inf")
        got = _call(ctx, q, k, v3, ql, None)[253:553, 4:, 0].float()
        assert torch.isfinite(got[:160]).all() and (got[160:170] == float("inf")).all() and torch.isnan(got[170:]).all()
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)


@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_finite_in_a_shared_item(d):
    """One item split along the keys: what is not finite in a part every row sees, in the part the mask cuts, and in another sequence."""
    Lq, Lk, Hq, Hkv = 60, 5000, 4, 1
    g = torch.Generator(device="cuda").manual_seed(d)
    q = torch.randn((Lq + 3, Hq, d), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((Lk + 3, Hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    k[Lk:], v[Lk:] = float("nan"), float("inf")
    ctx = _ctx(Hq, Hkv, d, 2)
    try:
        clean = _call(ctx, q, k, v, [Lq, 3], [Lk, 3])[:Lq]
        for at, value in ((0, float("inf")), (2000, float("nan")), (Lk - Lq, float("inf")), (Lk - Lq + 1, -float("inf")), (Lk - 20, float("nan")), (Lk - 1, float("inf"))):
            v3 = v.clone()
            v3[at, 0, 5] = value
            got = _call(ctx, q, k, v3, [Lq, 3], [Lk, 3])[:Lq]
            row = max(0, at - (Lk - Lq))                        # the first row that sees it
            assert torch.equal(got[:row].view(torch.int16), clean[:row].view(torch.int16))
            kept = torch.ones(d, dtype=torch.bool)
            kept[5] = False
            assert torch.equal(got[..., kept], clean[..., kept])
            behind = got[row:, :, 5].float()
            assert torch.isnan(behind).all() if value != value else (behind == value).all()
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("Lq,Lk", [(60, 5000), (9, 90), (300, 300)])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_and_keys_that_are_not_finite(d, Lq, Lk, path):
    """A query that is NaN, or infinite, makes its row NaN and no other, in whole items and in shared ones; a key that is NaN the rows that
    see it."""
    g = torch.Generator(device="cuda").manual_seed(d)
    q = torch.randn((Lq, 4, d), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((Lk, 1, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    ctx = _ctx(4, 1, d, 1, path)
    try:
        clean = _call(ctx, q, k, v, [Lq], [Lk])
        q2 = q.clone()
        q2[3, 1], q2[5, 2, 7] = float("nan"), float("inf")      # (an infinite element: scores of both signs' infinities, inf - inf)
        got = _call(ctx, q2, k, v, [Lq], [Lk])
        gone = torch.zeros((Lq, 4), dtype=torch.bool, device="cuda")
        gone[3, 1] = gone[5, 2] = True
        assert torch.isnan(got[gone]).all() and torch.equal(got[~gone], clean[~gone])
        k2, row = k.clone(), Lq // 2
        k2[Lk - Lq + row, 0, 1] = float("nan")
        got = _call(ctx, q, k2, v, [Lq], [Lk])
        assert torch.isnan(got[row:]).all() and torch.equal(got[:row], clean[:row])
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("size,scale", [(3e4, 1e-6), (1e-4, 300.0), (1.0, 0.5)])
def test_prompt_attention_scales(size, scale, path):
    q, k, v, ql, kl = _inputs("tile edges", False, seed=3)
    q = (q.float() * size).bfloat16()
    ctx = _ctx(8, 2, 128, len(ql), path, scale)
    try:
        got = _call(ctx, q, k, v, ql, None)
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)
    _check(got, q, k, v, ql, kl, "scale", scale)


def test_prompt_attention_many_tiles():
    """Tens of tiles and rounds, every SM busy for several items; sampled rows against 64 bits."""
    ql = [9000, 100, 4500]
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((sum(ql), 8, 128), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((sum(ql), 2, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    ctx = _ctx(8, 2, 128, 3)
    try:
        got = _call(ctx, q, k, v, ql, None)
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)
    _check(got, q, k, v, ql, ql, "many tiles")


def test_prompt_attention_captured_and_on_another_stream():
    Hq, Hkv, d, ql = 8, 2, 128, [100, 260, 3]
    T = sum(ql)
    lens = torch.tensor(ql, dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((T, h, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    out = torch.zeros_like(q)
    ctx = _ctx(Hq, Hkv, d, 3)
    try:
        call = lambda: fd.fd_attn_prompt(ctx, 3, T, T, q, Hq * d, k, v, Hkv * d, lens, None, out)  # noqa: E731
        call()
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
            call()
        for order in ([100, 260, 3], [3, 100, 260], [263, 0, 100]):
            g = torch.Generator().manual_seed(order[0])
            for t in (q, k, v):
                t.copy_(torch.randn(t.shape, generator=g))
            lens.copy_(torch.tensor(order, dtype=torch.int32))
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            _check(out, q, k, v, order, order, "replayed")
            replayed = out.clone()
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                call()
            side.synchronize()
            assert torch.equal(out, replayed)
        assert fd.fd_last_device_status(ctx) == 0
    finally:
        fd.fd_destroy(ctx)


@pytest.mark.parametrize("path", PATHS)
def test_prompt_attention_errors(path):
    Hq, Hkv, d, ql = 8, 2, 128, [40, 0, 90]
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((130, Hq, d), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((130, Hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    ctx = _ctx(Hq, Hkv, d, 3, path)
    try:
        for bad_q, bad_k in (([40, 1, 90], None), ([40, -1, 91], None), ([40, 0, 89], None), ([2 ** 31 - 1, 2 ** 31 - 1, 132], None),
                             (ql, [40, 1, 90]), (ql, [-1, 41, 90])):
            got = _call(ctx, q, k, v, bad_q, bad_k)
            assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_LENGTHS and (got == 0).all()
        got = _call(ctx, q, k, v, ql, None)
        assert fd.fd_last_device_status(ctx) == 0
        _check(got, q, k, v, ql, ql, "after errors")
        n, i, out = fd.fd_launch_count(ctx), torch.tensor(ql, dtype=torch.int32, device="cuda"), torch.zeros_like(q)
        good = [3, 130, 130, q, Hq * d, k, v, Hkv * d, i, None, out]
        for at, value in ((0, 4), (0, -1), (1, -1), (2, -1), (2, 129), (3, None), (3, q.data_ptr() + 2), (4, Hq * d - 8), (4, Hq * d + 4), (4, 2 ** 31),
                          (5, None), (6, k.data_ptr() + 8), (7, 8), (7, Hkv * d + 1), (8, None), (10, None), (10, q), (10, v), (10, q.data_ptr() + 1024),
                          (0, 0)):
            args = good[:at] + [value] + good[at + 1:]
            assert fd.fd_attn_prompt(ctx, *args, raise_on_error=False) == fd.FD_ERR_INVALID_ARG, (at, value)
        assert fd.fd_launch_count(ctx) == n
        assert fd.fd_attn_prompt(ctx, 0, 0, 0, None, Hq * d, None, None, Hkv * d, None, None, None) == fd.FD_OK
        zero = torch.zeros(3, dtype=torch.int32, device="cuda")
        assert fd.fd_attn_prompt(ctx, 3, 0, 0, None, Hq * d, None, None, Hkv * d, zero, None, None) == fd.FD_OK
        assert fd.fd_last_device_status(ctx) == 0
        assert fd.fd_attn_prompt(ctx, 3, 0, 5, None, Hq * d, k, v, Hkv * d, zero, i, None) == fd.FD_OK
        assert fd.fd_last_device_status(ctx) == fd.FD_DEV_BAD_LENGTHS
    finally:
        fd.fd_destroy(ctx)
