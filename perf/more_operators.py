"""Operators on either side of a draft-and-verify decode step, as cases that can be measured: a prompt on its way in, a cache held
in 8 bits, and the pages of a pool when sequences branch and end.

  prompt    causal attention of packed sequences over their own keys, whole prompts or chunks of them behind earlier keys
  append    K and V of the query block into 8-bit pages, and the pages' tokens read back as the values they stand for
  attend    attention of the query blocks [bonus | drafts | mask tokens] over 8-bit pages under the hybrid mask
  fork      samples that have ended give their pages back, new ones branch off the prompts: tables, shared pages, the copies
  compact   the pages in use move to the front of the pool: list of moves, tables, free list, the copies

8-bit pages: e4m3 codes, and one scale for the 16 tokens of a page, a head and K or V: a power of two, 2^-15 to 2^7, the smallest
for which the largest magnitude among the block's tokens is at most 448 times it.  A page holds, for each kv-head, K then V, each
as [16][d] codes followed by the scale in 32 bits and 12 bytes of zeros.  Tokens that a block holds already when others join it
keep their values, re-expressed in the new scale.
"""
import math

import torch

own = False  # True: the framework's calls; False: the plain forms below

PAGE = 16
TAIL = 16  # bytes behind the codes of a block


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a short question: pure latency
        dict(name="prompt b1 17 tokens", op="prompt", batch=1, lo=17, hi=17, plo=0, phi=0, hq=32, hkv=8, d=128, fused=False),
        # admission of a batch: prompts of all lengths, q, k and v where the projection left them
        dict(name="prompt b16 ragged", op="prompt", batch=16, lo=100, hi=4000, plo=0, phi=0, hq=32, hkv=8, d=128, fused=True),
        # a long document
        dict(name="prompt b1 32768", op="prompt", batch=1, lo=32768, hi=32768, plo=0, phi=0, hq=32, hkv=8, d=128, fused=False),
        # sequential mode's batch: a few rows of every sequence join the block at its end
        dict(name="append b64 sequential", op="append", batch=64, lo=1024, hi=4096, cand_lo=1, cand_hi=16, mask=0, blocks=1, hkv=8, d=128),
        # whole prompts of another head layout
        dict(name="append 24 prompts d64", op="append", batch=24, lo=0, hi=100, cand_lo=200, cand_hi=1500, mask=0, blocks=1, hkv=8, d=64),
        # one token of one sequence: ordinary decoding
        dict(name="attend b1 one token", op="attend", batch=1, lo=2048, hi=2048, cand_lo=1, cand_hi=1, mask=0, blocks=1, hq=32, hkv=8, d=128),
        # sequential mode: many sequences, candidates only
        dict(name="attend b64 sequential", op="attend", batch=64, lo=1024, hi=4096, cand_lo=1, cand_hi=16, mask=0, blocks=1,
             hq=32, hkv=8, d=128),
        # long context
        dict(name="attend b16 prefix 32768", op="attend", batch=16, lo=32768, hi=32768, cand_lo=16, cand_hi=16, mask=16, blocks=1,
             hq=32, hkv=8, d=128),
        # one more sample of one prompt
        dict(name="fork 1 sample", op="fork", batch=1, lo=1000, hi=1000, each=1, hkv=8, d=128, fp8=False),
        # several samples of every prompt of a batch
        dict(name="fork 64 prompts 8 samples", op="fork", batch=64, lo=200, hi=8000, each=8, hkv=8, d=128, fp8=True),
        # a small pool of another head layout
        dict(name="compact small pool", op="compact", batch=4, lo=100, hi=900, holes=100, hkv=2, d=64, fp8=False),
        # a pool half empty and scattered after long use
        dict(name="compact half a pool", op="compact", batch=96, lo=200, hi=4000, holes=12000, hkv=8, d=128, fp8=True),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "append", "attend", "attend", "fork", "compact"])
    d = rng.choice([64, 128, 128])
    hkv, g = rng.choice([(1, 4), (2, 4), (2, 8), (4, 4), (8, 4), (8, 1), (2, 6), (4, 5), (1, 16)])
    if op == "prompt":
        batch = _log(rng, 1, 64)
        most = int(min(20_000, math.sqrt(6e8 / batch)))
        hi = _log(rng, 1, most)
        phi = rng.choice([0, 0, _log(rng, 1, max(1, most - hi))])
        return dict(op=op, batch=batch, lo=_log(rng, 1, hi), hi=hi, plo=rng.randrange(0, phi + 1), phi=phi, hq=hkv * g, hkv=hkv, d=d,
                    fused=rng.random() < 0.5)
    if op in ("fork", "compact"):
        batch = _log(rng, 1, 64)
        hi = _log(rng, 1, 100_000 // batch if batch > 12 else 8000)
        case = dict(op=op, batch=batch, lo=_log(rng, 1, hi), hi=hi, hkv=hkv, d=d, fp8=rng.random() < 0.5)
        case.update(dict(each=_log(rng, 1, 8)) if op == "fork" else dict(holes=_log(rng, 1, 8000)))
        return case
    if op == "attend":
        batch = _log(rng, 1, 96)
        top = min(64, max(1, 128 // g))
    else:
        batch = _log(rng, 1, 128)
        top = max(1, min(2000, 8_000 // batch))
    hi_c = _log(rng, 1, top)
    lo_c = _log(rng, 1, hi_c)
    blocks = rng.choice([1, 1, 2, 3]) if lo_c >= 3 and hi_c <= 100 else 1
    mask = blocks * rng.choice([0, 1, 5, 7, 16]) if hi_c <= 100 else 0
    most = 32000 if op != "attend" else max(16, min(32000, 400_000 // batch))
    hi = _log(rng, 1, most)
    lo = rng.randrange(0, hi + 1)
    case = dict(op=op, batch=batch, lo=lo, hi=hi, cand_lo=lo_c, cand_hi=hi_c, mask=mask, blocks=blocks, hkv=hkv, d=d)
    if op == "attend":
        case["hq"] = hkv * g
    return case


def _whole(case, lo, hi, salt):
    """Lengths of the sequences: the same for every seed, so that a case's work is a property of the case."""
    g = torch.Generator().manual_seed(20022 + salt + case["batch"] * 7 + case["hi"])
    return torch.randint(lo, hi + 1, (case["batch"],), generator=g)


def _lengths(case):
    """(prefix, candidates) of every sequence (prompt: earlier keys, query rows)."""
    if case["op"] == "prompt":
        return _whole(case, case["plo"], case["phi"], 1), _whole(case, case["lo"], case["hi"], 2)
    return _whole(case, case["lo"], case["hi"], 3), _whole(case, case["cand_lo"], case["cand_hi"], 4)


def _page_bytes(case):
    return 2 * case["hkv"] * (PAGE * case["d"] + TAIL if case["fp8"] else 2 * PAGE * case["d"])


def _moves(case):
    """compact: how many pages move for seed 0 (the pool is scattered at random: other seeds differ a little)."""
    used = int(((_whole(case, case["lo"], case["hi"], 3) + PAGE - 1) // PAGE).sum())
    return used * case["holes"] // (used + case["holes"])


def work(case):
    op, hkv, d = case["op"], case["hkv"], case["d"]
    if op == "compact":
        n = _whole(case, case["lo"], case["hi"], 3)
        entries = int(((n + PAGE - 1) // PAGE).sum())
        return {"bytes": 2 * _moves(case) * _page_bytes(case) + 8 * entries + 8 * case["holes"], "flops": 0}
    if op == "fork":
        n = _whole(case, case["lo"], case["hi"], 3)
        pages = int(((n + PAGE - 1) // PAGE).sum()) * case["each"]
        return {"bytes": 2 * int((n % PAGE > 0).sum()) * case["each"] * _page_bytes(case) + 16 * pages, "flops": 0}
    n, c = _lengths(case)
    if op == "prompt":
        t, kv = int(c.sum()), int((n + c).sum())
        pairs = int((c * n + c * (c + 1) // 2).sum())
        return {"bytes": 4 * t * case["hq"] * d + 4 * kv * hkv * d, "flops": 4 * d * case["hq"] * pairs}
    rows, kv = c + case["mask"], n + c + case["mask"]
    t = int(rows.sum())
    if op == "append":  # in bf16, out in 8 bits; the last pages back: in 8 bits, out bf16
        held = int((rows + n % PAGE).sum())
        return {"bytes": 2 * hkv * d * (t * 3 + held * 3), "flops": 0}
    return {"bytes": int(kv.sum()) * 2 * hkv * (d + 1) + 4 * t * case["hq"] * d, "flops": 4 * d * case["hq"] * int((rows * kv).sum())}


# ------------------------------------------------------------------------------------------------ inputs
def _i32(x):
    return x.to(device="cuda", dtype=torch.int32)


def _random_pool(pages, case, g):
    """A pool of pages with N(0, 1) values in its format."""
    hkv, d = case["hkv"], case["d"]
    if not case.get("fp8", True):
        return torch.randn((pages, 2, hkv, PAGE, d), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    cache = torch.zeros((pages, hkv, 2, PAGE * d + TAIL), dtype=torch.uint8, device="cuda")
    for p in range(0, pages, 4096):
        q = min(pages, p + 4096)
        x = torch.randn((q - p, hkv, 2, PAGE, d), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16).float()
        codes, scale = _quantise(x)
        _codes(cache, d)[p:q] = codes
        _scales(cache, d)[p:q] = scale
    return cache


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    gc = torch.Generator().manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    op, b, hkv, d = case["op"], case["batch"], case["hkv"], case["d"]
    if op == "prompt":
        n, c = _lengths(case)
        t, tkv, hq = int(c.sum()), int((n + c).sum()), case["hq"]
        s = dict(case=case, total=t, total_kv=tkv, q_lens=_i32(c), kv_lens=_i32(n + c))
        if case["fused"] and case["phi"] == 0:
            x = randn(t, hq + 2 * hkv, d)
            s.update(q=x[:, :hq], k=x[:, hq: hq + hkv], v=x[:, hq + hkv:])
        elif case["fused"]:
            x = randn(tkv, 2 * hkv, d)
            s.update(q=randn(t, hq, d), k=x[:, :hkv], v=x[:, hkv:])
        else:
            s.update(q=randn(t, hq, d), k=randn(tkv, hkv, d), v=randn(tkv, hkv, d))
        s["out"] = torch.zeros((t, hq, d), dtype=torch.bfloat16, device="cuda")
        return s
    if op in ("fork", "compact"):
        return _prepare_pages(case, g, gc)
    n, c = _lengths(case)
    rows, kv = c + case["mask"], n + c + case["mask"]
    t = int(rows.sum())
    need = (kv + PAGE - 1) // PAGE
    width, pool = int(need.max()) + 2, int(need.sum()) + 64
    ids = torch.randperm(pool, generator=gc)
    col = torch.arange(width)[None, :]
    at = torch.cumsum(need, 0)[:, None] - need[:, None] + col
    table = torch.where(col < need[:, None], ids[at.clamp(max=pool - 1)], torch.full_like(at, -1))
    s = dict(case=case, total=t, num_pages=pool, page_table=_i32(table), prefix_lens=_i32(n), q_lens=_i32(rows),
             cache=_random_pool(pool, case, g))
    if op == "attend":
        s.update(n_mask=_i32(torch.full((b,), case["mask"])), n_blocks=_i32(torch.full((b,), case["blocks"])), q=randn(t, case["hq"], d))
        s["out"] = torch.zeros_like(s["q"])
        return s
    # a block's newcomers are of another magnitude now and then, so that tokens it holds change their scale
    loud = 2.0 ** torch.randint(-2, 3, (t, hkv, 1), generator=g, device="cuda")
    s.update(k=(randn(t, hkv, d) * loud).to(torch.bfloat16), v=(randn(t, hkv, d) * loud).to(torch.bfloat16))
    # what is read back: the new rows and the tokens in front of them in their first page
    held = int((rows + n % PAGE).sum())
    s.update(read_from=_i32(n - n % PAGE), read_lens=_i32(rows + n % PAGE), held=held)
    s.update(k_back=torch.zeros((held, hkv, d), dtype=torch.bfloat16, device="cuda"), v_back=torch.zeros((held, hkv, d), dtype=torch.bfloat16, device="cuda"))
    return s


def _prepare_pages(case, g, gc):
    b = case["batch"]
    n = _whole(case, case["lo"], case["hi"], 3)
    need = (n + PAGE - 1) // PAGE
    full = n // PAGE
    width = int(need.max()) + 2
    col = torch.arange(width)[None, :]
    if case["op"] == "compact":
        used = int(need.sum())
        pool = used + case["holes"]
        ids = torch.randperm(pool, generator=gc)
        at = torch.cumsum(need, 0)[:, None] - need[:, None] + col
        table = torch.where(col < need[:, None], ids[at.clamp(max=pool - 1)], torch.full_like(at, -1))
        free = torch.full((pool,), -1)
        free[: case["holes"]] = ids[used:]
        shared = torch.zeros(pool, dtype=torch.int64)
        shared[ids[:used]] = torch.randint(0, 3, (used,), generator=gc)
        s = dict(case=case, num_pages=pool, table0=_i32(table), free0=_i32(free), shared0=_i32(shared), n_free=_i32(torch.tensor([case["holes"]])))
        s.update(page_table=s["table0"].clone(), free_pages=s["free0"].clone(), shared=s["shared0"].clone(), most=min(used, case["holes"]))
        s.update(page_map=_i32(torch.zeros(pool)), copy_src=_i32(torch.full((s["most"],), -1)), copy_dst=_i32(torch.full((s["most"],), -1)),
                 n_copies=_i32(torch.zeros(1)))
        s["cache"] = _random_pool(pool, case, g)
        return s
    # prompts in the first rows of the table, their samples behind them; sample i belongs to prompt i % b to begin with
    each, kids = case["each"], b * case["each"]
    parent = torch.arange(kids) % b
    partial = n % PAGE > 0
    tails = int(partial[parent].sum())
    pool = int(need.sum()) + tails + 64
    ids = torch.randperm(pool, generator=gc)
    at = torch.cumsum(need, 0)[:, None] - need[:, None] + col
    table = torch.where(col < need[:, None], ids[at.clamp(max=pool - 1)], torch.full_like(at, -1))
    first = int(need.sum())
    kid = torch.where(col < full[parent][:, None], table[parent], torch.full((kids, width), -1))
    place = torch.cumsum(partial[parent].long(), 0) - 1
    kid[partial[parent], full[parent][partial[parent]]] = ids[first + place[partial[parent]]]
    shared = torch.zeros(pool, dtype=torch.int64)
    shared[table[col < full[:, None]]] = each
    free = torch.full((pool,), -1)
    free[: pool - first - tails] = ids[first + tails:]
    turn = torch.randperm(kids, generator=gc)  # which row of the table becomes which prompt's sample next
    return dict(case=case, num_pages=pool, rows=b + kids, page_table=_i32(torch.cat([table, kid])), prefix_lens=_i32(torch.cat([n, n[parent]])),
                shared=_i32(shared), free_pages=_i32(free), n_free=_i32(torch.tensor([pool - first - tails])), ended=_i32(b + torch.arange(kids)),
                parents=_i32(parent), children=_i32(b + turn), copy_src=_i32(torch.full((kids,), -1)), copy_dst=_i32(torch.full((kids,), -1)),
                cache=_random_pool(pool, case, g))


# ------------------------------------------------------------------------------------------------ plain forms
def _codes(cache, d):
    """View of the codes of 8-bit pages: [pages, Hkv, 2, 16, d]."""
    return cache[..., : PAGE * d].unflatten(-1, (PAGE, d))


def _scales(cache, d):
    """View of their scales: [pages, Hkv, 2], 32 bits."""
    return cache[..., PAGE * d: PAGE * d + 4].view(torch.float32)[..., 0]


def _quantise(x, valid=None):
    """(codes, scales) of blocks [..., 16, d] in 32 bits.  `valid`: which tokens count for the scale."""
    a = x.abs() if valid is None else torch.where(valid, x.abs(), torch.zeros_like(x))
    mant, ex = torch.frexp(a.amax((-1, -2)))
    e = torch.where(mant > 0.875, ex - 8, ex - 9)  # 448 is 0.875 times 2^9
    e = torch.where(mant > 0, e, torch.full_like(e, -15)).clamp(-15, 7)
    scale = ((e + 127) << 23).view(torch.float32)  # (2 to the e; a power taken on the GPU may be off in its last place)
    codes = (x / scale[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), scale


def _plain_prompt(s):
    c = s["case"]
    hkv, d, grp, b = c["hkv"], c["d"], c["hq"] // c["hkv"], c["batch"]
    rows, kv = s["q_lens"].long(), s["kv_lens"].long()
    n, r = _lengths(c)
    most, top = int(r.max()), int((n + r).max())
    row0, kv0 = torch.cumsum(rows, 0) - rows, torch.cumsum(kv, 0) - kv
    key = torch.arange(top, device="cuda")
    at = (kv0[:, None] + key).clamp(max=s["total_kv"] - 1)
    k, v = (s[x].float()[at].permute(0, 2, 1, 3) for x in ("k", "v"))  # [B, Hkv, keys, d]
    step = max(1, min(most, int(4e9 // (4 * b * c["hq"] * top))))
    out = torch.zeros((s["total"] + 1, c["hq"], d), dtype=torch.bfloat16, device="cuda")
    for lo in range(0, most, step):  # as many rows at a time as memory allows
        i = torch.arange(lo, min(most, lo + step), device="cuda")
        take = torch.where(i < rows[:, None], row0[:, None] + i, torch.full_like(rows[:, None], s["total"]))
        q = s["q"].float()[take.clamp(max=s["total"] - 1)].unflatten(2, (hkv, grp)).permute(0, 2, 3, 1, 4).flatten(2, 3)
        score = ((q @ k.transpose(2, 3)) * (1.0 / math.sqrt(d))).unflatten(2, (grp, -1))
        sees = key <= (kv - rows)[:, None, None] + i[None, :, None]
        score = score.masked_fill_(~sees[:, None, None], float("-inf"))
        score -= score.amax(-1, keepdim=True).clamp(min=-1e30)
        p = score.exp_()
        total = p.sum(-1, keepdim=True)
        o = (p.flatten(2, 3) @ v).unflatten(2, (grp, -1)) / total.clamp(min=1e-30)
        out[take] = o.permute(0, 3, 1, 2, 4).flatten(2, 3).to(torch.bfloat16)
    return out[: s["total"]]


def _plain_append(s):
    c = s["case"]
    d, n, rows = c["d"], s["prefix_lens"].long(), s["q_lens"].long()
    codes, scales = _codes(s["cache"], d), _scales(s["cache"], d)
    pn, pr = _lengths(c)
    blocks = int(((pn + pr + c["mask"] + PAGE - 1) // PAGE - pn // PAGE).sum())
    count = torch.where(rows > 0, (n + rows + PAGE - 1) // PAGE - n // PAGE, torch.zeros_like(n))
    seq = torch.repeat_interleave(torch.arange(c["batch"], device="cuda"), count, output_size=blocks)
    col = n[seq] // PAGE + torch.arange(blocks, device="cuda") - (torch.cumsum(count, 0) - count)[seq]
    page = s["page_table"][seq, col].long()
    pos = col[:, None] * PAGE + torch.arange(PAGE, device="cuda")
    new = (pos >= n[seq][:, None]) & (pos < (n + rows)[seq][:, None])
    valid = pos < (n + rows)[seq][:, None]
    take = ((torch.cumsum(rows, 0) - rows - n)[seq][:, None] + pos).clamp(0, s["total"] - 1)
    here = codes[page].view(torch.float8_e4m3fn).float() * scales[page][..., None, None]  # [blocks, Hkv, 2, 16, d]
    fresh = torch.stack([s["k"].float()[take], s["v"].float()[take]], 3).permute(0, 2, 3, 1, 4)
    x = torch.where(new[:, None, None, :, None], fresh, here)
    x = torch.where(valid[:, None, None, :, None], x, torch.zeros_like(x))
    got, by = _quantise(x)
    codes[page] = torch.where(valid[:, None, None, :, None], got, codes[page])
    scales[page] = by
    # the tokens of [read_from, read_from + read_lens) back
    start, lens = s["read_from"].long(), s["read_lens"].long()
    seq = torch.repeat_interleave(torch.arange(c["batch"], device="cuda"), lens, output_size=s["held"])
    j = start[seq] + torch.arange(s["held"], device="cuda") - (torch.cumsum(lens, 0) - lens)[seq]
    page = s["page_table"][seq, j // PAGE].long()
    back = codes[page, :, :, j % PAGE].view(torch.float8_e4m3fn).float() * scales[page][..., None]
    return [back[:, :, 0].to(torch.bfloat16), back[:, :, 1].to(torch.bfloat16)]


def _plain_attend(s):
    c = s["case"]
    hkv, d, grp = c["hkv"], c["d"], c["hq"] // c["hkv"]
    n, rows, b = s["prefix_lens"].long(), s["q_lens"].long(), c["batch"]
    most = int(_lengths(c)[1].max()) + c["mask"]
    top = s["page_table"].shape[1] - 2
    pages = s["page_table"][:, :top].long().clamp(min=0)

    def dense(which):  # [B, Hkv, tokens, d]
        x = _codes(s["cache"], d)[:, :, which][pages].view(torch.float8_e4m3fn).float() * _scales(s["cache"], d)[:, :, which][pages][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(b, hkv, top * PAGE, d)

    start = torch.cumsum(rows, 0) - rows
    i = torch.arange(most, device="cuda")
    real = i < rows[:, None]
    take = (start[:, None] + i).clamp(max=s["total"] - 1)
    q = s["q"].float()[take].reshape(b, most, hkv, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, grp * most, d)
    score = (q @ dense(0).transpose(2, 3)).reshape(b, hkv, grp, most, top * PAGE) * (1.0 / math.sqrt(d))
    key = torch.arange(top * PAGE, device="cuda") - n[:, None, None]  # [B, 1, tokens]: place in the query block
    cand = (rows - c["mask"])[:, None, None]
    ii = i[None, :, None]
    each = max(1, c["mask"] // c["blocks"])
    g = torch.div(ii - cand, each, rounding_mode="floor")
    sees = torch.where(ii < cand, key <= ii,
                       torch.where(key < cand, key <= cand - c["blocks"] + g, torch.div(key - cand, each, rounding_mode="floor") == g))
    sees = (sees | (key < 0)) & (key < rows[:, None, None])
    score = score.masked_fill_(~sees[:, None, None], float("-inf"))
    score = score - score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(score)
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(b, hkv, grp * most, -1) @ dense(1)).reshape(b, hkv, grp, most, d) / total.clamp(min=1e-30)
    return o.permute(0, 3, 1, 2, 4).reshape(b, most, c["hq"], d)[real].to(torch.bfloat16)


def _plain_free(s):
    """Sequences of `ended` give their pages back: the last one's last page first; a page goes to the list with its last owner."""
    seqs, pool, table = s["ended"].long(), s["num_pages"], s["page_table"]
    n = s["prefix_lens"].long()[seqs]
    col = torch.arange(table.shape[1], device="cuda")
    held = col < ((n + PAGE - 1) // PAGE)[:, None]
    page = torch.where(held, table[seqs].long(), torch.full((1, 1), pool, device="cuda")).flatten()
    e = torch.arange(page.numel(), device="cuda")
    owners = torch.zeros(pool + 1, dtype=torch.int64, device="cuda").scatter_add_(0, page, torch.ones_like(page))[:pool]
    left = s["shared"].long() - owners
    first = torch.full((pool + 1,), page.numel(), device="cuda").scatter_reduce_(0, page, e, "amin")
    gone = torch.cat([left < 0, torch.zeros(1, dtype=torch.bool, device="cuda")])
    push = gone[page] & (first[page] == e) & (page < pool)
    rank = push.flip(0).long().cumsum(0).flip(0) - 1
    at = torch.where(push, s["n_free"].long() + rank, torch.full_like(rank, pool))
    s["free_pages"].copy_(torch.cat([s["free_pages"], s["free_pages"][:1]]).scatter_(0, at, page.to(torch.int32))[:pool])
    s["n_free"] += push.sum().to(torch.int32)
    s["shared"].copy_(left.clamp(min=0))
    table[seqs] = torch.where(held, torch.full_like(table[seqs], -1), table[seqs])
    s["prefix_lens"][seqs] = 0


def _plain_fork(s):
    """The samples in `children` branch off `parents`: whole pages are shared, the rest of the prefix gets a page of its own."""
    parents, children, pool, table = s["parents"].long(), s["children"].long(), s["num_pages"], s["page_table"]
    n = s["prefix_lens"].long()[parents]
    full, part = n // PAGE, n % PAGE > 0
    rank = part.long().cumsum(0) - 1
    page = torch.where(part, s["free_pages"][(s["n_free"].long() - 1 - rank).clamp(min=0)], torch.full_like(parents, -1, dtype=torch.int32))
    col = torch.arange(table.shape[1], device="cuda")
    mine = table[parents]
    whole = col < full[:, None]
    s["copy_src"].copy_(torch.where(part, mine.gather(1, full.clamp(max=table.shape[1] - 1)[:, None])[:, 0], torch.full_like(page, -1)))
    s["copy_dst"].copy_(page)
    table[children] = torch.where(whole, mine, torch.where(col == full[:, None], page[:, None], torch.full_like(mine, -1)))
    at = torch.where(whole, mine.long(), torch.full((1, 1), pool, device="cuda")).flatten()
    s["shared"] += torch.zeros(pool + 1, dtype=torch.int32, device="cuda").scatter_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:pool]
    s["prefix_lens"][children] = n.to(torch.int32)
    s["n_free"] -= part.sum().to(torch.int32)


def _plain_compact(s):
    pool, used = s["num_pages"], s["num_pages"] - s["n_free"].long()
    i = torch.arange(pool, device="cuda")
    free = torch.where(i < s["n_free"], s["free_pages"].long(), torch.full_like(i, pool))
    live = torch.ones(pool + 1, dtype=torch.bool, device="cuda").scatter_(0, free, torch.zeros_like(free, dtype=torch.bool))[:pool]
    hole, mover = ~live & (i < used), live & (i >= used)
    most = s["most"]
    place = lambda m: torch.full((most + 1,), -1, device="cuda").scatter_(0, torch.where(m, m.long().cumsum(0) - 1, torch.full_like(i, most)), i)[:most]  # noqa: E731
    s["copy_dst"].copy_(place(hole))
    s["copy_src"].copy_(place(mover))
    s["n_copies"].copy_(mover.sum().to(torch.int32))
    to = s["copy_dst"].long()[(mover.long().cumsum(0) - 1).clamp(0, most - 1)]
    page_map = torch.where(live, torch.where(mover, to, i), torch.full_like(i, -1))
    s["page_map"].copy_(page_map)
    table = s["page_table"]
    table.copy_(torch.where(table >= 0, page_map[table.long().clamp(min=0)].to(torch.int32), table))
    moved = torch.zeros(pool + 1, dtype=torch.int32, device="cuda").scatter_(0, torch.where(live, page_map, torch.full_like(i, pool)), s["shared"])
    s["shared"].copy_(moved[:pool])
    s["free_pages"].copy_(torch.where(i < s["n_free"], pool - 1 - i, s["free_pages"].long()))


def _plain_copies(s):
    ok = s["copy_dst"] >= 0
    s["cache"][s["copy_dst"][ok].long()] = s["cache"][s["copy_src"][ok].long()]


# ------------------------------------------------------------------------------------------------ the pass
_contexts = {}


def _context(s):
    """The library's handle, one for each shape, as a program keeps it."""
    import paper_2605_20022_b200 as fd

    c = s["case"]
    width = s["page_table"].shape[1] if "page_table" in s else 64
    key = (c.get("hq", c["hkv"]), c["hkv"], c["d"], s.get("rows", c["batch"]), c.get("cand_hi", 1) + PAGE + c.get("mask", 0), width)
    if key not in _contexts:
        _contexts[key] = fd.fd_create(key[0], key[1], key[2], 1, key[3], key[4], key[5])
    return fd, _contexts[key]


def run(s):
    c = s["case"]
    op = c["op"]
    if op == "compact":  # the pool as it is found: the pass before has compacted these
        s["page_table"].copy_(s["table0"])
        s["free_pages"].copy_(s["free0"])
        s["shared"].copy_(s["shared0"])
    if own:
        fd, ctx = _context(s)
        fmt = fd.FD_KV_FP8 if c.get("fp8", True) else fd.FD_KV_BF16
        if op == "prompt":
            fd.fd_attn_prompt(ctx, c["batch"], s["total"], s["total_kv"], s["q"], s["q"].stride(0), s["k"], s["v"], s["k"].stride(0), s["q_lens"],
                              s["kv_lens"] if c["phi"] else None, s["out"])
            return [s["out"]]
        if op == "append":
            fd.fd_kv_append_fp8(ctx, c["batch"], s["total"], s["k"], s["v"], s["cache"], s["num_pages"], s["page_table"], s["prefix_lens"],
                                s["q_lens"])
            fd.fd_kv_read_fp8(ctx, c["batch"], s["held"], s["cache"], s["num_pages"], s["page_table"], s["read_from"], s["read_lens"],
                              s["k_back"], s["v_back"])
            return [s["k_back"], s["v_back"]]
        if op == "attend":
            fd.fd_attn_draft_verify_fp8(ctx, c["batch"], s["total"], s["q"], s["cache"], s["num_pages"], s["page_table"], s["prefix_lens"],
                                        s["q_lens"], s["n_mask"], s["n_blocks"], s["out"])
            return [s["out"]]
        if op == "fork":
            kids = s["ended"].shape[0]
            fd.fd_kv_free(ctx, kids, s["ended"], s["rows"], s["page_table"], s["prefix_lens"], s["shared"], s["free_pages"], s["n_free"],
                          s["n_free"], s["num_pages"])
            fd.fd_kv_fork(ctx, kids, s["parents"], s["children"], s["rows"], s["page_table"], s["prefix_lens"], s["shared"], s["free_pages"],
                          s["n_free"], s["n_free"], s["num_pages"], s["copy_src"], s["copy_dst"])
            fd.fd_kv_copy_pages(ctx, kids, None, s["copy_src"], s["copy_dst"], s["cache"], s["num_pages"], fmt)
        else:
            fd.fd_kv_compact(ctx, c["batch"], s["page_table"], s["shared"], s["free_pages"], s["n_free"], s["num_pages"], s["page_map"],
                             s["most"], s["copy_src"], s["copy_dst"], s["n_copies"])
            fd.fd_kv_copy_pages(ctx, s["most"], s["n_copies"], s["copy_src"], s["copy_dst"], s["cache"], s["num_pages"], fmt)
    elif op == "prompt":
        return [_plain_prompt(s)]
    elif op == "append":
        return _plain_append(s)
    elif op == "attend":
        return [_plain_attend(s)]
    elif op == "fork":
        _plain_free(s)
        _plain_fork(s)
        _plain_copies(s)
    else:
        _plain_compact(s)
        _plain_copies(s)
    if op == "fork":
        return [s["page_table"], s["prefix_lens"], s["shared"], s["free_pages"], s["n_free"], s["copy_src"], s["copy_dst"], s["cache"]]
    return [s["page_table"], s["shared"], s["free_pages"], s["page_map"], s["n_copies"], s["cache"]]


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def _nearest(x, grid):
    """Index of the value of an ascending grid nearest to x >= 0, of two the one with the even index."""
    hi = torch.searchsorted(grid, x).clamp(1, grid.numel() - 1)
    lo = hi - 1
    dl, dh = x - grid[lo], grid[hi] - x
    return torch.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)


def _e4m3_values(device):
    return torch.tensor([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127],
                        dtype=torch.float64, device=device)


def _exact_values(raw, d):
    """8-bit pages [..., 16 * d + 16] as 64-bit values [..., 16, d]."""
    code = raw[..., : PAGE * d].long()
    val = _e4m3_values(raw.device)[(code % 128).clamp(max=126)]
    val = torch.where(code >= 128, -val, val).unflatten(-1, (PAGE, d))
    bits = raw[..., PAGE * d + 2].long() // 128 + 2 * (raw[..., PAGE * d + 3].long() % 128)  # the exponent field of the scale
    return val * torch.tensor([2.0 ** (e - 127) for e in range(256)], dtype=torch.float64, device=raw.device)[bits][..., None, None]


def _exact_held(x):
    """What the 64-bit values of blocks [..., 16, d] stand for once they are held in 8 bits."""
    grid = _e4m3_values(x.device)
    powers = torch.tensor([2.0 ** e for e in range(-15, 8)], dtype=torch.float64, device=x.device)
    scale = powers[torch.searchsorted(448 * powers, x.abs().amax((-1, -2))).clamp(max=22)][..., None, None]
    return torch.sign(x) * grid[_nearest((x.abs() / scale).clamp(max=448), grid)] * scale


def exact(case, seed):
    op, hkv, d = case["op"], case["hkv"], case["d"]
    if op in ("fork", "compact"):
        return None
    s = prepare(case, seed)
    if op == "prompt":
        hq, rows, kv = case["hq"], s["q_lens"].tolist(), s["kv_lens"].tolist()
        out, grp, r0, k0 = torch.zeros((s["total"], hq, d), dtype=torch.float64, device="cuda"), hq // hkv, 0, 0
        for lq, lk in zip(rows, kv):
            for h in range(hkv):
                k, v = (s[x][k0: k0 + lk, h].double() for x in ("k", "v"))
                for lo in range(0, lq, 2048):
                    hi = min(lq, lo + 2048)
                    seen = lk - lq + hi
                    x = s["q"][r0 + lo: r0 + hi, h * grp:(h + 1) * grp].double().transpose(0, 1)
                    w = (x @ k[:seen].T) / math.sqrt(d)
                    later = torch.ones((hi - lo, seen), dtype=torch.bool, device="cuda").triu(lk - lq + lo + 1)
                    out[r0 + lo: r0 + hi, h * grp:(h + 1) * grp] = (torch.softmax(w.masked_fill_(later, float("-inf")), -1) @ v[:seen]).transpose(0, 1)
            r0, k0 = r0 + lq, k0 + lk
        return [out]
    n, rows = s["prefix_lens"].tolist(), s["q_lens"].tolist()
    row0 = 0
    if op == "append":
        got = [[], []]
        for b, lq in enumerate(rows):
            start = n[b] - n[b] % PAGE
            pages = s["page_table"][b, start // PAGE: -(-(n[b] + lq) // PAGE)].long()
            for which, x in ((0, s["k"]), (1, s["v"])):
                held = _exact_values(s["cache"][pages][:, :, which], d).permute(0, 2, 1, 3).reshape(-1, hkv, d)
                held[n[b] - start: n[b] - start + lq] = x[row0: row0 + lq].double()
                held[n[b] - start + lq:] = 0
                block = held.reshape(-1, PAGE, hkv, d).transpose(1, 2)
                got[which].append(_exact_held(block).transpose(1, 2).reshape(-1, hkv, d)[: n[b] - start + lq])
            row0 += lq
        return [torch.cat(x) for x in got]
    hq, grp = case["hq"], case["hq"] // hkv
    out = torch.zeros((s["total"], hq, d), dtype=torch.float64, device="cuda")
    for b, lq in enumerate(rows):
        total = n[b] + lq
        val = _exact_values(s["cache"][s["page_table"][b, : -(-total // PAGE)].long()], d)
        k, v = (val[:, :, w].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :total] for w in (0, 1))
        visible = torch.zeros((lq, total), dtype=torch.bool, device="cuda")
        visible[:, : n[b]] = True
        cand = lq - case["mask"]
        visible[:cand, n[b]: n[b] + cand] = torch.ones((cand, cand), device="cuda").tril().bool()
        each = case["mask"] // case["blocks"]
        for g in range(case["blocks"] if each else 0):
            lo = cand + g * each
            visible[lo: lo + each, n[b]: n[b] + cand - case["blocks"] + g + 1] = True
            visible[lo: lo + each, n[b] + lo: n[b] + lo + each] = True
        for h in range(hkv):
            x = s["q"][row0: row0 + lq, h * grp:(h + 1) * grp].double()
            w = torch.softmax((x.reshape(-1, d) @ k[h].T / math.sqrt(d)).reshape(lq, grp, total).masked_fill(~visible[:, None], float("-inf")), -1)
            out[row0: row0 + lq, h * grp:(h + 1) * grp] = (w.reshape(-1, total) @ v[h]).reshape(lq, grp, d)
        row0 += lq
    return [out]
