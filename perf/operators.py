"""Operators around a draft-and-verify decode step on a paged KV cache, as cases that can be measured.

Four operators, in the order in which a layer of a step uses them:

  reserve   pages for the query blocks out of a free list, and for every query row its cache slot and its position
  rope      norm of every query and key head, rotation by the position, K and V into the cache (bf16 pages or 4-bit pages)
  append    K and V of the query block into 4-bit pages, and read back out of them as the values they stand for
  attend    attention of the query blocks [bonus | drafts | mask tokens] over 4-bit pages under the hybrid mask

4-bit pages: codes of e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, the even element of a byte in its low half), and
one e4m3 scale for every 16 consecutive elements of a head's row; a number per call scales all of K, another all of V.
A page of 16 tokens holds, for each kv-head, K then V, each as [16][d / 2] codes followed by [16][d / 16] scales.
"""
import math

import torch

own = False  # True: the framework's calls; False: the plain forms below

PAGE = 16
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one sequence asks for its query block of bonus + 15 drafts + 16 mask tokens: pure latency
        dict(name="reserve b1 block32", op="reserve", batch=1, lo=2048, hi=2048, cand_lo=16, cand_hi=16, mask=16, blocks=1),
        # a serving batch in which every sequence prepares several branches
        dict(name="reserve b64 4 branches", op="reserve", batch=64, lo=1, hi=8192, cand_lo=4, cand_hi=16, mask=28, blocks=4),
        # admission of many prompts at once: their pages and the slots of all their tokens
        dict(name="reserve b256 prompts", op="reserve", batch=256, lo=0, hi=0, cand_lo=100, cand_hi=4096, mask=0, blocks=1),
        # one sequence's query block between projection and attention, bf16 pages
        dict(name="rope b1 block32 bf16", op="rope", batch=1, lo=2048, hi=2048, cand_lo=16, cand_hi=16, mask=16, blocks=1,
             hq=32, hkv=8, d=128, rot=128, adjacent=False, fp4=False),
        # the tokens of a batch of prompts in one call, 4-bit pages
        dict(name="rope 16 prompts fp4", op="rope", batch=16, lo=0, hi=700, cand_lo=300, cand_hi=900, mask=0, blocks=1,
             hq=32, hkv=8, d=128, rot=128, adjacent=False, fp4=True),
        # sequential mode's batch: a few rows of every sequence into its pages
        dict(name="append b64 sequential", op="append", batch=64, lo=1024, hi=4096, cand_lo=1, cand_hi=16, mask=0, blocks=1,
             hkv=8, d=128),
        # whole prompts of another head layout
        dict(name="append 24 prompts d64", op="append", batch=24, lo=0, hi=100, cand_lo=200, cand_hi=1500, mask=0, blocks=1,
             hkv=8, d=64),
        # one token of one sequence: ordinary decoding
        dict(name="attend b1 one token", op="attend", batch=1, lo=2048, hi=2048, cand_lo=1, cand_hi=1, mask=0, blocks=1,
             hq=32, hkv=8, d=128),
        # parallel mode: ragged prefixes, confidence-truncated candidates, 16 mask tokens
        dict(name="attend b8 parallel", op="attend", batch=8, lo=512, hi=8192, cand_lo=4, cand_hi=16, mask=16, blocks=1,
             hq=32, hkv=8, d=128),
        # sequential mode: many sequences, candidates only
        dict(name="attend b64 sequential", op="attend", batch=64, lo=1024, hi=4096, cand_lo=1, cand_hi=16, mask=0, blocks=1,
             hq=32, hkv=8, d=128),
        # long context
        dict(name="attend b16 prefix 32768", op="attend", batch=16, lo=32768, hi=32768, cand_lo=16, cand_hi=16, mask=16, blocks=1,
             hq=32, hkv=8, d=128),
        # every hypothesis prepared: 17 branches of 16 tokens, query blocks of 289 rows, head dimension 64
        dict(name="attend b4 all hypotheses d64", op="attend", batch=4, lo=512, hi=8192, cand_lo=17, cand_hi=17, mask=272, blocks=17,
             hq=16, hkv=2, d=64),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["reserve", "rope", "append", "attend", "attend"])
    d = rng.choice([64, 128, 128])
    hkv, g = rng.choice([(1, 4), (2, 4), (2, 8), (4, 4), (8, 4), (8, 1), (2, 6), (4, 5), (1, 16)])
    if op == "reserve":
        batch = _log(rng, 1, 1024)
        top = max(1, min(4096, 500_000 // batch))
    elif op == "attend":
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
    case = dict(op=op, batch=batch, lo=lo, hi=hi, cand_lo=lo_c, cand_hi=hi_c, mask=mask, blocks=blocks)
    if op == "rope":
        rot = rng.choice([d, d, d // 2])
        case.update(hq=hkv * g, hkv=hkv, d=d, rot=rot, adjacent=rng.random() < 0.3, fp4=rng.random() < 0.6)
    elif op == "append":
        case.update(hkv=hkv, d=d)
    elif op == "attend":
        case.update(hq=hkv * g, hkv=hkv, d=d)
    return case


def _lengths(case):
    """(prefix, candidates) of every sequence: the same for every seed, so that a case's work is a property of the case."""
    g = torch.Generator().manual_seed(20022 + case["batch"] * 7 + case["hi"] + case["cand_hi"] * 31)
    n = torch.randint(case["lo"], case["hi"] + 1, (case["batch"],), generator=g)
    c = torch.randint(case["cand_lo"], case["cand_hi"] + 1, (case["batch"],), generator=g)
    return n, c


def work(case):
    n, c = _lengths(case)
    rows, kv = c + case["mask"], n + c + case["mask"]
    t, b = int(rows.sum()), case["batch"]
    if case["op"] == "reserve":
        pages = int(((kv + PAGE - 1) // PAGE - (n + PAGE - 1) // PAGE).sum())
        return {"bytes": 16 * b + 8 * t + 8 * pages, "flops": 0}
    hkv, d = case["hkv"], case["d"]
    fp4_row = d // 2 + d // 16
    if case["op"] == "append":  # in bf16, out in 4 bits, and read back: in 4 bits, out bf16
        return {"bytes": t * 2 * hkv * (4 * d + 2 * fp4_row), "flops": 0}
    hq = case["hq"]
    if case["op"] == "rope":
        out = t * hq * d * 2 + t * 2 * hkv * (fp4_row if case["fp4"] else 2 * d)
        back = t * 2 * hkv * (fp4_row + 2 * d) if case["fp4"] else 0
        return {"bytes": t * (hq + 2 * hkv) * d * 2 + t * (8 + 4 * case["rot"]) + out + back, "flops": 8 * t * (hq + hkv) * d}
    return {"bytes": int(kv.sum()) * 2 * hkv * fp4_row + 2 * t * hq * d * 2, "flops": 4 * d * hq * int((rows * kv).sum())}


# ------------------------------------------------------------------------------------------------ inputs
def _i32(x):
    return x.to(device="cuda", dtype=torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    gc = torch.Generator().manual_seed(seed)
    n, c = _lengths(case)
    rows, kv, b = c + case["mask"], n + c + case["mask"], case["batch"]
    t = int(rows.sum())
    s = dict(case=case, total=t, prefix_lens=_i32(n), q_lens=_i32(rows), n_mask=_i32(torch.full((b,), case["mask"])),
             n_blocks=_i32(torch.full((b,), case["blocks"])))
    held = (n + PAGE - 1) // PAGE
    need = (kv + PAGE - 1) // PAGE
    width = int(need.max()) + 2
    pool = int(need.sum()) + 64
    ids = torch.randperm(pool, generator=gc)
    # the table as it stands in front of the call: for `reserve` the prefix's pages only, for the others the block's too
    have = held if case["op"] == "reserve" else need
    col = torch.arange(width)[None, :]
    at = torch.cumsum(have, 0)[:, None] - have[:, None] + col
    table = torch.where(col < have[:, None], ids[at.clamp(max=pool - 1)], torch.full_like(at, -1))
    s.update(num_pages=pool, page_table=_i32(table))
    if case["op"] == "reserve":
        rest = ids[int(have.sum()):]
        k = min(17, int(rest.numel()) // 2)  # some of the free pages were released by the last commit
        free = torch.full((pool,), -1)
        free[: rest.numel() - k] = rest[: rest.numel() - k]
        freed = torch.full((64,), -1)
        freed[:k] = rest[rest.numel() - k:]
        s.update(free_pages=_i32(free), n_free=_i32(torch.tensor([rest.numel() - k])), freed_pages=_i32(freed),
                 n_freed=_i32(torch.tensor([k])), n_free_out=_i32(torch.tensor([0])),
                 slot_map=_i32(torch.zeros(t)), positions=_i32(torch.zeros(t)))
        return s
    hkv, d = case["hkv"], case["d"]
    seq = torch.repeat_interleave(torch.arange(b), rows)
    pos = n[seq] + torch.arange(t) - (torch.cumsum(rows, 0) - rows)[seq]
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)  # noqa: E731
    page_bytes = PAGE * (d // 2 + d // 16)
    s.update(k_scale=0.75, v_scale=1.25)
    if case["op"] == "attend":
        s["q"] = randn(t, case["hq"], d)
        s["out"] = torch.zeros_like(s["q"])
        cache = torch.empty((pool, hkv, 2, page_bytes), dtype=torch.uint8, device="cuda")
        for p in range(0, pool, 4096):  # N(0, 1) values, quantised
            q = min(pool, p + 4096)
            x = torch.randn((q - p, hkv, 2, PAGE, d), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)
            cache[p:q] = _pack(*_quantise(x.float())).reshape(q - p, hkv, 2, page_bytes)
        s["cache"] = cache
        return s
    slot = table[seq, pos // PAGE] * PAGE + pos % PAGE
    s.update(slot_map=_i32(slot), positions=_i32(pos))
    if case["op"] == "append" or case["fp4"]:
        s["cache"] = torch.zeros((pool, hkv, 2, page_bytes), dtype=torch.uint8, device="cuda")
        s["k_back"] = torch.zeros((t, hkv, d), dtype=torch.bfloat16, device="cuda")
        s["v_back"] = torch.zeros((t, hkv, d), dtype=torch.bfloat16, device="cuda")
    else:
        s["cache"] = torch.zeros((pool, 2, hkv, PAGE, d), dtype=torch.bfloat16, device="cuda")
    if case["op"] == "append":
        s["k"], s["v"] = randn(t, hkv, d), randn(t, hkv, d)
        return s
    s["qkv"] = randn(t, (case["hq"] + 2 * hkv) * d)
    s["q_weight"] = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)
    s["k_weight"] = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16)
    s["eps"] = 1e-6
    rot = case["rot"]
    freq = torch.exp(torch.arange(rot // 2, dtype=torch.float64, device="cuda") * (-2.0 / rot * math.log(1e6)))
    angle = torch.arange(int(kv.max()) + 1, dtype=torch.float64, device="cuda")[:, None] * freq
    s["cos_sin"] = torch.cat([torch.cos(angle), torch.sin(angle)], 1).float().contiguous()
    s["q_out"] = torch.zeros((t, case["hq"], d), dtype=torch.bfloat16, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _quantise(x):
    """(codes, scales) of rows in 32 bits: 16 elements share the e4m3 scale nearest to a sixth of their largest magnitude; a code is
    the e2m1 value whose multiple of the scale is nearest, the even one of two (every threshold is exact in 32 bits)."""
    x = x.unflatten(-1, (-1, 16))
    scale = (x.abs().amax(-1, keepdim=True) / 6).clamp(max=448.0).to(torch.float8_e4m3fn)
    s, a = scale.float(), x.abs()
    code = ((a > 0.25 * s).to(torch.uint8) + (a >= 0.75 * s) + (a > 1.25 * s) + (a >= 1.75 * s) + (a > 2.5 * s) + (a >= 3.5 * s)
            + (a > 5 * s))
    code = torch.where(s > 0, code, torch.zeros_like(code)) + 8 * (x < 0).to(torch.uint8)
    return code.flatten(-2), scale.squeeze(-1).view(torch.uint8)


def _pack(codes, scales):
    """[..., 16 tokens, d] codes and their scales as the bytes of a page."""
    return torch.cat([(codes[..., 0::2] + 16 * codes[..., 1::2]).flatten(-2), scales.flatten(-2)], -1)


def _values(codes, scales):
    """[..., d / 2] code bytes and [..., d / 16] scale bytes as the values they stand for, in 32 bits."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    x = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    return x * scales.view(torch.float8_e4m3fn).float().repeat_interleave(16, -1)


def _split(cache, d):
    """Views of the codes [pages, Hkv, 2, 16, d / 2] and the scales [pages, Hkv, 2, 16, d / 16] of 4-bit pages."""
    return cache[..., : PAGE * d // 2].unflatten(-1, (PAGE, d // 2)), cache[..., PAGE * d // 2:].unflatten(-1, (PAGE, d // 16))


def _write(s, k, v):
    """K and V in 32 bits into the 4-bit pages, and the same slots as the values they stand for."""
    d = s["case"]["d"]
    page, at = s["slot_map"].long() // PAGE, s["slot_map"].long() % PAGE
    codes, scales = _split(s["cache"], d)
    back = []
    for which, (x, by) in enumerate(((k, s["k_scale"]), (v, s["v_scale"]))):
        c, sc = _quantise(x / by)
        codes[page, :, which, at] = c[..., 0::2] + 16 * c[..., 1::2]
        scales[page, :, which, at] = sc
        back.append((_values(codes[page, :, which, at], scales[page, :, which, at]) * by).to(torch.bfloat16))
    return back


def _turn(x, weight, s):
    """Norm and rotation of [T, H, d] in 32 bits."""
    rot, adjacent = s["case"]["rot"], s["case"]["adjacent"]
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight.float()
    cos, sin = s["cos_sin"][s["positions"].long()][:, None].split(rot // 2, -1)
    y, rest = x[..., :rot], x[..., rot:]
    a, b = (y[..., 0::2], y[..., 1::2]) if adjacent else (y[..., : rot // 2], y[..., rot // 2:])
    turned = (a * cos - b * sin, b * cos + a * sin)
    return torch.cat([torch.stack(turned, -1).flatten(-2) if adjacent else torch.cat(turned, -1), rest], -1)


def _plain_reserve(s):
    n, rows, mask, blocks = (s[k].long() for k in ("prefix_lens", "q_lens", "n_mask", "n_blocks"))
    free, b = s["free_pages"], s["case"]["batch"]
    n_free, n_freed = s["n_free"].long(), s["n_freed"].long()
    i = torch.arange(free.numel(), device="cuda")
    top = n_free + n_freed
    free = torch.where((i >= n_free) & (i < top), s["freed_pages"][(i - n_free).clamp(0, s["freed_pages"].numel() - 1)], free)
    first, last = (n + PAGE - 1) // PAGE, (n + rows + PAGE - 1) // PAGE
    need = last - first
    before = torch.cumsum(need, 0) - need
    col = torch.arange(s["page_table"].shape[1], device="cuda")[None, :]
    new = (col >= first[:, None]) & (col < last[:, None])
    take = (top - 1 - (before[:, None] + col - first[:, None])).clamp(0, free.numel() - 1)
    table = torch.where(new, free[take], s["page_table"])
    start = torch.cumsum(rows, 0) - rows
    row = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(start + rows, row, right=True)
    j = row - start[seq]
    pos = n[seq] + j
    slot = table[seq, pos // PAGE].long() * PAGE + pos % PAGE
    cand = (rows - mask)[seq]
    each = (mask // blocks.clamp(min=1))[seq].clamp(min=1)
    g, u = (j - cand) // each, (j - cand) % each
    position = torch.where(j < cand, pos, n[seq] + cand - blocks[seq] + g + 1 + u)
    return [table.to(torch.int32), (top - need.sum()).to(torch.int32), slot.to(torch.int32), position.to(torch.int32)]


def _plain_attend(s):
    c = s["case"]
    hkv, d, grp = c["hkv"], c["d"], c["hq"] // c["hkv"]
    n, rows, b = s["prefix_lens"].long(), s["q_lens"].long(), c["batch"]
    kv, most = n + rows, int(_lengths(c)[1].max()) + c["mask"]
    top = s["page_table"].shape[1] - 2
    codes, scales = _split(s["cache"], d)
    pages = s["page_table"][:, :top].long().clamp(min=0)

    def dense(which, by):  # [B, Hkv, tokens, d]
        x = _values(codes[:, :, which][pages], scales[:, :, which][pages]) * by
        return x.permute(0, 2, 1, 3, 4).reshape(b, hkv, top * PAGE, d)

    start = torch.cumsum(rows, 0) - rows
    i = torch.arange(most, device="cuda")
    real = i < rows[:, None]
    take = (start[:, None] + i).clamp(max=s["total"] - 1)
    q = s["q"].float()[take].reshape(b, most, hkv, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, grp * most, d)
    score = (q @ dense(0, s["k_scale"]).transpose(2, 3)).reshape(b, hkv, grp, most, top * PAGE) * (1.0 / math.sqrt(d))
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
    o = (p.reshape(b, hkv, grp * most, -1) @ dense(1, s["v_scale"])).reshape(b, hkv, grp, most, d) / total.clamp(min=1e-30)
    return o.permute(0, 3, 1, 2, 4).reshape(b, most, c["hq"], d)[real].to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ the pass
_contexts = {}


def _context(s):
    """The library's handle, one for each shape, as a program keeps it."""
    import paper_2605_20022_b200 as fd

    c = s["case"]
    key = (c.get("hq", c.get("hkv", 1)), c.get("hkv", 1), c.get("d", 128), c["batch"], c["cand_hi"] + c["mask"], s["page_table"].shape[1])
    if key not in _contexts:
        _contexts[key] = fd.fd_create(key[0], key[1], key[2], 1, key[3], key[4], key[5])
    return fd, _contexts[key]


def run(s):
    c = s["case"]
    if own:
        fd, ctx = _context(s)
        b, t = c["batch"], s["total"]
        if c["op"] == "reserve":
            fd.fd_kv_reserve(ctx, b, t, s["page_table"], s["prefix_lens"], s["q_lens"], s["n_mask"], s["n_blocks"], s["freed_pages"],
                             s["n_freed"], s["free_pages"], s["n_free"], s["n_free_out"], s["num_pages"], s["slot_map"], s["positions"])
            return [s["page_table"], s["n_free_out"], s["slot_map"], s["positions"]]
        if c["op"] == "attend":
            fd.fd_attn_draft_verify_fp4(ctx, b, t, s["q"], s["cache"], s["num_pages"], s["page_table"], s["prefix_lens"], s["q_lens"],
                                        s["n_mask"], s["n_blocks"], s["k_scale"], s["v_scale"], s["out"])
            return [s["out"]]
        if c["op"] == "rope":
            fd.fd_qk_norm_rope_append(ctx, t, s["qkv"], s["qkv"].stride(0), s["q_weight"], s["k_weight"], s["eps"], s["cos_sin"],
                                      s["cos_sin"].shape[0], c["rot"], fd.FD_ROPE_ADJACENT if c["adjacent"] else fd.FD_ROPE_HALVES,
                                      s["positions"], s["slot_map"], s["q_out"], s["cache"], s["num_pages"],
                                      fd.FD_KV_FP4 if c["fp4"] else fd.FD_KV_BF16, s["k_scale"], s["v_scale"])
            if not c["fp4"]:
                return [s["q_out"], s["cache"]]
        else:
            fd.fd_kv_append_fp4(ctx, b, t, s["k"], s["v"], s["cache"], s["num_pages"], s["page_table"], s["prefix_lens"], s["q_lens"],
                                s["k_scale"], s["v_scale"])
        fd.fd_kv_read_fp4(ctx, b, t, s["cache"], s["num_pages"], s["page_table"], s["prefix_lens"], s["q_lens"], s["k_scale"],
                          s["v_scale"], s["k_back"], s["v_back"])
        back = [s["k_back"], s["v_back"]]
        return [s["q_out"]] + back if c["op"] == "rope" else back
    if c["op"] == "reserve":
        return _plain_reserve(s)
    if c["op"] == "attend":
        return [_plain_attend(s)]
    if c["op"] == "append":
        return _write(s, s["k"].float(), s["v"].float())
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    x = s["qkv"].unflatten(1, (hq + 2 * hkv, d))
    q, k, v = _turn(x[:, :hq], s["q_weight"], s), _turn(x[:, hq: hq + hkv], s["k_weight"], s), x[:, hq + hkv:]
    if c["fp4"]:
        return [q.to(torch.bfloat16)] + _write(s, k, v.float())
    page, at = s["slot_map"].long() // PAGE, s["slot_map"].long() % PAGE
    s["cache"][page, 0, :, at] = k.to(torch.bfloat16)
    s["cache"][page, 1, :, at] = v
    return [q.to(torch.bfloat16), s["cache"]]


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def _nearest(x, grid):
    """Index of the value of an ascending grid nearest to x >= 0, of two the one with the even index."""
    hi = torch.searchsorted(grid, x).clamp(1, grid.numel() - 1)
    lo = hi - 1
    dl, dh = x - grid[lo], grid[hi] - x
    return torch.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)


def _exact_fp4(x, by):
    """What 64-bit rows stand for once they are held in 4 bits."""
    e4m3 = torch.tensor([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127],
                        dtype=torch.float64, device=x.device)
    e2m1 = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    y = (x / by).unflatten(-1, (-1, 16))
    scale = e4m3[_nearest(y.abs().amax(-1, keepdim=True) / 6, e4m3)]
    code = _nearest(y.abs() / torch.where(scale > 0, scale, torch.ones_like(scale)), e2m1)
    return (torch.sign(y) * e2m1[code] * scale).flatten(-2) * by


def exact(case, seed):
    if case["op"] == "reserve":
        return None
    s = prepare(case, seed)
    hkv, d = case["hkv"], case["d"]
    if case["op"] == "append":
        return [_exact_fp4(s["k"].double(), s["k_scale"]), _exact_fp4(s["v"].double(), s["v_scale"])]
    hq = case["hq"]
    if case["op"] == "rope":
        def turned(x, w):
            x = x.double()
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / d + s["eps"]) * w.double()
            h = case["rot"] // 2
            ca, sa = (s["cos_sin"][s["positions"].long()].double()[:, None, k * h:(k + 1) * h] for k in (0, 1))
            at = torch.arange(h, device="cuda")
            first, second = (2 * at, 2 * at + 1) if case["adjacent"] else (at, at + h)
            y = x.clone()
            y[..., first] = x[..., first] * ca - x[..., second] * sa
            y[..., second] = x[..., first] * sa + x[..., second] * ca
            return y

        heads = s["qkv"].reshape(s["total"], hq + 2 * hkv, d)
        q, k, v = turned(heads[:, :hq], s["q_weight"]), turned(heads[:, hq:hq + hkv], s["k_weight"]), heads[:, hq + hkv:].double()
        if case["fp4"]:
            return [q, _exact_fp4(k, s["k_scale"]), _exact_fp4(v, s["v_scale"])]
        cache = s["cache"].double()
        for which, x in ((0, k), (1, v)):
            cache[s["slot_map"].long() // PAGE, which, :, s["slot_map"].long() % PAGE] = x
        return [q, cache]
    n, rows = s["prefix_lens"].tolist(), s["q_lens"].tolist()
    out, row0 = torch.zeros((s["total"], hq, d), dtype=torch.float64, device="cuda"), 0
    for b in range(case["batch"]):
        lq, total = rows[b], n[b] + rows[b]
        raw = s["cache"][s["page_table"][b, : -(-total // PAGE)].long()]
        nib = raw[..., : PAGE * d // 2].long()
        nib = torch.stack([nib % 16, nib // 16], -1).reshape(-1, hkv, 2, PAGE, d)
        mag = nib % 8
        val = torch.where(mag < 2, mag.double() / 2, (2 + mag % 2).double() * 2.0 ** (mag // 2 - 2).double())
        val = torch.where(nib >= 8, -val, val)
        e = raw[..., PAGE * d // 2:].long().reshape(-1, hkv, 2, PAGE, d // 16)
        sc = torch.where(e < 8, e.double() / 512, (8 + e % 8).double() * 2.0 ** (e // 8 - 10).double())
        val = (val.unflatten(-1, (-1, 16)) * sc[..., None]).flatten(-2)
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
            grp = hq // hkv
            x = s["q"][row0: row0 + lq, h * grp:(h + 1) * grp].double()
            w = torch.softmax((x.reshape(-1, d) @ k[h].T * (s["k_scale"] / math.sqrt(d))).reshape(lq, grp, total)
                              .masked_fill(~visible[:, None], float("-inf")), -1)
            out[row0: row0 + lq, h * grp:(h + 1) * grp] = (w.reshape(-1, total) @ v[h]).reshape(lq, grp, d) * s["v_scale"]
        row0 += lq
    return [out]
