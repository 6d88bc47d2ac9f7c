"""64-bit references (numpy, plain definitions) of the 8-bit cache, of a pool's pages, and of the prompt attention.

Nothing here shares code with the kernels or with their plain torch forms."""
import numpy as np
import torch

from fp4_ref import E4M3, PAGE, nearest, rows_of

TAIL = 16
POWERS = 2.0 ** np.arange(-15, 8)


def block_bytes(d):
    return PAGE * d + TAIL


def scale_of(amax):
    """The smallest power of two from 2^-15 to 2^7 that 448 times reaches amax (none: 2^7)."""
    return POWERS[np.minimum(np.searchsorted(448 * POWERS, amax), len(POWERS) - 1)]


def code_of(x, scale):
    """float64 -> e4m3 bytes of x / scale: nearest, ties to even, at most 448; NaN -> 0x7f."""
    y = np.asarray(x, dtype=np.float64) / scale
    c = np.where(np.isnan(y), 127, nearest(np.minimum(np.abs(np.where(np.isnan(y), 0.0, y)), 448.0), E4M3))
    return (c + 128 * (np.signbit(y) & ~np.isnan(y))).astype(np.uint8)


def values(codes, scales):
    """(codes [..., 16, d], scales [...]) -> float64; codes 127 and 255 are NaN."""
    grid = np.concatenate([E4M3, [np.nan]])
    return grid[codes & 127] * np.where(codes & 128, -1.0, 1.0) * np.asarray(scales, dtype=np.float64)[..., None, None]


def split(cache, d):
    """[pages, Hkv, 2, bytes] uint8 -> (codes [pages, Hkv, 2, 16, d], scales [pages, Hkv, 2] float32), both copies."""
    codes = cache[..., :PAGE * d].reshape(cache.shape[:3] + (PAGE, d)).copy()
    return codes, np.ascontiguousarray(cache[..., PAGE * d:PAGE * d + 4]).view(np.float32)[..., 0].copy()


def join(codes, scales):
    tail = np.zeros(scales.shape + (TAIL,), dtype=np.uint8)
    tail[..., :4] = np.ascontiguousarray(scales.astype(np.float32)).view(np.uint8).reshape(scales.shape + (4,))
    return np.concatenate([codes.reshape(codes.shape[:3] + (-1,)), tail], -1)


def as_bf16_cache(cache, d):
    """The values of an 8-bit cache as [pages, 2, Hkv, 16, d] bf16 (exact: 4 significant bits)."""
    with np.errstate(invalid="ignore"):
        v = values(*split(cache, d)).transpose(0, 2, 1, 3, 4)
    return torch.from_numpy(np.ascontiguousarray(v)).to(torch.bfloat16)


def make_cache(kv, rng_seed=None):
    """bf16 cache [pages, 2, Hkv, 16, d] -> 8-bit cache (numpy uint8).  A slot whose bf16 values are not finite or beyond 1e20
    (poison: no token owns it) does not count for the scale; with a seed it gets random bytes, NaN among them."""
    x = kv.double().numpy().transpose(0, 2, 1, 3, 4)
    live = (np.abs(x) < 1e20).all(-1)
    scales = scale_of(np.where(live[..., None], np.abs(x), 0.0).max((-1, -2)))
    with np.errstate(invalid="ignore", over="ignore"):
        codes = code_of(np.where(live[..., None], x, 0.0), scales[..., None, None])
    if rng_seed is not None:
        r = np.random.default_rng(rng_seed)
        junk = r.integers(0, 256, codes[~live].shape)
        junk[..., 0] = 127                                      # a NaN
        codes[~live] = junk
        none = ~live.any(-1)                                    # a block without tokens: any scale
        scales[none] = r.choice([np.nan, np.inf, 0.0, -3e38, 1.0], scales[none].shape)
    return join(codes, scales)


def append(cache, d, step, k, v, page_table=None, skip=()):
    """A copy of the cache with the block's rows written, block by block."""
    pt = step.page_table if page_table is None else page_table
    codes, scales = split(cache, d)
    out = cache.copy()
    rows = {}
    for row, (b, _, j) in enumerate(rows_of(step)):
        rows.setdefault((b, j // PAGE), []).append((j % PAGE, row))
    for (b, col), new in rows.items():
        page, n = int(pt[b, col]), int(step.prefix_lens[b])
        if not 0 <= page < cache.shape[0] or b in skip:
            continue
        kept = np.arange(max(0, min(PAGE, n - col * PAGE)))
        at, src = [t for t, _ in new], [r for _, r in new]
        for which, x in enumerate((k, v)):
            for h in range(cache.shape[1]):
                held = values(codes[page, h, which][kept], scales[page, h, which]) if len(kept) else np.zeros((0, d))
                fresh = x[src, h].double().numpy()
                mags = np.abs(np.concatenate([held, fresh]))
                s = scale_of(np.where(np.isnan(mags), 0.0, mags).max())
                c = codes[page, h, which].copy()
                if len(kept) and s != scales[page, h, which]:
                    c[kept] = code_of(held, s)
                c[at] = code_of(fresh, s)
                out[page, h, which] = join(c[None, None, None], np.array([[[s]]]))[0, 0, 0]
    return out


# ------------------------------------------------------------------------------------------------ pages
def fork(parents, children, table, prefix, shared, free):
    """(table, prefix, shared, free list, copies) by the definition, one fork at a time; shared and table are copied."""
    table, prefix, shared, stack, copies = np.array(table), np.array(prefix), np.array(shared), list(free), []
    for s, t in zip(parents, children):
        n = int(prefix[s])
        row = np.full(table.shape[1], -1)
        row[:n // PAGE] = table[s, :n // PAGE]
        shared[row[:n // PAGE]] += 1
        copies.append((-1, -1))
        if n % PAGE:
            row[n // PAGE] = stack.pop()
            copies[-1] = (int(table[s, n // PAGE]), int(row[n // PAGE]))
        table[t], prefix[t] = row, n
    return table, prefix, shared, stack, copies


def free(seqs, table, prefix, shared, stack):
    table, prefix, shared, stack = np.array(table), np.array(prefix), np.array(shared), list(stack)
    for b in reversed(list(seqs)):
        for p in reversed(range(-(-int(prefix[b]) // PAGE))):
            page = table[b, p]
            if shared[page] > 0:
                shared[page] -= 1
            else:
                stack.append(int(page))
            table[b, p] = -1
        prefix[b] = 0
    return table, prefix, shared, stack


def compact(table, shared, stack, num_pages):
    """(table, shared, free list, page_map, moves)."""
    used = sorted(set(range(num_pages)) - set(stack))
    m = len(used)
    holes = sorted(i for i in stack if i < m)
    moves = list(zip([i for i in used if i >= m], holes))
    page_map = np.full(num_pages, -1)
    page_map[used] = used
    for a, b in moves:
        page_map[a] = b
    shared2 = np.zeros_like(shared)
    shared2[page_map[used]] = np.asarray(shared)[used]
    table = np.array([[page_map[x] if 0 <= x < num_pages else x for x in row] for row in table])
    return table, shared2, [num_pages - 1 - k for k in range(len(stack))], page_map, moves


# ------------------------------------------------------------------------------------------------ prompt attention
def prompt(q, k, v, q_lens, kv_lens, scale=None):
    """(out, sum_j p_j |v_j|) in float64, torch on the inputs' device."""
    Hq, d, Hkv = q.shape[1], q.shape[2], k.shape[1]
    out, size = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    scale = 1 / np.sqrt(d) if scale is None else scale
    r0 = k0 = 0
    for Lq, Lk in zip(q_lens, kv_lens):
        i, j = torch.arange(Lq, device=q.device)[:, None], torch.arange(Lk, device=q.device)[None]
        sees = j <= i + Lk - Lq
        for h in range(Hq):
            if not (Lq and Lk):
                continue
            kk, vv = k[k0:k0 + Lk, h * Hkv // Hq].double(), v[k0:k0 + Lk, h * Hkv // Hq].double()
            s = (q[r0:r0 + Lq, h].double() @ kk.T * scale).masked_fill(~sees, -float("inf"))
            w = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e300))
            w = w.masked_fill(~sees, 0.0)
            w = w / w.sum(-1, keepdim=True).clamp(min=1e-300)
            out[r0:r0 + Lq, h], size[r0:r0 + Lq, h] = w @ vv, w @ vv.abs()
        r0, k0 = r0 + Lq, k0 + Lk
    return out, size
