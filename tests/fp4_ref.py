"""64-bit references (numpy, plain loops and definitions) of the operators around the 4-bit cache.

Nothing here shares code with the kernels or with their plain torch forms."""
import numpy as np
import torch

PAGE = 16
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# the 127 finite non-negative e4m3 numbers, by their byte
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def nearest(x, grid):
    """Index of the grid value nearest to each x >= 0 (above the grid: the last), ties to the even index."""
    x = np.asarray(x, dtype=np.float64)
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    with np.errstate(invalid="ignore"):
        dl, dh = x - grid[lo], grid[hi] - x
    return np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)


def quantise(x, by=1.0):
    """float64 [..., d] -> (codes [..., d] in 0..15, scale bytes [..., d / 16]).  NaN -> code 0, infinities saturate."""
    y = np.asarray(x, dtype=np.float64) / by
    y = y.reshape(y.shape[:-1] + (-1, 16))
    mag = np.where(np.isnan(y), 0.0, np.abs(y))
    scale = nearest(np.minimum(mag.max(-1) / 6, 448.0), E4M3)
    s = E4M3[scale][..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        code = np.where(s > 0, nearest(np.where(s > 0, np.minimum(mag / s, 1e9), 0.0), E2M1), 0)
    code = code + 8 * ((y < 0) & ~np.isnan(y))
    return code.reshape(code.shape[:-2] + (-1,)).astype(np.uint8), scale.astype(np.uint8)


def values(codes, scales):
    """(codes, scale bytes) -> float64; a NaN scale byte (127, 255) gives NaN, a negative one a negative value."""
    grid = np.concatenate([E4M3, [np.nan]])
    s = grid[scales & 127] * np.where(scales & 128, -1.0, 1.0)
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return (v.reshape(v.shape[:-1] + (-1, 16)) * s[..., None]).reshape(v.shape)


def page_bytes(d):
    return PAGE * (d // 2 + d // 16)


def split(cache, d):
    """[pages, Hkv, 2, bytes] uint8 -> (codes [pages, Hkv, 2, 16, d], scale bytes [pages, Hkv, 2, 16, d / 16])."""
    raw = cache[..., :PAGE * d // 2].reshape(cache.shape[:3] + (PAGE, d // 2))
    codes = np.stack([raw & 15, raw >> 4], -1).reshape(cache.shape[:3] + (PAGE, d))
    return codes, cache[..., PAGE * d // 2:].reshape(cache.shape[:3] + (PAGE, d // 16))


def join(codes, scales):
    raw = (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)
    return np.concatenate([raw.reshape(raw.shape[:3] + (-1,)), scales.reshape(scales.shape[:3] + (-1,))], -1)


def as_bf16_cache(cache, d):
    """The values of a 4-bit cache as [pages, 2, Hkv, 16, d] bf16 (exact: at most 6 significant bits)."""
    v = values(*split(cache, d)).transpose(0, 2, 1, 3, 4)
    t = torch.from_numpy(np.ascontiguousarray(v)).to(torch.bfloat16)
    assert np.array_equal(t.double().numpy(), v, equal_nan=True)
    return t


def make_cache(kv, rng_seed=None):
    """bf16 cache [pages, 2, Hkv, 16, d] -> 4-bit cache (numpy uint8); with a seed, every slot whose bf16 values are not
    finite or beyond 1e20 (poison: no token owns it) gets random bytes instead, NaN scales among them."""
    x = kv.double().numpy().transpose(0, 2, 1, 3, 4)
    codes, scales = quantise(x)
    if rng_seed is not None:
        r = np.random.default_rng(rng_seed)
        dead = ~(np.abs(x) < 1e20).all(-1)
        codes[dead] = r.integers(0, 16, codes[dead].shape)
        junk = r.integers(0, 256, scales[dead].shape)
        junk[..., 0] = 127                                      # a NaN
        scales[dead] = junk
    return join(codes, scales)


def rows_of(step):
    """For every query row: (sequence, index in the block, logical position)."""
    for b in range(step.batch):
        for i in range(int(step.q_lens[b])):
            yield b, i, int(step.prefix_lens[b]) + i


def append(cache, d, step, k, v, k_scale, v_scale, page_table=None):
    """A copy of the cache with the block's rows written."""
    pt = step.page_table if page_table is None else page_table
    codes, scales = split(cache.copy(), d)
    codes, scales = codes.copy(), scales.copy()
    qk, qv = quantise(k.double().numpy(), k_scale), quantise(v.double().numpy(), v_scale)
    for row, (b, _, j) in enumerate(rows_of(step)):
        page = int(pt[b, j // PAGE])
        if not 0 <= page < cache.shape[0]:
            continue
        for which, (c, s) in enumerate((qk, qv)):
            codes[page, :, which, j % PAGE], scales[page, :, which, j % PAGE] = c[row], s[row]
    return join(codes, scales)


def reserve(page_table, prefix, q_lens, n_mask, n_blocks, freed, free, num_pages):
    """(page_table, free list, slots, positions, shortage) by the definition, one page at a time."""
    table, stack = np.array(page_table, dtype=np.int64), list(free) + list(freed)
    first = [-(-int(n) // PAGE) for n in prefix]
    last = [-(-(int(n) + int(L)) // PAGE) for n, L in zip(prefix, q_lens)]
    short = sum(b - a for a, b in zip(first, last)) > len(stack)
    slots, positions = [], []
    for b, (n, L, M) in enumerate(zip(prefix, q_lens, n_mask)):
        n, L, M = int(n), int(L), int(M)
        if not short:
            for p in range(first[b], last[b]):
                table[b, p] = stack.pop()
                if not 0 <= table[b, p] < num_pages:
                    table[b, p] = -1
        nb = max(1, int(n_blocks[b])) if n_blocks is not None else 1
        C = L - M
        for i in range(L):
            j = n + i
            page = table[b, j // PAGE]
            slots.append(page * PAGE + j % PAGE if not short and 0 <= page < num_pages else -1)
            if i < C:
                positions.append(j)
            else:
                g, u = divmod(i - C, M // nb)
                positions.append(n + (C - nb + g) + 1 + u)
    return table, stack, np.array(slots, dtype=np.int64), np.array(positions, dtype=np.int64), short


def norm_rope(x, weight, eps, cos_sin, positions, rot, adjacent):
    """x [T, H, d] float64 -> (result, magnitude sum of the two terms of every element, for error bounds)."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    y, size = x.copy(), np.abs(x)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
        c = np.asarray(cos_sin[positions, i], dtype=np.float64)[:, None]
        s = np.asarray(cos_sin[positions, rot // 2 + i], dtype=np.float64)[:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a] = np.abs(x[..., a] * c) + np.abs(x[..., b] * s)
        size[..., b] = np.abs(x[..., b] * c) + np.abs(x[..., a] * s)
    return y, size
