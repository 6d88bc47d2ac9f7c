"""The 64-bit references of the 4-bit cache and of page reservation, pinned on the CPU; refusals that need no GPU."""
import numpy as np
import pytest
import torch

import fp4_ref as ref
import paper_2605_20022_b200 as fd


def test_e4m3_grid_is_torchs():
    by = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ref.E4M3, by)


def test_quantise_picks_the_nearest_of_all_codes():
    """Against every code of the scale that was picked, and every scale, one by one."""
    r = np.random.default_rng(1)
    x = np.concatenate([r.standard_normal((40, 32)) * 10.0 ** r.integers(-4, 4, (40, 1)), np.zeros((1, 32)), np.full((1, 32), 1e9)])
    codes, scales = ref.quantise(x)
    held = ref.values(codes, scales)
    for row in range(x.shape[0]):
        for g in range(2):
            part = x[row, 16 * g:16 * g + 16]
            want = min(np.abs(part).max() / 6, 448)
            assert np.abs(ref.E4M3 - want).min() == abs(ref.E4M3[scales[row, g]] - want)
            s = ref.E4M3[scales[row, g]]
            every = np.concatenate([ref.E2M1, -ref.E2M1]) * s
            best = np.abs(part[:, None] - every[None]).min(1)
            np.testing.assert_allclose(np.abs(part - held[row, 16 * g:16 * g + 16]), best, rtol=1e-12, atol=0)


def test_ties_go_to_the_even_code_and_a_nan_is_zero():
    x = np.array([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, np.nan, 0.26, 0.74, 4.99, 5.01])
    codes, scales = ref.quantise(x)
    assert ref.E4M3[scales[0]] == 1.0
    assert codes.tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 10, 14, 0, 1, 1, 6, 7]
    codes, scales = ref.quantise(np.array([np.inf, -np.inf] + [1.0] * 14))
    assert ref.E4M3[scales[0]] == 448 and codes[:3].tolist() == [7, 15, 0]


def test_values_of_a_cache_are_exact_in_bf16_and_requantise_to_themselves():
    r = np.random.default_rng(2)
    codes, scales = ref.quantise(r.standard_normal((3, 2, 2, 16, 64)) * 3)
    cache = ref.join(codes, scales)
    assert cache.shape[-1] == ref.page_bytes(64) == fd.fd_kv_fp4_page_bytes(64)
    c2, s2 = ref.split(cache, 64)
    np.testing.assert_array_equal(c2, codes)
    np.testing.assert_array_equal(s2, scales)
    kv = ref.as_bf16_cache(cache, 64)                            # asserts exactness
    again = ref.quantise(kv.double().numpy().transpose(0, 2, 1, 3, 4))
    np.testing.assert_array_equal(ref.values(*again), ref.values(codes, scales))


def test_reserve_reference_mirrors_the_commit():
    """What the commit released, the reservation hands out again: pages are neither lost nor handed out twice."""
    import oracle
    r = np.random.default_rng(3)
    B, width, pool = 5, 12, 64
    table = np.full((B, width), -1)
    prefix, stack, released = np.zeros(B, dtype=np.int64), list(range(pool)), []
    for _ in range(30):
        prefix = np.where(prefix > 120, 0, prefix)
        for b in range(B):                                      # a sequence that starts afresh gives its pages back
            if prefix[b] == 0:
                stack += [p for p in table[b] if p >= 0]
                table[b] = -1
        M = r.integers(0, 3, B) * 4
        L = r.integers(1, 30, B) + M
        table, stack, slots, pos, short = ref.reserve(table, prefix, L, M, None, released, stack, pool)
        assert not short and len(set(slots)) == len(slots) == L.sum()
        held = table[table >= 0]
        assert len(set(held)) == len(held) and sorted(list(held) + stack) == list(range(pool))
        assert (pos[:L[0] - M[0]] == prefix[0] + np.arange(L[0] - M[0])).all()
        acc = np.array([r.integers(0, l) for l in L])
        table, prefix, released = oracle.commit(table, prefix, L, acc)
        table, prefix, released = table.astype(np.int64), prefix.astype(np.int64), [int(p) for p in released]


def test_positions_of_branches_continue_behind_their_hypothesis():
    _, _, _, pos, _ = ref.reserve(np.zeros((1, 4)), [10], [3 + 4], [4], [2], [], list(range(9)), 9)
    assert pos.tolist() == [10, 11, 12, 12, 13, 13, 14]          # r = 1: 12, 13;  r = 2: 13, 14


@pytest.mark.parametrize("adjacent", [False, True])
def test_norm_rope_reference_keeps_lengths_and_composes(adjacent):
    r = np.random.default_rng(4)
    angle = np.arange(20)[:, None] * np.array([1.0, 0.3, 0.1, 0.01, 0.5, 0.25, 2.0, 0.7])
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1)
    x = r.standard_normal((20, 3, 32))
    y, _ = ref.norm_rope(x, None, 0.0, table, np.arange(20), 16, adjacent)
    np.testing.assert_allclose((y[..., :16] ** 2).sum(-1), (x[..., :16] ** 2).sum(-1))
    np.testing.assert_array_equal(y[..., 16:], x[..., 16:])
    z, _ = ref.norm_rope(y, None, 0.0, np.concatenate([np.cos(angle), -np.sin(angle)], 1), np.arange(20), 16, adjacent)
    np.testing.assert_allclose(z, x, atol=1e-12)                 # turned back
    n, _ = ref.norm_rope(x, np.full(32, 2.0), 1e-6, table, np.arange(20), 0, adjacent)
    np.testing.assert_allclose((n ** 2).mean(-1), 4.0, rtol=1e-4)


def test_calls_without_a_context_are_refused():
    bad = fd.FD_ERR_INVALID_ARG
    assert fd.fd_kv_reserve(None, 1, 1, 1, 1, 1, 1, None, None, None, 1, 1, 1, 8, 1, 1, stream=1, raise_on_error=False) == bad
    assert fd.fd_qk_norm_rope_append(None, 1, 16, 1024, None, None, 0.0, None, 0, 0, 0, None, 1, 16, 128, 8, stream=1, raise_on_error=False) == bad
    assert fd.fd_kv_append_fp4(None, 1, 1, 16, 16, 16, 8, 4, 4, 4, stream=1, raise_on_error=False) == bad
    assert fd.fd_kv_read_fp4(None, 1, 1, 16, 8, 4, 4, 4, 1.0, 1.0, 16, 16, stream=1, raise_on_error=False) == bad
    assert fd.fd_attn_draft_verify_fp4(None, 1, 1, 16, 16, 8, 4, 4, 4, 4, None, 1.0, 1.0, 16, stream=1, raise_on_error=False) == bad
