"""Pages from reservation to compaction with fd_kv_commit in between: whatever the commit releases has one owner afterwards."""
import numpy as np
import pytest
import torch

import fp8_ref as ref
import paper_2605_20022_b200 as fd

I32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731


def assert_one_owner(table, shared, stack):
    """Every page is in the tables, as often as shared says and once more, or once on the list."""
    owners = np.bincount(np.asarray(table)[np.asarray(table) >= 0], minlength=len(shared))
    listed = np.bincount(np.asarray(stack, dtype=int), minlength=len(shared))
    np.testing.assert_array_equal(listed, owners == 0)
    np.testing.assert_array_equal(shared, np.maximum(owners - 1, 0))


def test_ids_held_back_over_a_compaction():
    """The definitions themselves: an id that a commit released and that is not on the list is renamed as a page in use."""
    table, shared, stack, released = np.array([[0, 11], [9, 1]]), np.zeros(12, int), list(range(2, 9)), [10]
    t, s, st, page_map, _ = ref.compact(table, shared, stack, 12)
    with pytest.raises(AssertionError):
        assert_one_owner(t, s, st + released)
    assert_one_owner(t, s, st + [int(page_map[i]) for i in released])
    t, s, st, _, _ = ref.compact(table, shared, stack + released, 12)
    assert_one_owner(t, s, st)


@pytest.mark.gpu
@pytest.mark.parametrize("pushed", [True, False])
@pytest.mark.parametrize("seed,B,longest", [(1, 2, 40), (2, 9, 64), (3, 120, 64), (4, 700, 20)])
def test_commit_free_fork_compact_reserve(seed, B, longest, pushed):
    """Rounds of steps.  The released ids are pushed by a reservation for no sequence, or held back and replaced by page_map."""
    r = np.random.default_rng(seed)
    width, pool = 4 + 6 * (longest // 16 + 2), B * (4 + 6 * (longest // 16 + 2)) + 30
    ctx = fd.fd_create(2, 1, 64, 10, B, longest, width)
    z = lambda n, v=0: I32(np.full(max(n, 1), v))  # noqa: E731
    table, prefix, shared, free, n = I32(np.full((B, width), -1)), z(B), z(pool), I32(r.permutation(pool)), I32([pool])
    freed, n_freed, none = z(B * (longest // 16 + 2), -7), I32([0]), z(B)
    page_map, src, dst, moves = z(pool), z(pool), z(pool), z(1)
    try:
        for _ in range(6):
            q_lens = r.integers(1, longest + 1, B)
            T = int(q_lens.sum())
            fd.fd_kv_reserve(ctx, B, T, table, prefix, I32(q_lens), none, None, None if pushed else freed, None if pushed else n_freed, free, n, n, pool,
                             z(T), z(T))
            fd.fd_kv_commit(ctx, B, table, prefix, I32(q_lens), I32(r.integers(0, q_lens)), freed, n_freed)
            if pushed:
                fd.fd_kv_reserve(ctx, 0, 0, None, None, None, None, None, freed, n_freed, free, n, n, pool, None, None)
            ended = r.permutation(B)[: B // 3]
            stay = np.setdiff1d(np.arange(B), ended)
            fd.fd_kv_free(ctx, len(ended), I32(ended), B, table, prefix, shared, free, n, n, pool)
            fd.fd_kv_fork(ctx, len(ended), I32(r.choice(stay, len(ended))), I32(ended), B, table, prefix, shared, free, n, n, pool, src, dst)
            fd.fd_kv_compact(ctx, B, table, shared, free, n, pool, page_map, pool, src, dst, moves)
            if not pushed:
                k = int(n_freed)
                freed[:k] = page_map[freed[:k].long()]
            assert fd.fd_last_device_status(ctx) == 0
            stack = free[: int(n)].tolist() + ([] if pushed else freed[: int(n_freed)].tolist())
            assert_one_owner(table.cpu().numpy(), shared.cpu().numpy(), stack)
    finally:
        fd.fd_destroy(ctx)


@pytest.mark.gpu
def test_a_fork_takes_pages_that_the_commit_released():
    ctx = fd.fd_create(2, 1, 64, 10, 2, 64, 4)
    table, prefix, shared, free, n = I32([[0, 1, 2, 3], [-1] * 4]), I32([20, 0]), I32([0] * 4), I32([-1] * 4), I32([0])
    freed, n_freed, src, dst = I32([-1] * 8), I32([0]), I32([5]), I32([5])
    try:
        fd.fd_kv_commit(ctx, 2, table, prefix, I32([40, 0]), I32([9, -1]), freed, n_freed)   # 30 tokens stay: pages 2 and 3 go
        args = [ctx, 1, I32([0]), I32([1]), 2, table, prefix, shared, free, n, n, 4, src, dst]
        fd.fd_kv_fork(*args)
        assert fd.fd_last_device_status(ctx) == fd.FD_DEV_NO_PAGES and src.tolist() == dst.tolist() == [-1]
        fd.fd_kv_reserve(ctx, 0, 0, None, None, None, None, None, freed, n_freed, free, n, n, 4, None, None)
        fd.fd_kv_fork(*args)
        assert fd.fd_last_device_status(ctx) == 0 and table.tolist() == [[0, 1, -1, -1], [0, 3, -1, -1]] and src.tolist() == [1] and dst.tolist() == [3]
        assert_one_owner(table.cpu().numpy(), shared.cpu().numpy(), free[: int(n)].tolist())
    finally:
        fd.fd_destroy(ctx)
