"""Counts below zero are free pages, for all calls alike."""
import numpy as np
import pytest

from test_gpu_pages import DEV, H, i32   # noqa: F401

pytestmark = pytest.mark.gpu

# of 45 pages; thread 0 and 1 of a take look at sixteen counts each, thread 2 at what is left
COUNTS = [1, -1, 0, -7, 1, -2 ** 31] + [1] * 10 + [-1, 1] * 8 + [1, 0, -3, 1, 1, -1, 1, 1, 1, 1, -2, 1, 1]


def cache_of(H, table):   # noqa: F811
    import torch
    g = torch.Generator().manual_seed(2)
    pools = [torch.randn(2, len(COUNTS), 2, 4, 8, generator=g).to(DEV) for _ in range(2)]
    return H.PagedCache(*pools, table), [p.clone() for p in pools]


def test_pages_of_negative_counts_are_taken(H):   # noqa: F811
    free = [p for p, n in enumerate(COUNTS) if n <= 0]
    table = np.full((3, 8), -1)
    table[0, 0] = 0
    t, refs, past = i32(table), i32(COUNTS), i32([3, 0, 0])
    cache, _ = cache_of(H, t)
    n = len(free)
    want = [1 + 4 * 2, 4 * 8, 4 * (n - 10)]               # 2, 8 and all other free pages
    short = cache.take(refs, past, i32(want))
    assert short.tolist() == [0, 0, 0]
    for s, (first, k) in enumerate(((1, 2), (0, 8), (0, n - 10))):
        table[s, first:first + k] = free[:k]
        del free[:k]
    assert not free and t.tolist() == table.tolist()
    assert refs.tolist() == [max(x, 0) or 1 for x in COUNTS]
    assert cache.take(refs, i32([0, 32, 31]), i32([0, 0, 1])).tolist() == [0, 0, 1]


@pytest.mark.parametrize("in_place", [False, True])
def test_compaction_leaves_no_negative_counts(H, in_place):   # noqa: F811
    import torch
    used = [p for p, n in enumerate(COUNTS) if n > 0]
    table = np.full((len(used) + 1, 1), -1)
    table[:-1, 0] = used
    table[-1, 0] = 3                                      # a place whose page is not in use
    t, refs = i32(table), i32(COUNTS)
    cache, old = cache_of(H, t)
    new, counts, n = cache.compact(refs, table=t, refs_out=refs) if in_place else cache.compact(refs)
    assert n.item() == len(used)
    assert counts.tolist() == [1] * len(used) + [0] * (len(COUNTS) - len(used))
    assert sorted(new[:-1, 0].tolist()) == list(range(len(used))) and new[-1, 0].item() == -1
    for pool, before in zip((cache.k, cache.v), old):
        assert torch.equal(pool[:, new[:-1, 0].long()], before[:, torch.tensor(used, device=DEV)])
