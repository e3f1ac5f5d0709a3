"""Adapters, filtered draws and page copies whose rows, adapters and pages lie further apart than 32 bits reach, and as many rows as a plan holds."""
import numpy as np
import pytest

from test_gpu_adapters import DEV, Case, H, check, dt, i32   # noqa: F401
from test_gpu_filtered import check as check_draws, logits

pytestmark = pytest.mark.gpu

FAR = 1 << 24       # elements between rows or pages: 260 of them are beyond 2^32


def apart(t, dtype=None):
    """The rows of a tensor 2^24 elements apart, in memory that holds nothing else that counts."""
    import torch
    out = torch.empty((t.shape[0] - 1) * FAR + t.shape[1], dtype=dtype or t.dtype, device=DEV).as_strided(t.shape, (FAR, 1))
    out.copy_(t)
    return out


@pytest.mark.parametrize("x,out,rank,d_in", [("bf16", "bf16", 16, 264), ("fp16", "fp32", 128, 4096)])
def test_rows_and_adapters_far_apart(H, x, out, rank, d_in):   # noqa: F811
    import torch
    c = Case(41, [1, 200, 59], [2, 0, 1], 3, rank, d_in, 136, x, out)
    a = torch.empty((1 << 32) + (1 << 20), dtype=dt(x), device=DEV).as_strided((3, rank, d_in), (1 << 31, d_in, 1))
    b = torch.empty((1 << 32) + (1 << 20), dtype=dt(x), device=DEV).as_strided((3, 136, rank), (1 << 31, rank, 1))
    a.copy_(c.a)
    b.copy_(c.b)
    base = apart(c.base)
    y = c.plan(H).apply(apart(c.x), a, b, base=base, scale=c.dev("scale"), out=base)
    check(c, y)


@pytest.mark.parametrize("n", [1000, 20000])
def test_rows_of_logits_far_apart(H, n):   # noqa: F811
    r = np.random.RandomState(n)
    check_draws(H, logits(n, 260, n), k=r.randint(0, n, 260), p=r.uniform(0.3, 1.2, 260), m=r.choice([0, 0.05], 260), dtype="bfloat16", view=apart)


def test_pages_far_apart(H):   # noqa: F811
    import torch
    g = torch.Generator().manual_seed(1)
    pools, mirrors = [], []
    for _ in range(2):
        pool = torch.empty(263 * FAR, dtype=torch.float16, device=DEV).as_strided((1, 263, 2, 4, 8), (263 * FAR, FAR, 32, 8, 1))
        pool.copy_(torch.randn(1, 263, 2, 4, 8, generator=g))
        pools.append(pool)
        mirrors.append(pool.cpu())
    refs, table = np.ones(263), np.full((2, 3), -1)
    refs[[0, 5, 258, 261]] = 0                            # two free pages before and one behind what 32 bits reach, and the last but one
    table[0] = [262, 260, 259]
    table[1] = [262, -1, -1]
    refs[262] = 2
    t, c_refs, past = i32(table), i32(refs), i32([12, 3])
    cache = H.PagedCache(*pools, t)
    cache.copy_pages(i32([260, 1]), i32([258, 261]))
    for m in mirrors:
        m[:, [258, 261]] = m[:, [260, 1]]
    assert cache.take(c_refs, past, i32([0, 9])).tolist() == [0, 0]       # 262 has another holder: its three entries go to page 0; then 5 and 258
    for m in mirrors:
        m[:, 0, :, :3] = m[:, 262, :, :3]
    assert t.tolist() == [[262, 260, 259], [0, 5, 258]]
    c_refs[[1, 2]] = 0                                    # (nobody's)
    new, counts, used = cache.compact(c_refs)
    # in use: all but 1, 2 and 261; 260 and 262 go to 1 and 2
    assert used.item() == 260 and new.tolist() == [[2, 1, 259], [0, 5, 258]]
    for m in mirrors:
        m[:, 1], m[:, 2] = m[:, 260], m[:, 262]
    for pool, m in zip(pools, mirrors):
        assert torch.equal(pool.cpu(), m)


def test_the_most_rows_of_a_plan(H):   # noqa: F811
    # 2^22 rows of six sequences; every row's result is its adapter's number but for two that are compared in full
    import torch
    rows = 1 << 22
    start = [0, 5, 1 << 20, (1 << 20) + 1, 3 << 20, rows - 7, rows]
    adapter = [1, 0, -1, 2, 1, 0]
    x = torch.zeros(rows, 8, dtype=torch.bfloat16, device=DEV)
    x[:, 0] = torch.arange(rows, device=DEV).remainder(251).to(torch.bfloat16)
    a = torch.zeros(3, 8, 8, dtype=torch.bfloat16, device=DEV)
    a[:, 3, 0] = 1
    b = torch.zeros(3, 8, 8, dtype=torch.bfloat16, device=DEV)
    b[0, 1, 3], b[1, 2, 3], b[2, 7, 3] = 1, 2, -1
    y = H.AdapterPlan(i32(start), i32(adapter), rows, 3).apply(x, a, b)
    want = torch.zeros_like(y)
    for s, i in enumerate(adapter):
        if i >= 0:
            col, w = [(1, 1), (2, 2), (7, -1)][i]
            want[start[s]:start[s + 1], col] = x[start[s]:start[s + 1], 0] * w
    assert torch.equal(y, want)
