"""Calls over a paged cache that are easily forgotten: row starts out of order, infinities
among the values of a long history."""
import numpy as np
import pytest

from test_gpu_paged import DEV, Setup, attention_reference, check_attention, dt, plan, weight_step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    import torch
    import paper_2510_25739_amd as H
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return H


STARTS = {3: [[0, 90, 0, 5], [100, 60, 30, 0], [-2 ** 31, 2 ** 31 - 1, -1, 100], [50, 1000, 16, 99]],
          100: [list(range(100, -1, -1)), [0, 90] * 50 + [100], [(37 * i) % 131 - 10 for i in range(101)], [2 ** 31 - 1, -5] * 50 + [7]]}


@pytest.mark.parametrize("n_seq,heads,tile", [(3, 2, 16), (3, 16, 128), (100, 4, 16)])
def test_row_starts_out_of_order_reach_nothing_but_the_rows(H, n_seq, heads, tile):
    # what rows get is not said; memory around them and pages of no sequence stay, and a call in order is right behind it
    import torch
    rows, hd, guard = 100, 64, 300
    each = [30, 40, 30] if n_seq == 3 else [1] * n_seq
    su = Setup(H, n_seq + heads, "bf16", 2, hd, 16, each, [20 + i % 50 for i in range(n_seq)], spare=400000 // 16)
    su.fill()
    assert su.total == rows and plan(H, su, heads)[0] == tile
    q = su.randn(rows, heads, hd)
    want = attention_reference(su, q, lambda s, i, e: e <= su.past[s] + i, hd ** -0.5)
    free = sorted(set(range(su.n_pages)) - set(su.table_np[su.table_np >= 0].tolist()))
    fresh = lambda: torch.full((rows + 2 * guard, heads, hd), 7.0, dtype=dt("bf16"), device=DEV)
    around = lambda t: bool((t[:guard] == 7).all()) and bool((t[-guard:] == 7).all())
    for starts in STARTS[n_seq]:
        row_start = torch.tensor(starts, dtype=torch.int32, device=DEV)
        for max_len in (0, 1):
            out = fresh()
            su.cache.attend(q.to(DEV), row_start, su.n_past, max_len=max_len, out=out[guard:-guard])
            assert around(out), starts
        k, v = su.k.clone(), su.v.clone()
        k[:, free], v[:, free] = 3.0, 3.0
        out = fresh()
        kv = su.randn(rows, 2, hd).to(DEV)
        H.PagedCache(k, v, su.table).append(kv, kv, row_start, su.n_past, q=q.to(DEV), q_out=out[guard:-guard])
        assert around(out) and bool((k[:, free] == 3).all()) and bool((v[:, free] == 3).all()), starts
    check_attention(su, su.cache.attend(q.to(DEV), su.row_start, su.n_past), want, "bf16", weight_step("bf16", tile))
