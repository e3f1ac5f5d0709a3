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


HISTORIES = [
    # cache, heads, kv_heads, hd, page, rows, past, rows of a tile, in parts?, scale of the keys
    ("bf16", 4, 2, 64, 16, [3, 1], [700, 90], 16, False, 1.0),
    ("fp16", 4, 2, 64, 6, [3, 1], [700, 90], 16, False, 1.0),
    ("fp32", 4, 2, 64, 16, [3, 1], [700, 90], 16, False, 1.0),
    ("bf16", 8, 2, 128, 16, [4], [2100], 16, True, 1.0),
    ("fp16", 2, 2, 200, 16, [4], [2100], 16, True, 1.0),
    ("fp32", 2, 2, 80, 5, [4], [2100], 16, True, 1.0),
    ("bf16", 4, 2, 64, 16, [3, 1], [700, 90], 16, False, 30.0),      # weights that are zero in 32 bits
    ("fp32", 4, 2, 96, 16, [3], [700], 16, None, 30.0),
    ("bf16", 8, 2, 128, 16, [4], [2100], 16, True, 30.0),            # whole parts of weights that are zero
    ("fp16", 24, 2, 64, 16, [9], [1500], 128, True, 1.0),
    ("bf16", 24, 2, 128, 6, [9], [1500], 128, True, 30.0),
    ("fp16", 24, 2, 200, 16, [9], [1500], 128, True, 1.0),
    ("bf16", 64, 8, 64, 16, [70, 64] * 5, [300, 90] * 5, 128, False, 1.0),
    ("fp16", 32, 2, 64, 16, [150, 131] * 10, [340, 300] * 10, 256, None, 30.0),
]


@pytest.mark.parametrize("cache,heads,kv_heads,hd,page,rows,past,tile,parts,scale", HISTORIES)
def test_infinities_and_nan_of_a_history(H, cache, heads, kv_heads, hd, page, rows, past, tile, parts, scale):
    # wherever they lie and whatever follows: an infinity is in the result of every row that sees it, both signs and NaN are NaN, and no
    # other feature changes
    import torch
    su = Setup(H, hd + page + sum(rows), cache, kv_heads, hd, page, rows, past, spare=400000 // page)
    su.fill(scale=scale)
    most = max(p + n for p, n in zip(past, rows))
    max_len = 0 if parts or tile > 16 else most
    cut = plan(H, su, heads, max_len)
    assert cut[0] == tile and parts in (None, cut[2] > 1)
    q = su.randn(su.total, heads, hd)
    inf, nan = float("inf"), float("nan")
    # entry, cache head, feature, value; in every sequence
    bad = [(0, 0, 1, inf), (3, 0, 2, -inf), (17, 0, 5, nan), (20, 0, 7, inf), (70, 0, 7, -inf), (33, 0, 11, inf), (60, 0, 11, inf), (64, 1, hd - 1, -inf),
           (past[0] // 2, 1, 3, inf), (past[0] - 1, 0, 13, -inf), (past[0], 0, 14, inf)]
    group, want = heads // kv_heads, {}
    for s, (n, p) in enumerate(zip(rows, past)):
        for e, h, f, x in bad:
            if e >= p + n:
                continue
            pg, sl = su.where(s, e)
            su.v[0, pg, h, sl, f] = x
            for i in range(n):
                if e <= p + i:
                    for g in range(group):
                        key = (int(su.start_np[s]) + i, h * group + g, f)
                        want[key] = want.get(key, 0.0) + x
    out = su.cache.attend(q.to(DEV), su.row_start, su.n_past, max_len=max_len).double().cpu()
    clean = torch.ones(out.shape, dtype=torch.bool)
    for key, x in want.items():
        clean[key] = False
        got = float(out[key])
        assert got == x or (got != got and x != x), (key, x, got)
    o, m, er = attention_reference(su, q, lambda s, i, e: e <= past[s] + i, hd ** -0.5)
    keep = lambda t: torch.where(clean, t, torch.zeros((), dtype=torch.float64))
    check_attention(su, keep(out), (keep(o), m, er), cache, weight_step(cache, tile))


@pytest.mark.parametrize("cache,heads,rows,past,tile", [("bf16", 2, [3], [200], 16), ("fp16", 2, [3], [2100], 16), ("fp32", 2, [3], [2100], 16),
                                                        ("bf16", 24, [9], [1500], 128), ("fp16", 24, [9], [90], 128)])
def test_rows_of_which_every_score_is_minus_infinity_give_zeros(H, cache, heads, rows, past, tile):
    # among finite values, and among infinities and NaN: a weight of nothing is not a small weight
    import torch
    su = Setup(H, 11, cache, 2, 64, 16, rows, past, spare=400000 // 16)
    su.fill()
    assert plan(H, su, heads)[0] == tile
    q = su.randn(su.total, heads, 64)
    q[:, :, 9] = q[:, :, 9].abs() + 1
    q[0, :, 9] = 0.5
    for e in range(past[0] + rows[0]):
        pg, sl = su.where(0, e)
        su.k[0, pg, :, sl, 9] = float("-inf")
    for odd in (False, True):
        if odd:
            for e, f, x in ((1, 3, float("inf")), (64, 4, float("nan")), (past[0], 5, float("-inf")), (past[0] - 1, 63, float("inf"))):
                pg, sl = su.where(0, e)
                su.v[0, pg, :, sl, f] = x
        for max_len in (0, past[0] + rows[0]):
            out = su.cache.attend(q.to(DEV), su.row_start, su.n_past, max_len=max_len)
            assert bool((out == 0).all()), odd


@pytest.mark.parametrize("cache,heads", [("bf16", 2), ("fp16", 2), ("fp32", 2), ("bf16", 24)])
def test_a_score_that_is_nan_or_plus_infinity_is_nan_whatever_the_values(H, cache, heads):
    import torch
    past = 1500
    for key in (float("nan"), float("inf")):
        su = Setup(H, 12, cache, 2, 64, 16, [9], [past], spare=400000 // 16)
        su.fill()
        q = su.randn(9, heads, 64)
        q[:, :, 9] = q[:, :, 9].abs() + 1
        pg, sl = su.where(0, 40)
        su.k[0, pg, 0, sl, 9] = key
        for e, x in ((3, float("inf")), (past + 1, float("-inf"))):
            pg, sl = su.where(0, e)
            su.v[0, pg, :, sl, 5] = x
        out = su.cache.attend(q.to(DEV), su.row_start, su.n_past)
        assert bool(out[:, :heads // 2].isnan().all())
        other = out[:, heads // 2:]
        assert bool((other[0, :, 5] == float("inf")).all()) and bool(other[1:, :, 5].isnan().all()) and int(other.isnan().sum()) == 8 * (heads // 2)


LARGE = [
    # cache, heads, kv_heads, hd, page, rows, past, rows of a tile, log2 of the largest query and key
    ("bf16", 2, 2, 64, 16, [9], [700], 16, 20, 18),
    ("fp16", 2, 2, 128, 16, [9], [2100], 16, 15, 15),
    ("fp32", 2, 2, 96, 6, [9], [700], 16, 20, 18),
    ("bf16", 48, 2, 64, 16, [9], [1500], 128, 20, 18),
    ("bf16", 48, 2, 128, 6, [9], [1500], 128, 26, 20),
    ("fp16", 48, 2, 128, 16, [9], [1500], 128, 15, 15),
    ("fp16", 48, 2, 200, 16, [9], [1500], 128, 13, 13),
    ("bf16", 64, 8, 64, 16, [70, 64] * 5, [300, 90] * 5, 128, 18, 14),
    ("fp16", 32, 2, 64, 16, [150, 131] * 10, [340, 300] * 10, 256, 15, 15),
]


@pytest.mark.parametrize("cache,heads,kv_heads,hd,page,rows,past,tile,q_log,k_log", LARGE)
def test_scores_of_which_one_step_is_more_than_a_power_of_two(H, cache, heads, kv_heads, hd, page, rows, past, tile, q_log, k_log):
    # One feature makes the score, so that it is exact, and two scores of a large query are equal or far apart: the weights are one (or a few
    # equal ones) and zero.  Queries of ordinary size lie between them, in the same tile.
    import torch
    su = Setup(H, hd + tile, cache, kv_heads, hd, page, rows, past, spare=400000 // page)
    su.fill()
    assert plan(H, su, heads)[0] == tile
    for s, K in enumerate(su.K):
        K.zero_()
        K[:, :, 5] = (torch.randn(len(K), kv_heads, generator=su.g) * 2.0 ** (k_log - 2)).clamp(-2.0 ** k_log, 2.0 ** k_log).to(dt(cache)).double()
        e = torch.arange(len(K))
        pg = torch.from_numpy(su.table_np[s].astype(np.int64))[e // page]
        su.k[0].index_put_((pg.to(DEV)[:, None], torch.arange(kv_heads, device=DEV)[None], (e % page).to(DEV)[:, None]), K.to(dt(cache)).to(DEV))
    q = su.randn(su.total, heads, hd)
    large = torch.rand(su.total, heads, generator=su.g) < 0.6
    sign = torch.where(torch.rand(su.total, heads, generator=su.g) < 0.5, -1.0, 1.0)
    q[:, :, 5] = (sign * torch.where(large, 2.0 ** q_log, 2.0 ** (1 - k_log))).to(dt(cache))
    o, m, er = attention_reference(su, q, lambda s, i, e: e <= past[s] + i, hd ** -0.5)
    er = torch.where(large[..., None], torch.zeros((), dtype=torch.float64), er)
    for max_len in (0, max(p + n for p, n in zip(past, rows))):
        got = su.cache.attend(q.to(DEV), su.row_start, su.n_past, max_len=max_len)
        check_attention(su, got, (o, m, er), cache, weight_step(cache, plan(H, su, heads, max_len)[0]))
