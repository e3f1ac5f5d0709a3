"""Draws from rows cut by top-k, top-p and min-p against numpy in 64 bits: what is kept, which token is drawn and with which probability.

Tokens and counts are equal: decisions are taken on sums that the call holds to 2^-35 of the largest weight or better (see the header) and that
numpy rounds at 2^-52; that a border of one of these few thousand seeded draws lies between is as likely as 1e-8.  The probability, of
64-bit weights and sums, is rounded to fp32 once: half a step, and 2^-30 for the weights' own rounding."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def H():
    import torch
    import paper_2510_25739_amd as H
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return H


def draw(logits, u, T, k, p, m):
    """Token, probability, entries kept of one row; logits as stored, in fp32."""
    n = logits.size
    if not T > 0:
        ok = ~np.isnan(logits) & (logits > -np.inf)
        return (int(np.flatnonzero(ok & (logits == logits[ok].max()))[0]), 1.0, 1) if ok.any() else (-1, 0.0, 0)
    with np.errstate(all="ignore"):
        z = logits * np.float32(1.0 / np.float64(np.float32(T)))
    there = np.flatnonzero(z > -np.inf)                  # (a NaN is not)
    if there.size == 0:
        return -1, 0.0, 0
    if np.isposinf(z[there]).any():
        there = there[np.isposinf(z[there])]
        z = np.zeros(n, dtype=np.float32)
    z = z.astype(np.float64)
    order = there[np.lexsort((there, -z[there]))]
    if 1 <= k < n:
        order = order[:k]
    w = np.exp(z[order] - z[order[0]])
    c = order.size
    if p < 1:
        c = max(1, int((np.concatenate([[0.0], np.cumsum(w)[:-1]]) < float(np.float32(p)) * w.sum()).sum()))
    if m > 0:
        c = min(c, int((w >= min(float(np.float32(m)), 1.0)).sum()))
    law = np.zeros(n)
    law[order[:c]] = w[:c]
    sums = np.cumsum(law)
    j = int(np.searchsorted(sums, float(u) * sums[-1], side="right"))
    j = j if j < n else int(np.flatnonzero(law)[-1])
    return j, law[j] / sums[-1], c


def check(H, logits, u=None, T=1.0, k=0, p=1.0, m=0.0, skip=None, dtype="float32", view=None, seed=0):
    import torch
    rows, n = logits.shape
    r = np.random.RandomState(seed + rows + n)
    u = (r.randint(0, 1 << 24, rows) / float(1 << 24)).astype(np.float32) if u is None else np.asarray(u, dtype=np.float32)
    par = [np.broadcast_to(np.asarray(v, dtype=t), (rows,)).copy() for v, t in ((T, np.float32), (k, np.int32), (p, np.float32), (m, np.float32))]
    x = torch.from_numpy(logits).to(getattr(torch, dtype))
    d = view(x) if view else x.to(DEV)
    t = lambda a: torch.from_numpy(a).to(DEV)
    tok, prob, kept = H.sample_filtered(d, t(u), temperature=t(par[0]), top_k=t(par[1]), top_p=t(par[2]), min_p=t(par[3]),
                                        skip=None if skip is None else t(np.asarray(skip, dtype=np.int32)))
    tok, prob, kept, x = tok.cpu().numpy(), prob.cpu().numpy(), kept.cpu().numpy(), x.float().numpy()
    for i in range(rows):
        want = (-1, 0.0, 0) if skip is not None and skip[i] < 0 else draw(x[i], u[i], *(a[i] for a in par))
        assert (tok[i], kept[i]) == (want[0], want[2]), (i, tok[i], kept[i], prob[i], want)
        assert abs(prob[i] - want[1]) <= want[1] * (2.0 ** -24 + 2.0 ** -30), (i, prob[i], want)
    return tok, prob, kept


def logits(seed, rows, n, scale=2.5):
    return (np.random.RandomState(seed).standard_normal((rows, n)) * scale).astype(np.float32)


SIZES = [1, 2, 3, 5, 64, 1000, 4095, 4096, 4097, 9999, 16384, 16385, 40000, 65536, 65537, 70001, 200003]


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_sizes_and_types(H, n, dtype):
    rows = 8
    k = [0, 1, 2, 40, 1000, n, 2 * n, -3]
    p = [0.9, 1.0, 0.5, 0.99, 0.8, 1.0, 0.3, 0.95]
    m = [0.0, 0.0, 0.1, 0.0, 0.05, 0.2, 0.0, 0.001]
    T = [1.0, 0.7, 1.3, 0.8, 1.0, 2.0, 0.5, 0.0]
    check(H, logits(n, rows, n), T=T, k=k, p=p, m=m, dtype=dtype)


@pytest.mark.parametrize("n", [16384, 65536, 600000, 1 << 20])
def test_each_cut_alone_and_none(H, n):
    z = logits(n + 1, 6, n)
    check(H, z, k=[0, 500, 0, 0, n - 1, 0], p=[1.0, 1.0, 0.9, 1.0, 1.0, 0.999], m=[0, 0, 0, 0.02, 0, 0])


@pytest.mark.parametrize("u", [0.0, 1 - 2.0 ** -24, 0.5])
def test_first_and_last_uniform(H, u):
    check(H, logits(3, 5, 5000), u=[u] * 5, k=[0, 10, 0, 1, 100], p=[1.0, 1.0, 0.8, 1.0, 0.9])


@pytest.mark.parametrize("n", [4000, 16384, 50000, 100000])
def test_ties(H, n):
    # few values: the border of every cut lies among equal entries, more of them than are ranked against each other
    z = np.round(logits(n, 9, n, 1.0) * 2) / 2
    check(H, z, k=[7, 3000, n // 2, 0, 0, 0, 2500, 0, 17], p=[1, 1, 1, 0.5, 0.9, 0.999, 0.7, 0.1, 0.9], m=[0, 0, 0, 0, 0, 0, 0, 0.3, 0])


@pytest.mark.parametrize("n", [8192, 30000, 131072])
def test_all_alike(H, n):
    # weights of one: sums are whole numbers, and a border that is met exactly is inside
    z = np.zeros((6, n), dtype=np.float32)
    _, _, kept = check(H, z, k=[0, 100, 0, 0, n, 5000], p=[1, 1, 0.5, 0.25, 0.75, 0.5], m=[0, 0, 0, 0, 1.0, 0])
    assert list(kept) == [n, 100, n // 2, n // 4, 3 * n // 4, 2500]


@pytest.mark.parametrize("n", [2000, 16384, 90000])
def test_far_tails_and_wide_ranges(H, n):
    r = np.random.RandomState(n)
    z = (-np.exp(r.uniform(-3, 7, (7, n)))).astype(np.float32)              # down to a thousand below the maximum
    z[1] = -40 - r.uniform(0, 1, n)
    z[1, n // 3] = 0                                                          # one entry, and a bulk behind the bins' reach
    z[2] = np.linspace(-90, 0, n)
    check(H, z, k=[0, n // 2, n // 2, n - 5, 0, 300, 0], p=[0.9, 1, 1, 1, 0.999, 0.9, 1], m=[0, 0, 0, 0, 0, 0, 1e-6], T=[1, 1, 1, 1, 0.1, 3, 1])


@pytest.mark.parametrize("n", [16384, 40000, 200003, 1 << 20])
@pytest.mark.parametrize("scale", [0.01, 0.2, 1.0, 8.0])
def test_narrow_and_wide_rows(H, n, scale):
    # thousands of entries where the border lies, or all of them
    check(H, logits(n, 5, n, scale), k=[0, n // 3, 0, 5000, n // 2], p=[0.9, 1, 0.3, 0.9, 0.95], m=[0, 0, 0.3, 0, 0])


@pytest.mark.parametrize("n", [300, 16384, 70000])
def test_infinities_and_nan(H, n):
    z = logits(n, 10, n)
    z[0, :] = -np.inf
    z[1, :] = np.nan
    z[2, 1:] = -np.inf
    z[3, ::2] = np.nan
    z[4, ::3] = -np.inf
    z[5, [5, 17, 200]] = np.inf
    z[6, 100] = np.inf
    z[6, 50] = np.nan
    z[7, :] = np.inf
    z[8, 10:] = -np.inf
    z[9, ::2] = -np.inf
    k = [0, 5, 3, 50, 0, 2, 9, 100, 200, n // 2 + n // 4]
    p = [1, 0.9, 0.5, 0.9, 0.9, 1, 0.5, 0.5, 0.99, 1]
    check(H, z, k=k, p=p)
    check(H, z, T=0.0)
    check(H, z, T=[1] * 10, m=0.3)


def test_parameters_at_and_beyond_their_ends(H):
    z = logits(11, 12, 3000)
    nan, inf = float("nan"), float("inf")
    check(H, z, T=[nan, -1, inf, 1, 1, 1, 1, 1, 1, 1e-3, 100, 1], k=[0, 0, 0, -2 ** 31, 2 ** 31 - 1, 0, 0, 0, 0, 0, 0, 1],
          p=[1, 1, 1, 1, 1, 0, -1, nan, 2, 1, 1, 0.5], m=[0, 0, 0, nan, -1, 0, 0, 1, 5, 0, 0, 0])
    r, got = np.random.RandomState(2), H.sample_filtered
    import torch
    x, u = torch.from_numpy(z).to(DEV), torch.from_numpy(r.rand(12).astype(np.float32)).to(DEV)
    tok, prob, kept = got(x, u)                          # no parameters: the whole distribution
    for i in range(12):
        want = draw(z[i], u[i].item(), 1.0, 0, 1.0, 0.0)
        assert (tok[i].item(), kept[i].item()) == (want[0], want[2])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strided_and_misaligned_rows(H, dtype):
    import torch
    for n, pad, first in ((1001, 3, 1), (1000, 1, 0), (20000, 5, 3), (70000, 7, 2)):
        def view(x):
            w = torch.full((x.shape[0], n + pad), float("nan"), dtype=x.dtype, device=DEV)
            w[:, first:first + n] = x.to(DEV)
            return w[:, first:first + n]
        check(H, logits(n, 5, n), k=[0, 50, 0, 700, 0], p=[0.9, 1, 1, 0.9, 0.5], dtype=dtype, view=view)


def test_skipped_rows_and_many_rows(H):
    z = logits(12, 700, 257)
    r = np.random.RandomState(1)
    check(H, z, k=r.randint(0, 257, 700), p=r.uniform(0.2, 1.1, 700), m=r.choice([0, 0.1], 700), T=r.choice([0, 0.5, 1.0], 700), skip=r.randint(-1, 2, 700))
    import torch
    e = torch.empty(0, 10, device=DEV)
    assert H.sample_filtered(e, torch.empty(0, device=DEV))[0].shape == (0,)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n", [16384, 20001, 150000])
def test_many_alike_of_16_bits(H, n, dtype):
    # borders among thousands of equal logits whose neighbours are as near as the type has them, divided by temperatures that keep them
    # apart, bring them as near as 24 bits do, and (the last two) make them one, or numbers below the smallest of 24 bits
    import torch
    r = np.random.RandomState(n)
    t = getattr(torch, dtype)
    for centre, T in ((1.0, 1.0), (-1.99, 1.0), (0.07, 0.7), (3.0, 1.4142135), (-0.004, 0.0078), (1.0, 1e-3), (1.0, 3e37), (1.5, 3e38)):
        step = torch.finfo(t).eps * abs(centre)
        x = (centre + step * r.randint(-3, 4, (6, n))).astype(np.float32)
        x[3:] = -x[3:]
        x = torch.from_numpy(x).to(t).float().numpy()
        check(H, x, T=T, k=[0, 100, n // 2, 0, n // 3, 0], p=[0.5, 1.0, 0.7, 0.03, 1.0, 0.9], dtype=dtype)


def test_the_most_rows_there_can_be(H):
    import torch
    rows = 1 << 22                                       # more workgroups than one launch has
    r = np.random.RandomState(3)
    x = torch.from_numpy(r.randn(5).astype(np.float32)).to(DEV).repeat(rows, 1)
    u = torch.arange(rows, dtype=torch.int32, device=DEV).remainder(1 << 12).float() / (1 << 12)
    skip = torch.zeros(rows, dtype=torch.int32, device=DEV)
    skip[:-4096] = -1                                    # (one pass over u)
    token, _, kept = H.sample_filtered(x, u, skip=skip)
    want = [draw(x[0].cpu().numpy(), v, 1.0, 0, 1.0, 0.0)[0] for v in u[-4096:].cpu().numpy()]
    assert token[-4096:].tolist() == want and bool((kept[-4096:] == 5).all())
    assert bool((token[:-4096] == -1).all()) and bool((kept[:-4096] == 0).all())


def test_draws_follow_the_cut_distribution(H):
    # 2^16 draws of one row: counts within five standard deviations of what the probabilities say (one in 10^6 a token, 9 tokens)
    import torch
    z = logits(5, 1, 50, 1.5)
    n = 1 << 16
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    x = torch.from_numpy(np.repeat(z, n, 0)).to(DEV)
    tok, prob, kept = H.sample_filtered(x, torch.from_numpy(u).to(DEV), top_k=torch.full((n,), 9, dtype=torch.int32, device=DEV))
    tok, prob = tok.cpu().numpy(), prob.cpu().numpy()
    for t in np.unique(tok):
        q = float(prob[tok == t][0])
        assert abs((tok == t).sum() - n * q) <= 2                             # a regular grid of uniforms: an interval holds n q of them but for its ends
    assert np.unique(tok).size == 9 and bool((kept == 9).all())


def test_refusals_of_the_binding(H):
    import torch
    x, u = torch.zeros(4, 20, device=DEV), torch.zeros(4, device=DEV)
    i = torch.zeros(4, dtype=torch.int32, device=DEV)
    for a, kw in (((x.double(), u), {}), ((x, u[:3]), {}), ((x, u.double()), {}), ((x, None), {}), ((x[0], u), {}), ((x.t().contiguous().t(), u), {}), ((x.cpu(), u), {}),
                  ((x, u), dict(top_k=u)), ((x, u), dict(top_p=i)), ((x, u), dict(temperature=u[:1])), ((x, u), dict(skip=u)), ((x, u), dict(min_p=u.cpu())),
                  ((x[:, :0], u), {}), ((x[:1].expand(4, 20), u), {})):
        with pytest.raises(H.HawkError):
            H.sample_filtered(*a, **kw)


def test_captured_and_replayed(H):
    import torch
    n, rows = 20000, 6
    x, u = torch.zeros(rows, n, device=DEV), torch.zeros(rows, device=DEV)
    k, p = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.ones(rows, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        H.sample_filtered(x, u, top_k=k, top_p=p)
        torch.cuda.current_stream().synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = H.sample_filtered(x, u, top_k=k, top_p=p)
    for s in range(4):
        z, r = logits(40 + s, rows, n), np.random.RandomState(s)
        v, kk, pp = r.rand(rows).astype(np.float32), r.randint(0, 3000, rows).astype(np.int32), r.uniform(0.5, 1.1, rows).astype(np.float32)
        x.copy_(torch.from_numpy(z)); u.copy_(torch.from_numpy(v)); k.copy_(torch.from_numpy(kk)); p.copy_(torch.from_numpy(pp))
        eager = H.sample_filtered(x, u, top_k=k, top_p=p)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)
        for i in range(rows):
            want = draw(z[i], v[i], 1.0, kk[i], pp[i], 0.0)
            assert (out[0][i].item(), out[2][i].item()) == (want[0], want[2])
