"""Low-rank adapters of many requests against plain float64 arithmetic, at ranks, widths, strides and groupings where they can go wrong.

Tolerances: a value rounded to a type is off by at most half a step, finfo(type).eps / 2 of it; fp32 sums of n terms are off by n 2^-24
of the terms' absolute sum at most.  A x, of d_in terms (and eight partial sums), enters the second product off by 2^-16 (bf16 operands; 2^-24
for results of 32 bits), 2^-22 of itself and 2^-38 of its row's largest (fp16), nothing (fp32)."""
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


def dt(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


class Case:
    """Inputs on the CPU in their types, and what a call has to give with how far it may be off."""

    def __init__(self, seed, rows, adapter, n_adapters, rank, d_in, d_out, x="bf16", out="bf16", base=True, scale=True, extra=0, spread=1.0):
        import torch
        self.g = torch.Generator().manual_seed(seed)
        self.adapter, self.n, self.rank, self.d_in, self.d_out = list(adapter), n_adapters, rank, d_in, d_out
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.total = int(self.start[-1]) + extra
        self.tx, self.tout = x, out
        r = lambda *s: torch.randn(*s, generator=self.g)
        self.x = (r(self.total, d_in) * spread).to(dt(x))
        self.a = (r(n_adapters, rank, d_in) * max(d_in, 1) ** -0.5).to(dt(x))
        self.b = (r(n_adapters, d_out, rank) * rank ** -0.5).to(dt(x))
        self.base = r(self.total, d_out).to(dt(out)) if base else None
        self.scale = 0.5 + torch.rand(n_adapters, generator=self.g) if scale else None

    def owner(self):
        """The adapter of every row, -1: none, -2: no sequence (the last sequence that starts at or before the row, if it goes as far)."""
        out = np.full(self.total, -2)
        for r in range(self.total):
            s = int(np.searchsorted(self.start[:-1], r, side="right")) - 1
            if s >= 0 and r < self.start[s + 1]:
                out[r] = self.adapter[s] if 0 <= self.adapter[s] < self.n else -1
        return out

    def expected(self):
        import torch
        who = self.owner()
        y = self.base.double().clone() if self.base is not None else torch.zeros(self.total, self.d_out, dtype=torch.float64)
        off = torch.zeros_like(y)
        for i in range(self.n):
            rows = torch.from_numpy(np.flatnonzero(who == i))
            if rows.numel() == 0:
                continue
            x, a, b = self.x[rows].double(), self.a[i].double(), self.b[i].double()
            h, size = x @ a.T, x.abs() @ a.abs().T
            part = {"bf16": h.abs() * (2.0 ** -24 if self.tout == "fp32" else 2.0 ** -16),
                    "fp16": h.abs() * 2.0 ** -22 + h.abs().amax(1, keepdim=True) * 2.0 ** -38, "fp32": 0 * h}[self.tx]
            eh = part * 1.01 + (self.d_in + 10) * 2.0 ** -24 * size
            s = float(self.scale[i]) if self.scale is not None else 1.0
            y[rows] += s * (h @ b.T)
            off[rows] += s * ((eh @ b.abs().T) + (3 * self.rank + 6) * 2.0 ** -24 * (h.abs() @ b.abs().T))
        off += 2.0 ** -23 * y.abs()
        off = off * 1.01 + torch.finfo(dt(self.tout)).eps / 2 * (y.abs() + off) + torch.finfo(dt(self.tout)).tiny * torch.finfo(dt(self.tout)).eps
        return y, off, who

    def dev(self, name):
        t = getattr(self, name)
        return None if t is None else t.to(DEV)

    def plan(self, H):
        return H.AdapterPlan(i32(self.start), i32(self.adapter), self.total, self.n)


def check(case, got, untouched=None):
    import torch
    y, off, who = case.expected()
    got = got.double().cpu()
    for r in np.flatnonzero(who == -2):
        assert untouched is None or torch.equal(got[r], untouched[r].double()), r
    rows = torch.from_numpy(np.flatnonzero(who != -2))
    worst = ((got - y).abs() / off.clamp(min=1e-300))[rows]
    assert rows.numel() == 0 or bool((worst <= 1).all()), float(worst.max())
    none = torch.from_numpy(np.flatnonzero(who == -1))
    assert torch.equal(got[none], y[none])               # what is only copied is copied


RANKS = [8, 16, 24, 32, 40, 64, 72, 128]


@pytest.mark.parametrize("x,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32"), ("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp16")])
@pytest.mark.parametrize("rank", RANKS)
def test_types_and_ranks(H, x, out, rank):
    c = Case(rank, [1, 6, 0, 17, 33, 2], [2, 0, 1, -1, 2, 1], 3, rank, 264, 136, x, out)
    check(c, c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale")))


@pytest.mark.parametrize("d_in,d_out", [(8, 8), (16, 72), (32, 64), (40, 1000), (256, 56), (1288, 8), (4096, 520), (11008, 128)])
@pytest.mark.parametrize("x", ["bf16", "fp32"])
def test_widths(H, d_in, d_out, x):
    c = Case(d_in + d_out, [3, 20], [0, 1], 2, 16, d_in, d_out, x, x)
    check(c, c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale")))


@pytest.mark.parametrize("rows,adapter,n", [([1], [0], 1), ([0], [0], 1), ([5], [-1], 2), ([1] * 300, None, 7), ([1] * 64, None, 64), ([2000], [3], 4),
                                            ([700, 0, 1, 1300], [1, 0, 1, 0], 2), ([3, 4], [0, 2 ** 31 - 1], 2), ([3, 4], [-2 ** 31, 1], 2),
                                            ([1] * 1500, None, 3), ([16, 16, 16], [0, 0, 0], 1), ([15, 1, 17], [1, 1, 1], 2), ([2, 2], [0, 0], 8192)])
def test_groupings(H, rows, adapter, n):
    if adapter is None:
        adapter = np.random.RandomState(len(rows)).randint(-1, n, len(rows))
    c = Case(len(rows) + n, rows, adapter, n, 8, 64, 40)
    check(c, c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale")))


def shared(H, c):
    """Whether a tile's sum over d_in is shared by several workgroups (two launches)."""
    import ctypes
    from paper_2510_25739_amd import hawk
    w = hawk.HawkAdapters(dtype=hawk._dtype_of(c.a), n_adapters=c.n, rank=c.rank, d_in=c.d_in, d_out=c.d_out)
    return H.load_library().hawk_adapter_apply_workspace_bytes(ctypes.byref(w), c.total) > 0


WIDE = [("bf16", "bf16", 128, 4096, 264), ("bf16", "fp32", 64, 11008, 72), ("bf16", "bf16", 32, 12296, 1000), ("fp16", "fp16", 120, 5000, 136),
        ("fp16", "fp32", 64, 8192, 40), ("fp32", "fp32", 40, 8200, 264), ("fp32", "bf16", 128, 2056, 200), ("bf16", "fp16", 16, 40000, 64)]


@pytest.mark.parametrize("x,out,rank,d_in,d_out", WIDE)
@pytest.mark.parametrize("rows,adapter,n", [([1], [0], 1), ([1, 6, 0, 17, 33, 2], [2, 0, 1, -1, 2, 1], 3), ([200, 130], [1, 0], 2)])
def test_sums_that_workgroups_share(H, x, out, rank, d_in, d_out, rows, adapter, n):
    c = Case(rank + d_in, rows, adapter, n, rank, d_in, d_out, x, out, extra=3)
    assert shared(H, c)
    kept = c.dev("base")
    got = c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=kept, scale=c.dev("scale"), out=kept)
    check(c, got, c.base)


def test_shared_sums_on_two_streams_and_replayed(H):
    import torch
    cs = [Case(s, [1, 6, 3], [1, 0, 1], 2, 128, 4096, 264) for s in (1, 2)]
    assert all(shared(H, c) for c in cs)
    plan = cs[0].plan(H)                                 # both have the same rows: one plan
    dev = [[c.dev(k) for k in ("x", "a", "b", "base", "scale")] for c in cs]
    run = lambda d: plan.apply(d[0], d[1], d[2], base=d[3], scale=d[4])
    one = [run(d) for d in dev]
    for c, y in zip(cs, one):
        check(c, y)
    streams = [torch.cuda.Stream() for _ in dev]
    torch.cuda.synchronize()
    many = [[], []]
    for _ in range(20):
        for s, d, m in zip(streams, dev, many):
            with torch.cuda.stream(s):
                m.append(run(d))
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for m, w in zip(many, one) for y in m)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [run(d) for d in dev]
    for _ in range(3):
        for y in outs:
            y.zero_()
        graph.replay()
        again = run(dev[0])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], one[0]) and torch.equal(outs[1], one[1]) and torch.equal(again, one[0])


@pytest.mark.parametrize("base,scale", [(True, False), (False, True), (False, False)])
def test_without_a_base_or_a_scale(H, base, scale):
    c = Case(5, [4, 30, 9], [1, -1, 0], 2, 16, 128, 200, base=base, scale=scale)
    check(c, c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale")))


def test_no_adapters_and_no_rows(H):
    import torch
    c = Case(6, [4, 3], [0, -1], 0, 8, 32, 40)
    check(c, c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base")))
    plan = H.AdapterPlan(i32([0]), i32([]), 0, 2)
    e = torch.empty(0, 32, dtype=torch.bfloat16, device=DEV)
    assert plan.apply(e, torch.zeros(2, 8, 32, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 40, 8, dtype=torch.bfloat16, device=DEV)).shape == (0, 40)


def test_in_place_and_rows_behind_the_last_sequence(H):
    c = Case(7, [6, 1, 40], [1, -1, 0], 2, 16, 256, 96, extra=5)
    y = c.dev("base")
    assert c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=y, scale=c.dev("scale"), out=y) is y
    check(c, y, untouched=c.base)
    out = c.dev("base") * 0 + 3
    c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale"), out=out)
    check(c, out, untouched=out.cpu() * 0 + 3)


def test_strided_rows_and_weights(H):
    import torch
    c = Case(8, [6, 21], [1, 0], 2, 24, 120, 72)
    wide = torch.full((27, 120 + 40), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:128] = c.dev("x")
    out = torch.full((27, 200), 7.0, dtype=torch.bfloat16, device=DEV)
    base = torch.full((27, 88), float("nan"), dtype=torch.bfloat16, device=DEV)
    base[:, 16:] = c.dev("base")
    # the weights of one layer and one projection of several in a pool
    a = torch.full((2, 3, 24, 136), float("nan"), dtype=torch.bfloat16, device=DEV)
    a[:, 1, :, 8:128] = c.dev("a")
    b = torch.full((2, 5, 72, 40), float("nan"), dtype=torch.bfloat16, device=DEV)
    b[:, 4, :, 16:] = c.dev("b")
    c.plan(H).apply(wide[:, 8:128], a[:, 1, :, 8:128], b[:, 4, :, 16:], base=base[:, 16:], scale=c.dev("scale"), out=out[:, 64:136])
    check(c, out[:, 64:136])
    assert bool((out[:, :64] == 7).all()) and bool((out[:, 136:] == 7).all())


def test_what_a_row_holds_stays_in_it(H):
    import torch
    # infinities and NaN in rows of a tile, in rows without an adapter, and in adapters that nobody has
    c = Case(9, [4, 3, 5], [0, -1, 2], 3, 16, 128, 64, "fp16", "fp32")
    clean = c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale"))
    c.x[1, 3], c.x[4:7], c.x[8, 0] = float("inf"), float("nan"), float("nan")
    c.a[1], c.b[1] = float("nan"), float("inf")
    got = c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale"))
    rows = [0, 2, 3, 7, 9, 10, 11]
    assert torch.equal(got[rows], clean[rows]) and torch.equal(got[4:7], c.dev("base")[4:7])
    assert bool(got[8].isnan().all()) and not bool(got[1].isfinite().any())


@pytest.mark.parametrize("x", ["bf16", "fp16"])
def test_an_infinite_intermediate_value_is_infinite_and_has_its_sign(H, x):
    import torch
    c = Case(10, [1], [0], 1, 8, 64, 40, x, "fp32", base=False, scale=False)
    c.x[0, 5] = float("inf")
    c.a[0, 1:] = 0
    c.a[0, 1:, 5] = 1.0
    got = c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b")).cpu().double()[0]
    h = torch.where(c.a[0, :, 5] > 0, float("inf"), float("-inf")).double()
    want = c.b[0].double() @ h
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~want.isnan()], want[~want.isnan()])


def test_large_and_small_intermediate_values_of_halves(H):
    # A x up to 2^22 and down to 2^-20 in one batch: beyond what a half holds
    for spread in (30000.0, 2.0 ** -14):
        c = Case(11, [5, 20], [0, 1], 2, 16, 2048, 48, "fp16", "fp32", spread=1.0)
        c.x = (c.x.float() * spread).clamp(-60000, 60000).to(c.x.dtype)
        c.a = (c.a.float() * 40).to(c.a.dtype)
        check(c, c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale")))


def test_row_starts_that_do_not_ascend_lead_nowhere_else(H):
    c = Case(12, [5, 3, 8], [0, 1, 0], 2, 8, 64, 40)
    c.start = np.array([0, 9, 4, 16], dtype=np.int32)
    who = np.full(16, -2)
    for r in range(16):                                  # the search of the plan over starts 0, 9, 4
        lo, hi = 0, 3
        while lo < hi:
            mid = (lo + hi) // 2
            lo, hi = (mid + 1, hi) if c.start[mid] <= r else (lo, mid)
        if r < c.start[lo]:
            who[r] = c.adapter[lo - 1]
    c.owner = lambda: who
    y = c.dev("base")
    c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), base=y, scale=c.dev("scale"), out=y)
    check(c, y, untouched=c.base)


def test_refusals_of_the_binding(H):
    import torch
    c = Case(13, [4], [0], 2, 8, 64, 40)
    p, x, a, b, y = c.plan(H), c.dev("x"), c.dev("a"), c.dev("b"), c.dev("base")
    bad = [dict(x=x[:3]), dict(x=x[:, :56]), dict(x=x.float()), dict(a=a[:1]), dict(b=b[:, :, :4]), dict(a=a.float()), dict(b=b.transpose(1, 2)),
           dict(base=y.float(), out=y), dict(base=y[:, :32]), dict(scale=torch.ones(3, device=DEV)), dict(scale=torch.ones(2, dtype=torch.float64, device=DEV)),
           dict(out=torch.empty(4, 48, dtype=torch.bfloat16, device=DEV)), dict(x=x.cpu()), dict(a=a[:, :, 1:57]), dict(x=x.t().contiguous().t())]
    for kw in bad:
        with pytest.raises(H.HawkError):
            p.apply(**{**dict(x=x, a=a, b=b, base=y), **kw})
    with pytest.raises(H.HawkError):
        p.update(i32([0, 4]), i32([0, 0]))
    with pytest.raises(H.HawkError):
        H.AdapterPlan(i32([0, 4]).long(), i32([0]), 4, 2)


def test_captured_with_its_plan_and_replayed_on_other_batches(H):
    import torch
    c = Case(14, [6, 6, 6, 2], [0, 1, -1, 2], 3, 16, 512, 264)
    start, adapter, x, y = i32(c.start), i32(c.adapter), c.dev("x"), c.dev("base")
    a, b, s = c.dev("a"), c.dev("b"), c.dev("scale")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan = H.AdapterPlan(start, adapter, c.total, c.n)
        out = plan.apply(x, a, b, base=y, scale=s)       # on a stream that is not the default one
        torch.cuda.current_stream().synchronize()
        check(c, out)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            plan.update(start, adapter)
            plan.apply(x, a, b, base=y, scale=s, out=out)
    torch.cuda.synchronize()
    for k, (rows, who) in enumerate([([6, 6, 6, 2], [2, 2, 2, 2]), ([20, 0, 0, 0], [1, 0, 0, 0]), ([1, 1, 1, 17], [0, -1, 7, 1])]):
        n = Case(20 + k, rows, who, 3, 16, 512, 264)
        n.a, n.b, n.scale = c.a, c.b, c.scale
        start.copy_(i32(n.start)); adapter.copy_(i32(n.adapter)); x.copy_(n.x); y.copy_(n.base)
        g.replay()
        torch.cuda.synchronize()
        check(n, out)
