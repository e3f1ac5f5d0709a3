"""Calls on one plan of adapters behind one another: refused ones before others, rows that are one row for all, other streams than the plan's."""
import pytest

from test_gpu_adapters import DEV, Case, H, check, dt, i32, shared   # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_refused_call_leaves_the_next_one_as_it_was(H):   # noqa: F811
    import torch
    c = Case(31, [5], [1], 2, 128, 4096, 264)
    assert shared(H, c)
    plan, x, a = c.plan(H), c.dev("x"), c.dev("a")
    with pytest.raises(H.HawkError):                     # a width that is no multiple of 8, of a rank and an input whose sums are shared
        plan.apply(x, a, torch.zeros(2, 100, 128, dtype=torch.bfloat16, device=DEV))
    check(c, plan.apply(x, a, c.dev("b"), base=c.dev("base"), scale=c.dev("scale")))


def test_a_plan_that_is_dropped_while_another_stream_works_with_it(H):   # noqa: F811
    # the other stream is busy, the plan goes, and what takes its memory is written at once on the plan's own stream
    import torch
    c = Case(32, [1, 6, 0, 17, 33, 2], [2, 0, 1, -1, 2, 1], 3, 16, 264, 136)
    x, a, b, base, scale = (c.dev(k) for k in ("x", "a", "b", "base", "scale"))
    side = torch.cuda.Stream()
    for how in ("apply", "update"):
        plan = c.plan(H)
        out, start, adapter = base.clone(), i32(c.start), i32(c.adapter)
        n = plan._plan.numel()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(int(2e7))                  # some ms
            if how == "update":
                plan.update(start, adapter)
            plan.apply(x, a, b, base=base, scale=scale, out=out)
        del plan
        others = [torch.full((n,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]
        torch.cuda.synchronize()
        check(c, out)
        assert all(bool((t == 255).all()) for t in others)


def test_a_plan_captured_on_another_stream_and_replayed(H):   # noqa: F811
    import torch
    c = Case(33, [6, 6, 2], [1, -1, 0], 2, 16, 512, 264)
    plan, x, a, b, base, scale = c.plan(H), *(c.dev(k) for k in ("x", "a", "b", "base", "scale"))
    eager = plan.apply(x, a, b, base=base, scale=scale)
    check(c, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                        # (captures on a stream of its own)
        out = plan.apply(x, a, b, base=base, scale=scale)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    del graph, plan
    torch.cuda.synchronize()


def test_inputs_of_one_row_for_all(H):   # noqa: F811
    # x and base with a row stride of zero
    c = Case(34, [3, 20, 4], [1, 0, -1], 2, 24, 72, 136)
    c.x[1:], c.base[1:] = c.x[:1].clone(), c.base[:1].clone()
    x, base = c.dev("x")[:1].expand(27, 72), c.dev("base")[:1].expand(27, 136)
    check(c, c.plan(H).apply(x, c.dev("a"), c.dev("b"), base=base, scale=c.dev("scale")))
    check(c, c.plan(H).apply(x, c.dev("a"), c.dev("b"), base=c.dev("base"), scale=c.dev("scale")))


def test_columns_of_one_buffer(H):   # noqa: F811
    # x, base and out side by side in one: nothing overlaps
    import torch
    c = Case(35, [3, 20, 4], [1, 0, -1], 2, 16, 64, 48, extra=2)
    one = torch.full((c.total, 64 + 48 + 48 + 8), 9.0, dtype=torch.bfloat16, device=DEV)
    one[:, :64], one[:, 112:160] = c.dev("x"), c.dev("base")
    was = one.clone()
    c.plan(H).apply(one[:, :64], c.dev("a"), c.dev("b"), base=one[:, 112:160], scale=c.dev("scale"), out=one[:, 64:112])
    check(c, one[:, 64:112], was[:, 64:112].cpu())
    was[:, 64:112] = one[:, 64:112]
    assert torch.equal(one, was)
    with pytest.raises(H.HawkError):
        c.plan(H).apply(one[:, :64], c.dev("a"), c.dev("b"), out=one[:, 56:104])
    with pytest.raises(H.HawkError):
        c.plan(H).apply(one[:, :64], c.dev("a"), c.dev("b"), base=one[:, 112:160], out=one[:, 104:152])


@pytest.mark.parametrize("out", ["fp16", "fp32"])
@pytest.mark.parametrize("where", ["x", "weights", "parts"])
def test_small_halves(H, out, where):   # noqa: F811
    # numbers below the smallest normal half: in x, in both weights, and as the second parts of A x in a row with one large value
    c = Case(36, [5, 18], [0, 1], 2, 16, 256, 72, "fp16", out, base=False, spread=2.0 ** -16 if where == "x" else 1.0)
    if where == "weights":
        c.a, c.b = (c.a.float() * 2.0 ** -13).to(c.a.dtype), (c.b.float() * 2.0 ** -17).to(c.b.dtype)
        c.scale = c.scale * 2.0 ** 20
    elif where == "parts":
        c.a[:, 1:] = (c.a[:, 1:].float() * 2.0 ** -13).to(c.a.dtype)
        c.a[:, 0] = (c.a[:, 0].float() * 2.0 ** 12).to(c.a.dtype)
        c.b[:, :, 0] = 0                                 # (the large one has no part in the result)
    check(c, c.plan(H).apply(c.dev("x"), c.dev("a"), c.dev("b"), scale=c.dev("scale"), dtype=dt(out)))
