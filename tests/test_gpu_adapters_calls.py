"""Calls on one plan of adapters behind one another: refused ones before others, rows that are one row for all, other streams than the plan's."""
import pytest

from test_gpu_adapters import DEV, Case, H, check, shared   # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_refused_call_leaves_the_next_one_as_it_was(H):   # noqa: F811
    import torch
    c = Case(31, [5], [1], 2, 128, 4096, 264)
    assert shared(H, c)
    plan, x, a = c.plan(H), c.dev("x"), c.dev("a")
    with pytest.raises(H.HawkError):                     # a width that is no multiple of 8, of a rank and an input whose sums are shared
        plan.apply(x, a, torch.zeros(2, 100, 128, dtype=torch.bfloat16, device=DEV))
    check(c, plan.apply(x, a, c.dev("b"), base=c.dev("base"), scale=c.dev("scale")))
