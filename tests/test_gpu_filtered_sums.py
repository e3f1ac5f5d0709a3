"""Sums of many small weights next to a top-p's border in rows of parts."""
import math
from fractions import Fraction

import numpy as np
import pytest

from test_gpu_filtered import DEV, H   # noqa: F401

pytestmark = pytest.mark.gpu


def unit(n, z):
    """Weights of a row of more than 16384 entries whose largest is 0, as the header has them: multiples of 2^-S of e^(1/16)."""
    s = min(51, 62 - math.ceil(math.log2(n)))
    x = math.exp(z - 0.0625) * 2.0 ** s
    assert abs(x % 1 - 0.5) > 1e-4                        # (far from where 64 bits could round it otherwise)
    return round(x)


@pytest.mark.parametrize("n,z", [(200003, -20.0), (1 << 20, -17.0), (65536, -22.0), (500000, -19.5)])
def test_many_small_weights_at_the_border_of_a_top_p(H, n, z):   # noqa: F811
    # One entry of 1 and m equal ones far below it, all of them a top-k's.  Their weights' roundings are all the same way, so that
    # the sum of the whole numbers is up to m / 2 units from what the parts of the row sum up with a unit of their own: a top-p whose border lies
    # in between has to be found by the whole numbers.
    import torch
    top, best = unit(n, 0.0), None
    for step in range(400):                               # the z near the one given whose roundings are largest, up and then down
        v = float(np.float32(z - step * 0.001))
        x = math.exp(v - 0.0625) * 2.0 ** min(51, 62 - math.ceil(math.log2(n)))
        off = round(x) - x
        if abs(off) < 0.499 and (best is None or off > best[0]):
            best = (off, v)
    off, v = best
    w = unit(n, v)
    assert off > 0.4
    found = []
    for m in range(n - 3, n - 4000, -1):
        total = top + m * w
        p = np.float32(top / (total - 0.5 * off * m))     # the border in the middle between both sums
        for q in (p, np.nextafter(p, np.float32(0)), np.nextafter(p, np.float32(2))):
            share = math.ceil(Fraction(float(q)) * total)
            if top + 0.3 * off * m < share < top + 0.9 * off * m:
                found.append((m, q, share))
        if len(found) >= 4:
            break
    assert found
    for m, q, share in found:
        row = np.full((1, n), -np.inf, dtype=np.float32)
        at = np.random.RandomState(m).permutation(n)[:m + 1]
        row[0, at] = v
        row[0, at[0]] = 0
        kept = 1 + -(-(share - top) // w)                 # entries before which less than the share lies
        t = lambda a, d: torch.tensor([a], dtype=d, device=DEV)
        _, _, got = H.sample_filtered(torch.from_numpy(row).to(DEV), t(0.5, torch.float32), top_k=t(m + 1, torch.int32), top_p=t(float(q), torch.float32))
        assert got.item() == kept, (m, q, share - top, w)
