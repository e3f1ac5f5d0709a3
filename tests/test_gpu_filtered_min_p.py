"""Entries that min-p keeps where the least weight is small, far below the weights' own unit or next to one: by 64 bits."""
import math

import numpy as np
import pytest

from test_gpu_filtered import DEV, H, check, draw   # noqa: F401

pytestmark = pytest.mark.gpu


def check_beside_top_p(H, z, m, k, p):   # noqa: F811
    """Like check, where a top-p's border may be another one.  It is found with weights that are held as multiples of 2^-S of a number up to e^(1/16)
    times the largest, S = min(51, 62 - log2 n rounded up): each is off by half of that, the sum before an entry and p times the whole by n / 2 of it
    at most, so that entries before which the mass is within n 2^-S e^(1/16) of p times the whole may be on either side.  In rows of 2^20 entries that
    is 2.5e-7, and near the border of a top-p of 1 - 10^-7 are entries of a weight of 1.2e-7 each."""
    import torch
    rows, n = z.shape
    u = (np.random.RandomState(rows + n).randint(0, 1 << 24, rows) / float(1 << 24)).astype(np.float32)
    t = lambda a: torch.from_numpy(a).to(DEV)
    tok, prob, kept = (x.cpu().numpy() for x in H.sample_filtered(t(z), t(u), top_k=t(k), top_p=t(p), min_p=t(m)))
    off = n * 2.0 ** -min(51, 62 - math.ceil(math.log2(n))) * math.exp(1 / 16)
    for i in range(rows):
        token, share, count = draw(z[i], u[i], 1.0, k[i], p[i], m[i])
        assert tok[i] == token and abs(prob[i] - share) <= share * (2.0 ** -24 + 2.0 ** -30), (i, tok[i], prob[i], token, share)
        least = most = count
        if p[i] < 1:
            w = np.sort(np.exp(z[i].astype(np.float64) - z[i].max()))[::-1][:k[i] if 1 <= k[i] < n else n]
            before, cut, small = np.cumsum(w) - w, float(p[i]) * w.sum(), int((w >= float(m[i])).sum())
            least, most = min(small, int((before < cut - off).sum())), min(small, int((before < cut + off).sum()))
            assert least <= count <= most <= least + 8
        assert least <= kept[i] <= most, (i, kept[i], least, most)


@pytest.mark.parametrize("n", [300, 4097, 16384, 20000, 100000, 200003, 1 << 20])
def test_small_min_p(H, n):   # noqa: F811
    # entries of weights from one down to 2^-149 and below, hundreds of them between half and twice the least; the shares that an
    # fp32 number holds, the smallest of them among these
    m = np.array([1e-6, 1e-9, 1e-11, 1e-13, 3e-15, 1e-16, 1e-20, 1e-30, 1.2e-38, 2.0 ** -149], dtype=np.float32)
    z = -np.random.RandomState(n).uniform(0, 110, (m.size, n)).astype(np.float32)
    check(H, z, m=m)
    check_beside_top_p(H, z + np.float32(37.25), m, np.array([0, n // 3] * 5, dtype=np.int32), np.array([1, 1, 1, 0.9999999, 1] * 2, dtype=np.float32))
    check(H, z * 2, T=[1.0, 0.5, 3.0, 2.0, 0.7] * 2, m=m)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("n", [16384, 70000])
def test_min_p_at_a_logit_of_16_bits(H, n, dtype):   # noqa: F811
    # many equal logits, and a least weight that is one's own but for the rounding of min-p to 24 bits
    import torch
    z = torch.from_numpy(-np.random.RandomState(n).uniform(0, 40, (12, n)).astype(np.float32)).to(getattr(torch, dtype)).float().numpy()
    z[:, 7] = 0
    at = np.array([z[i, 100 + i] for i in range(12)], dtype=np.float64)
    m = np.exp(at).astype(np.float32)
    assert (np.abs(m - np.exp(at)) > 1e-12 * m).all()     # (no border that 64 bits could see otherwise)
    check(H, z, m=m, dtype=dtype)


def test_min_p_beside_extreme_maxima(H):   # noqa: F811
    # where z has few bits left behind the maximum, and where it has all of them next to zero
    r = np.random.RandomState(5)
    for n in (5000, 40000):
        z = -r.uniform(0, 30, (6, n)).astype(np.float32)
        z += np.array([2.0 ** 20, -2.0 ** 18, 1e5, math.log(20), 5.5, -1e-3], dtype=np.float32)[:, None]
        check(H, z, m=[0.05, 1e-4, 0.3, 0.05, 0.004, 1 - 2.0 ** -24])
