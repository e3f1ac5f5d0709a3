"""hawk_verify_chains on long slices cut by top-k, with logits at the borders of the bins that the threshold is looked for in: a scaled logit
lies at the start of a bin, and the logit's product with 1 / temperature, before it is rounded, in the one above.  Which entries are kept and what is drawn equals the
oracle's."""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
STEP = 32.0      # bins of a unit below the maximum


@pytest.fixture(scope="module")
def H():
    import torch
    import paper_2510_25739_amd as H
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return H


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def at_borders(top, temperature):
    """Logits whose rounded product with 1 / temperature lies in a bin behind the one of the product itself, and that bin."""
    inv = np.float32(1) / np.float32(temperature)
    ztop = np.float32(top) * inv
    found = []
    for m in range(20, 400):
        v = np.float32((float(ztop) - m / STEP) / float(inv))
        for _ in range(4):
            v = np.nextafter(v, np.float32(-np.inf))
        for _ in range(9):
            rounded = int((ztop - v * inv) * np.float32(STEP))
            product = int(np.float32(float(ztop) - float(v) * float(inv)) * np.float32(STEP))
            if rounded == product + 1:
                found.append((v, rounded))
            v = np.nextafter(v, np.float32(np.inf))
    return found


@pytest.mark.parametrize("n", [20000, 20003, 65536])
@pytest.mark.parametrize("threshold", ["rounded", "product"])      # the bin that the threshold lies in
@pytest.mark.parametrize("temperature", [0.7, 1.3])
def test_entries_at_a_bins_border(H, temperature, threshold, n):
    import torch
    rng = np.random.RandomState(n + int(10 * temperature))
    top = np.float32(9.3)
    inv, choices = np.float32(1) / np.float32(temperature), at_borders(top, temperature)
    v, rounded = choices[len(choices) // 2]
    bin_at = rounded if threshold == "rounded" else rounded - 1
    ztop = float(top * inv)
    logits = lambda lo, hi, size: ((ztop - rng.uniform(lo, hi, size) / STEP) / float(inv)).astype(np.float32)
    above, tied, inside = 700, 300, 260
    low = rounded - 1
    parts = [np.full(1, top), logits(0.5, low - 0.5, above), np.full(tied, v), logits(low + 0.1, low + 0.9, inside), logits(low + 1.1, low + 1.9, inside)]
    rest = n - sum(map(len, parts))
    row = np.concatenate(parts + [logits(low + 3, low + 40, rest)]).astype(np.float32)
    rng.shuffle(row)
    z = row * inv
    bins = (np.float32(z.max()) - z) * np.float32(STEP)
    top_k = int((bins.astype(int) < bin_at).sum()) + (inside if bin_at == low else inside + tied) // 2
    w, total = oracle.warp(row, temperature, top_k)
    w = np.asarray(w, dtype=np.float64)
    assert int((w > 0).sum()) == top_k
    # one draft a sequence, a certain one with u = 0: accepted if it is kept; and a draw of the row for each
    near = np.flatnonzero((row == v) | (np.abs(bins - low - 1) < 1))
    draft = np.concatenate([near, rng.choice(n, 64, replace=False)]).astype(np.int32)[:, None]
    n_seq = len(draft)
    u = ((np.arange(n_seq) + 0.5) / n_seq).astype(np.float32)
    drawn = lambda weights: np.searchsorted(np.cumsum(weights), u.astype(np.float64) * weights.sum(), side="right")
    plain = drawn(w)
    rows = dev(np.stack([row, row]))
    count, toks = H.verify_chains(rows, None, dev(draft), torch.zeros((n_seq, 1), device=DEV), dev(u), temperature, top_k,
                                  p_start=torch.zeros(n_seq, dtype=torch.int32, device=DEV))
    count, toks = count.cpu().numpy(), toks.cpu().numpy()
    kept = w[draft[:, 0]] > 0
    print(f"bin {bin_at}, top_k {top_k}: {int((count != kept).sum())} of {n_seq} drafts judged otherwise, "
          f"{int((toks[np.arange(n_seq), count] != plain).sum())} other tokens")
    assert np.array_equal(count == 1, kept)
    # an accepted draft's next token and a rejected one's replacement (nothing to take from the row) are draws of the same row
    assert np.array_equal(toks[np.arange(n_seq), count], plain) and np.array_equal(toks[kept, 0], draft[kept, 0])
