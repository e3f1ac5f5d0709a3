"""hawk_verify_chains against the oracle's warp and draws, chain by chain: counts and tokens are equal, since both sides take
their decisions in float64 on the same fp32 logits."""
import numpy as np
import pytest

import oracle
import synth

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def H():
    import torch
    import paper_2510_25739_amd as H
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return H


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def law(row, temperature, top_k):
    """Probabilities of a row (its weights over their sum)."""
    w, z = oracle.warp(row, temperature, top_k)
    return np.asarray(w, dtype=np.float64) / float(z)


def drawn(p, u):
    c = np.cumsum(p)
    over = np.flatnonzero((c > u * p.sum()) & (p > 0))
    return int(over[0]) if len(over) else int(np.flatnonzero(p > 0)[-1])


def chain(p_rows, q_rows, draft, u_acc, u_fin, temperature, top_k):
    n = p_rows.shape[1]
    for i, d in enumerate(draft):
        p = law(p_rows[i], temperature, top_k)
        q = np.zeros(n)
        if q_rows is not None:
            q = law(q_rows[i], temperature, top_k)
        elif 0 <= d < n:
            q[d] = 1.0
        if 0 <= d < n and float(u_acc[i]) * q[d] < p[d]:
            continue
        left = np.maximum(p - q, 0.0)
        return i, list(draft[:i]) + [drawn(left if left.sum() > 0 else p, float(u_fin))]
    return len(draft), list(draft) + [drawn(law(p_rows[len(draft)], temperature, top_k), float(u_fin))]


def make(seed, n_seq, k, n, temperature, top_k, near=0.5):
    p = synth.make_logit_rows(seed, (n_seq, k + 1, n))
    q = (p[:, :k] + near * synth.make_logit_rows(seed + 1, (n_seq, k, n))).astype(np.float32)
    u_draw, u_acc, u_fin = (synth.make_uniforms(seed + i, s) for i, s in ((2, (n_seq, k)), (3, (n_seq, k)), (4, (n_seq,))))
    draft = np.zeros((n_seq, k), dtype=np.int32)
    for s in range(n_seq):
        for i in range(k):
            draft[s, i] = drawn(law(q[s, i], temperature, top_k), float(u_draw[s, i]))
    return p, q, draft, u_acc, u_fin


def compare(count, toks, want, k):
    count, toks = count.cpu().numpy(), toks.cpu().numpy()
    for s, (a, t) in enumerate(want):
        assert count[s] == a and list(toks[s]) == t + [-1] * (k + 1 - len(t)), (s, count[s], toks[s], a, t)


CHAINS = [
    # n_seq, k, n, temperature, top_k
    (3, 5, 16384, 1.0, 1000),
    (4, 3, 1008, 0.7, 1008),        # every entry kept
    (2, 63, 64, 1.0, 20),           # the longest chain
    (5, 2, 1, 1.0, 1),              # one entry
    (3, 4, 5000, 0.0, 10),          # greedy
    (2, 1, 16384, 1.0, 16384),
    (3, 2, 10000, 1.3, 4000),       # more kept than a list holds
    (2, 3, 40001, 1.0, 40001),      # slices beyond the registers, no multiple of four
    (2, 2, 65536, 0.8, 2000),
    (2, 2, 20000, 1.0, 1),
    (1, 1, 300000, 1.0, 300000),
]


@pytest.mark.parametrize("proposals", [True, False])
@pytest.mark.parametrize("n_seq,k,n,temperature,top_k", CHAINS)
def test_chains_match_the_rule(H, n_seq, k, n, temperature, top_k, proposals):
    p, q, draft, u_acc, u_fin = make(n + k, n_seq, k, n, temperature, top_k)
    if n_seq > 1:
        u_acc[0] = 0.0            # everything with target mass is accepted
    count, toks = H.verify_chains(dev(p.reshape(-1, n)), dev(q) if proposals else None, dev(draft), dev(u_acc), dev(u_fin), temperature, top_k)
    want = [chain(p[s], q[s] if proposals else None, draft[s], u_acc[s], u_fin[s], temperature, top_k) for s in range(n_seq)]
    compare(count, toks, want, k)


def test_every_length_is_accepted_somewhere(H):
    n_seq, k, n = 96, 3, 500
    p, q, draft, u_acc, u_fin = make(40, n_seq, k, n, 1.0, 300)
    want = [chain(p[s], q[s], draft[s], u_acc[s], u_fin[s], 1.0, 300) for s in range(n_seq)]
    assert {a for a, _ in want} == {0, 1, 2, 3}
    count, toks = H.verify_chains(dev(p.reshape(-1, n)), dev(q), dev(draft), dev(u_acc), dev(u_fin), 1.0, 300)
    compare(count, toks, want, k)


@pytest.mark.parametrize("n,top_k", [(2000, 100), (2000, 2000), (30000, 30000), (30000, 50)])
def test_ragged_chains_strided_rows_and_sequences_left_out(H, n, top_k):
    import torch
    n_seq, k, t = 7, 4, 1.0
    p, q, draft, u_acc, u_fin = make(5, n_seq, k, n, t, top_k)
    nd = np.array([4, 0, 2, -1, 9, 3, 1], dtype=np.int32)
    real = [min(x, k) for x in nd]
    # the sequences' rows packed one behind the other in another order, rows 24 floats longer than the slice
    order, start, at = [2, 0, 6, 4, 1, 5, 3], np.zeros(n_seq, dtype=np.int32), 0
    packed = np.zeros((64, n + 24), dtype=np.float32)
    for s in order:
        start[s] = at
        packed[at:at + max(real[s], 0) + 1, :n] = p[s, :max(real[s], 0) + 1]
        at += max(real[s], 0) + 1
    rows = dev(packed[:at])[:, :n]
    qq = torch.full((n_seq, k, n + 8), float("nan"), device=DEV)
    for s in range(n_seq):
        qq[s, :max(real[s], 0), :n] = dev(q[s, :max(real[s], 0)])
    start[5] = at - 3                # its last row would lie behind the others: left out
    draft[2, 1] = n                  # outside the slice: rejected
    draft[4, 2] = -7
    u_acc[2, 0] = u_acc[4, :2] = 0.0
    want = [(-1, []) if s in (3, 5) else chain(p[s], q[s], draft[s, :real[s]], u_acc[s], u_fin[s], t, top_k) for s in range(n_seq)]
    assert want[2][0] <= 1 and want[4][0] <= 2
    for _ in range(2):
        count, toks = H.verify_chains(rows, qq[:, :, :n], dev(draft), dev(u_acc), dev(u_fin), t, top_k, n_draft=dev(nd), p_start=dev(start))
        compare(count, toks, want, k)


@pytest.mark.parametrize("n,top_k", [(3000, 3000), (3000, 64), (40000, 40000), (40000, 64)])
def test_masked_entries_ties_and_residuals_without_mass(H, n, top_k):
    # most logits minus infinity or the type's lowest value; equal logits at the border of what is kept; the proposal equal
    # to the target, so that a rejection leaves nothing and the token comes from the target
    n_seq, k, t = 4, 2, 1.0
    p, q, draft, u_acc, u_fin = make(9, n_seq, k, n, t, top_k)
    lowest = np.finfo(np.float32).min
    p[0, :, 50:] = -np.inf
    q[0, :, 60:] = -np.inf
    p[1, :, ::2] = lowest
    p[2] = np.round(p[2] * 2) / 2
    q[2] = np.round(q[2] * 2) / 2
    q[3] = p[3, :k]
    draft[0], draft[3] = (7, 55), (draft[3, 0], n - 1)
    u_acc[0, 0] = 0.0
    p[3, 1, n - 1] = q[3, 1, n - 1] = -np.inf      # no mass: rejected, and p - q is nothing
    count, toks = H.verify_chains(dev(p.reshape(-1, n)), dev(q), dev(draft), dev(u_acc), dev(u_fin), t, top_k)
    compare(count, toks, [chain(p[s], q[s], draft[s], u_acc[s], u_fin[s], t, top_k) for s in range(n_seq)], k)


def test_no_drafts_is_a_draw(H):
    import torch
    n = 5000
    p = synth.make_logit_rows(3, (6, n))
    u = synth.make_uniforms(4, (6,))
    empty = torch.zeros((6, 0), device=DEV)
    count, toks = H.verify_chains(dev(p), None, empty.int(), empty, dev(u), 1.0, 100)
    assert count.tolist() == [0] * 6 and toks[:, 0].tolist() == H.sample_rows(dev(p), dev(u), 1.0, 100).tolist()


@pytest.mark.parametrize("n", [4096, 30000])
@pytest.mark.parametrize("temperature,top_k", [(1.0, 50), (1.0, 1 << 20), (0.0, 5)])
def test_not_a_number_ends_with_tokens_of_the_slice(H, n, temperature, top_k):
    p, q, draft, u_acc, u_fin = make(2, 3, 2, n, 1.0, 100)
    p[0] = np.nan
    q[1] = np.nan
    p[2, :, ::3] = np.nan
    count, toks = H.verify_chains(dev(p.reshape(-1, n)), dev(q), dev(draft), dev(u_acc), dev(u_fin), temperature, top_k)
    count, toks = count.cpu().numpy(), toks.cpu().numpy()
    for s in range(3):
        assert 0 <= count[s] <= 2 and (toks[s, :count[s] + 1] >= 0).all() and (toks[s, :count[s] + 1] < n).all()
