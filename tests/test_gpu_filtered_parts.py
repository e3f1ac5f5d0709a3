"""Long rows of filtered draws on every way they can take: parts of 8, 16 and 32 entries a thread, more rows than go at a time, and logits that
are beyond the parts' grid."""
import numpy as np
import pytest

from test_gpu_filtered import DEV, H, check, logits   # noqa: F401

pytestmark = pytest.mark.gpu


def entries_a_thread(rows, n):
    """The rule of filtered.hip: parts as small as leave 256 of them, and no more than 32 a row."""
    e = 8
    while e < 32 and (-(-n // (e * 1024)) > 32 or rows * -(-n // (e * 1024)) > 256):
        e *= 2
    return e


def mixed(seed, rows, n):
    r = np.random.RandomState(seed)
    z = logits(seed, rows, n)
    for i in range(0, rows, 5):                          # few values; as near as lists do not hold; all alike but for a few
        z[i] = np.round(z[i] * 2) / 2
    for i in range(1, rows, 5):
        z[i] *= r.choice([0.02, 0.1])
    for i in range(2, rows, 5):
        z[i, r.permutation(n)[n // 50:]] = -3.0
    return z, dict(k=np.where(r.rand(rows) < 0.5, 0, r.randint(1, n, rows)), p=np.where(r.rand(rows) < 0.3, 1.0, r.uniform(0.2, 0.999, rows)),
                   m=np.where(r.rand(rows) < 0.6, 0.0, r.uniform(0.001, 0.4, rows)), T=np.where(r.rand(rows) < 0.1, 0.0, r.uniform(0.5, 1.5, rows)))


@pytest.mark.parametrize("rows,n,e,dtype", [(10, 65536, 8, "float32"), (48, 65536, 16, "float32"), (48, 65536, 16, "bfloat16"), (3, 393216, 16, "float32"), (19, 200003, 16, "float16"),
                                            (60, 70001, 32, "float32"), (100, 40000, 32, "bfloat16"), (2, 1 << 20, 32, "float16")])
def test_parts_of_every_size(H, rows, n, e, dtype):   # noqa: F811
    assert entries_a_thread(rows, n) == e
    z, par = mixed(rows + n, rows, n)
    check(H, z, dtype=dtype, **par)


@pytest.mark.parametrize("rows,n,at_once", [(2051, 16385, 2048), (700, 98305, 512)])
def test_more_rows_than_go_at_a_time(H, rows, n, at_once):   # noqa: F811
    # 2048 parts at a time share the workspace; rows on both sides of the border, and the last ones, are compared
    import torch
    assert entries_a_thread(rows, n) == 32 and 2048 // -(-n // 32768) == at_once
    live = [0, 3, at_once - 2, at_once - 1, at_once, at_once + 1, rows - 1]
    assert len(set(live)) == len(live)
    z, par = mixed(n, len(live), n)
    r = np.random.RandomState(1)
    x = torch.full((rows, n), float("nan"), device=DEV)
    x[live] = torch.from_numpy(z).to(DEV)
    skip = np.full(rows, -1, dtype=np.int32)
    skip[live] = 0
    u = (r.randint(0, 1 << 24, rows) / float(1 << 24)).astype(np.float32)
    spread = {"T": ("temperature", np.float32, 1.0), "k": ("top_k", np.int32, 0), "p": ("top_p", np.float32, 1.0), "m": ("min_p", np.float32, 0.0)}
    kw = {}
    for name, (arg, dt, fill) in spread.items():
        v = np.full(rows, fill, dtype=dt)
        v[live] = par[name]
        kw[arg] = torch.from_numpy(v).to(DEV)
    t = lambda a: torch.from_numpy(a).to(DEV)
    tok, prob, kept = (a.cpu().numpy() for a in H.sample_filtered(x, t(u), skip=t(skip), **kw))
    alone = check(H, z, u=u[live], **par)
    for got, want in zip((tok, prob, kept), alone):
        assert np.array_equal(got[live], want)
    rest = np.setdiff1d(np.arange(rows), live)
    assert (tok[rest] == -1).all() and (kept[rest] == 0).all() and (prob[rest] == 0).all()


@pytest.mark.parametrize("n", [16385, 70000, 300000])
def test_logits_beyond_the_grid(H, n):   # noqa: F811
    # 2^25 and more: distinct, finite, and with temperatures that bring them there; neighbours of 24 bits are two and more apart there
    r = np.random.RandomState(n)
    z = logits(n, 9, n)
    z[0] = 2.0 ** 25 + 8 * r.randint(0, 12, n)
    z[1] = -2.0 ** 26 - 8 * r.randint(0, 5, n)
    z[2] = r.choice(np.float32([3e38, 2.9e38, -3e38, 1.0]), n)
    z[3, ::2] = 2.0 ** 30                                # alike, among ordinary ones
    z[4, n // 2] = 2.0 ** 27                             # one alone
    z[5, : n - 100] = -2.0 ** 28                         # parts that are far below, the maximum an ordinary one
    z[6] = 2.0 ** 24 + 2 * r.randint(0, 20, n)
    z[7] = 1e-3 * z[7]
    T = [1, 1, 1, 1, 1, 1, 0.25, 1e-11, 1e-9]
    check(H, z, T=T, k=[0, n // 7, 3 * n // 8, 0, 5, 0, n // 2, 40, 0], p=[0.9, 0.5, 1.0, 0.3, 0.9, 0.99, 0.7, 1.0, 0.9], m=[0, 0, 0, 0, 0.1, 0.01, 0, 0, 0])
    check(H, z, T=T, k=[7, 0, 0, n // 2 - 1, 0, 99, 0, 0, 3], p=[1.0, 1.0, 0.4, 1.0, 1.0, 1.0, 0.05, 0.9, 1.0], m=[0, 0.5, 1.0, 0, 0, 0, 0.3, 0, 0])
    check(H, z, T=0.0)
