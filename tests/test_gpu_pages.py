"""Taking, sharing, giving back, moving and copying pages of a cache against a plain simulation on the host: tables, counts and every value
of the pools are equal."""
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


def i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


class Pool:
    """A cache and its mirror on the host."""

    def __init__(self, H, seed, n_seq, max_pages, n_pages, page=4, layers=2, heads=2, hd=8, dtype="float16", order="heads"):
        import torch
        self.g = torch.Generator().manual_seed(seed)
        self.page, self.n_pages, self.max_pages, self.n_seq = page, n_pages, max_pages, n_seq
        shape = {"heads": (layers, n_pages, heads, page, hd), "entries": (layers, n_pages, page, heads, hd), "pages": (n_pages, layers, heads, page, hd),
                 "pair": (layers, n_pages, 2, heads, page, hd)}[order]
        back = {"heads": lambda t: t, "entries": lambda t: t.permute(0, 1, 3, 2, 4), "pages": lambda t: t.transpose(0, 1)}.get(order)
        if order == "pair":                              # keys and values of a page side by side
            both = torch.randn(*shape, generator=self.g).to(getattr(torch, dtype)).to(DEV)
            self.k, self.v = both[:, :, 0], both[:, :, 1]
        else:
            self.k, self.v = (back(torch.randn(*shape, generator=self.g).to(getattr(torch, dtype)).to(DEV)) for _ in range(2))
        self.table = torch.full((n_seq, max_pages), -1, dtype=torch.int32, device=DEV)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        self.n_past = torch.zeros(n_seq, dtype=torch.int32, device=DEV)
        self.cache = H.PagedCache(self.k, self.v, self.table)
        self.t = [[-1] * max_pages for _ in range(n_seq)]
        self.r = [0] * n_pages
        self.past = [0] * n_seq
        self.hk, self.hv = self.k.cpu().clone(), self.v.cpu().clone()

    def check(self):
        import torch
        torch.cuda.synchronize()
        assert self.table.cpu().tolist() == self.t
        assert self.refs.cpu().tolist() == self.r
        assert self.n_past.cpu().tolist() == self.past
        assert torch.equal(self.k.cpu(), self.hk) and torch.equal(self.v.cpu(), self.hv)

    def counted(self):
        n = [0] * self.n_pages
        for row in self.t:
            for p in row:
                if 0 <= p < self.n_pages:
                    n[p] += 1
        return n

    def real(self, p):
        return 0 <= p < self.n_pages

    def places(self, entries):
        return min(-(-max(entries, 0) // self.page), self.max_pages)

    def fork(self, src, dst):
        self.cache.fork(self.refs, self.n_past, i32(src), i32(dst))
        ok = [0 <= a < self.n_seq and 0 <= b < self.n_seq and a != b for a, b in zip(src, dst)]
        use = [ok[i] and not any(ok[j] and dst[j] == dst[i] for j in range(i)) and not any(ok[j] and dst[j] == src[i] for j in range(len(src)))
               for i in range(len(src))]
        for a, b, yes in zip(src, dst, use):
            if not yes:
                continue
            for p in self.t[b]:
                if self.real(p):
                    self.r[p] -= 1
            self.t[b] = [p if i < self.places(self.past[a]) else -1 for i, p in enumerate(self.t[a])]
            for p in self.t[b]:
                if self.real(p):
                    self.r[p] += 1
            self.past[b] = self.past[a]

    def take(self, new):
        short = self.cache.take(self.refs, self.n_past, i32(new))
        before, free, asked, out = list(self.r), [p for p, n in enumerate(self.r) if n == 0], 0, []
        room = len(free)
        for s in range(self.n_seq):
            lack = []
            if new[s] > 0 and 0 <= self.past[s] < self.max_pages * self.page:
                for i in range(self.past[s] // self.page, self.places(self.past[s] + new[s])):
                    if not self.real(self.t[s][i]) or before[self.t[s][i]] > 1:
                        lack.append(i)
            asked += len(lack)
            out.append(len(lack) if asked > room else 0)
            if asked > room:
                continue
            for i in lack:
                old, p = self.t[s][i], free.pop(0)
                if self.real(old):
                    self.r[old] -= 1
                    n = self.past[s] - i * self.page
                    if n > 0:
                        for h in (self.hk, self.hv):
                            h[:, p, :, :n] = h[:, old, :, :n]
                self.r[p] = 1
                self.t[s][i] = p
        assert short.cpu().tolist() == out
        return out

    def trim(self, past):
        self.n_past.copy_(i32(past))
        self.past = list(past)
        self.cache.trim(self.refs, self.n_past)
        for s, n in enumerate(past):
            if n < 0:
                continue
            for i in range(self.places(n), self.max_pages):
                if self.real(self.t[s][i]):
                    self.r[self.t[s][i]] -= 1
                self.t[s][i] = -1

    def compact(self, in_place=False):
        old = (self.table.clone(), self.refs.clone())
        table, refs, used = self.cache.compact(self.refs, table=self.table, refs_out=self.refs) if in_place else self.cache.compact(self.refs)
        n = sum(1 for x in self.r if x > 0)
        holes, to = [p for p in range(n) if self.r[p] <= 0], {}
        for p in range(n, self.n_pages):
            if self.r[p] > 0:
                to[p] = holes.pop(0)
                for h in (self.hk, self.hv):
                    h[:, to[p]] = h[:, p]
        there = [x > 0 for x in self.r]
        self.t = [[to.get(p, p) if self.real(p) and there[p] else -1 for p in row] for row in self.t]
        for a, b in to.items():
            self.r[b], self.r[a] = self.r[a], 0
        assert used.item() == n
        if not in_place:
            import torch
            assert torch.equal(self.table, old[0]) and torch.equal(self.refs, old[1])
            self.table, self.refs = table, refs
            self.cache.table = table
        return len(to)

    def write(self, new):
        """What a step does with the pages it took: its entries, by their places."""
        import torch
        for s, n in enumerate(new):
            for e in range(self.past[s], self.past[s] + max(n, 0)):
                p = self.t[s][e // self.page]
                assert self.real(p) and self.r[p] == 1
                x = torch.randn(2, self.hk.shape[0], self.hk.shape[2], self.hk.shape[4], generator=self.g).to(self.hk.dtype)
                for pool, h, y in ((self.k, self.hk, x[0]), (self.v, self.hv, x[1])):
                    h[:, p, :, e % self.page] = y
                    pool[:, p, :, e % self.page] = y.to(DEV)
            if n > 0:
                self.past[s] += n
        self.n_past.copy_(i32(self.past))


SHAPES = [dict(), dict(order="entries", hd=24), dict(order="pages", dtype="bfloat16", hd=64), dict(order="pair", hd=16), dict(page=1), dict(page=3, dtype="float32"),
          dict(page=16, heads=1, hd=256), dict(layers=1, heads=5, hd=80, page=7), dict(layers=3, heads=3, hd=96, page=33, dtype="float32")]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_a_life_of_a_pool(H, shape):
    page = shape.get("page", 4)
    p = Pool(H, 1, 6, 8, 40, **shape)
    new = [3 * page, 2 * page + page // 2, 1, 0, -1, 0]
    assert p.take(new) == [0] * 6
    p.check()
    p.write(new)
    p.fork([0, 1, 1], [3, 4, 5])                         # two images of the second prompt, one of the first
    p.check()
    assert p.counted() == p.r
    new = [0, 2, 0, 1, page + 1, 1]                      # the second prompt's three holders go on inside a page, or at its end
    assert p.take(new) == [0] * 6
    p.check()
    p.write(new)
    p.check()
    past = list(p.past)
    past[0], past[3] = 0, past[3] - page                 # one ends, one goes back a page
    p.trim(past)
    p.check()
    p.compact()
    p.check()
    assert p.counted() == p.r and all((n > 0) == (i < sum(x > 0 for x in p.r)) for i, n in enumerate(p.r))
    p.fork([4], [0])
    p.take([page, 0, 0, 0, 1, 0])
    p.check()


@pytest.mark.parametrize("seed", range(6))
def test_random_lives(H, seed):
    r = np.random.RandomState(seed)
    n_seq, page = int(r.choice([1, 2, 5, 17, 40])), int(r.choice([1, 2, 5, 16]))
    p = Pool(H, seed, n_seq, 6, int(r.choice([8, 30, 4 * n_seq + 3])), page=page, layers=int(r.randint(1, 4)), hd=int(r.choice([8, 40])), order=str(r.choice(["heads", "entries", "pages"])))
    for _ in range(25):
        what = r.choice(["take", "take", "fork", "trim", "compact"])
        if what == "take":
            new = [int(x) for x in r.randint(-1, 2 * page + 2, n_seq)]
            new = [min(n, 6 * page - q) for n, q in zip(new, p.past)]
            short = p.take(new)
            p.check()
            p.write([0 if s else n for n, s in zip(new, short)])
        elif what == "fork":
            n = int(r.randint(1, n_seq + 1))
            p.fork([int(x) for x in r.randint(-1, n_seq + 1, n)], [int(x) for x in r.randint(-1, n_seq + 1, n)])
        elif what == "trim":
            p.trim([int(r.choice([0, q // 2, q, q])) for q in p.past])
        else:
            p.compact(in_place=bool(r.randint(2)))
        p.check()
        assert p.counted() == p.r


def test_too_few_pages(H):
    p = Pool(H, 3, 4, 4, 5)
    assert p.take([8, 9, 4, 0]) == [0, 0, 1, 0]          # 2 and 3 pages; the third finds none, the fourth needs none
    p.check()
    assert p.take([0, 0, 16, 1]) == [0, 0, 4, 1]
    p.check()
    p.write([8, 9, 0, 0])
    p.trim([0, 9, 0, 0])
    assert p.take([0, 0, 9, 4]) == [0, 0, 3, 1]          # two free ones: the third needs three, and the fourth stands behind it
    assert p.take([0, 0, 8, 0]) == [0] * 4
    p.check()


def test_entries_behind_the_table(H):
    p = Pool(H, 4, 3, 2, 9)
    p.past = [7, 8, 2 ** 31 - 1]
    p.n_past.copy_(i32(p.past))
    assert p.take([2 ** 31 - 1, 5, 2 ** 31 - 1]) == [0, 0, 0]      # a table of two pages: the first gets its second place, the others are at the end
    assert [x >= 0 for x in p.t[0]] == [False, True]
    p.check()


def test_numbers_that_are_none(H):
    p = Pool(H, 5, 4, 3, 6)
    assert p.take([5, 3, 1, 0]) == [0] * 4
    p.write([5, 3, 1, 0])
    p.fork([0, 0, 7, -1, 2][:4], [1, 1, 0, 2][:4])       # twice the same; no such sequences
    p.check()
    p.fork([0, 1], [1, 3])                               # the second's source changes
    p.check()
    # tables and counts that hold anything: pages outside the pool are none
    p.t[3] = [6, -2 ** 31, 2 ** 31 - 1]
    p.table.copy_(i32(p.t))
    p.past[3] = 12
    p.n_past.copy_(i32(p.past))
    p.fork([3], [2])
    p.check()
    p.compact()
    p.check()
    p.trim([0, -1, 0, 0])
    p.check()


@pytest.mark.parametrize("n_seq,n_pages", [(1500, 5000), (3, 40000), (1100, 1200)])
def test_many_sequences_and_pages(H, n_seq, n_pages):
    r = np.random.RandomState(n_seq)
    p = Pool(H, 6, n_seq, 4, n_pages, page=2, layers=1, heads=1)
    new = [int(x) for x in r.randint(0, 9, n_seq)]
    short = p.take(new)
    p.check()
    assert (max(short) > 0) == (n_pages == 1200)
    p.past = [0 if s else n for n, s in zip(new, short)]
    p.n_past.copy_(i32(p.past))
    half = n_seq // 2
    p.fork(list(range(half)), list(range(n_seq - half, n_seq)))
    p.check()
    p.take([1 if i % 3 == 0 and q < 8 else 0 for i, q in enumerate(p.past)])
    p.check()
    p.trim([q if i % 2 else 0 for i, q in enumerate(p.past)])
    assert p.compact() > 0 or n_seq == 3
    p.check()


def test_a_pool_in_use_far_behind(H):
    import torch
    p = Pool(H, 7, 2, 600, 50000, page=1, layers=1, heads=1)
    for s, first in ((0, 49000), (1, 20000)):
        p.t[s] = [first + i for i in range(600)]
        for x in p.t[s]:
            p.r[x] += 1
    p.table.copy_(i32(p.t))
    p.refs.copy_(i32(p.r))
    p.past = [600, 600]
    p.n_past.copy_(i32(p.past))
    assert p.compact() == 1200
    p.check()
    assert torch.equal(p.table.cpu(), torch.arange(1200, dtype=torch.int32).view(2, 600).flip(0))


def test_pages_to_another_pool(H):
    import torch
    a = Pool(H, 8, 1, 2, 12, page=6, hd=24, layers=3)
    b = Pool(H, 9, 2, 3, 5, page=6, hd=24, layers=3, order="entries")
    src, dst = [11, 0, 5, 12, -1, 3], [4, 0, 2, 1, 3, 5]
    a.cache.copy_pages(i32(src), i32(dst), to=b.cache)
    for s, d in zip(src[:3], dst[:3]):
        b.hk[:, d], b.hv[:, d] = a.hk[:, s], a.hv[:, s]
    a.check()
    b.check()
    a.cache.copy_pages(i32([1, 2]), i32([7, 8]))
    a.hk[:, 7:9], a.hv[:, 7:9] = a.hk[:, 1:3].clone(), a.hv[:, 1:3].clone()
    a.check()
    a.cache.copy_pages(i32([]), i32([]))
    other = Pool(H, 9, 1, 1, 3, page=5, hd=24, layers=3)
    for kw in (dict(to=other.cache), dict(src=i32([1, 2, 3])), dict(dst=i32([1, 2]).long())):
        with pytest.raises(H.HawkError):
            a.cache.copy_pages(**{**dict(src=i32([1, 2]), dst=i32([3, 4])), **kw})


def test_refusals_of_the_binding(H):
    p = Pool(H, 10, 3, 2, 6)
    c, refs, past = p.cache, p.refs, p.n_past
    for f in (lambda: c.take(refs[:5], past, past), lambda: c.take(refs, past[:2], past), lambda: c.take(refs, past, past.long()), lambda: c.trim(refs.long(), past),
              lambda: c.take(refs, past, past, short_by=refs), lambda: c.trim(refs, past.cpu()), lambda: c.fork(refs, past, i32([0]), i32([1, 2])),
              lambda: c.fork(refs, past, i32([0, 1, 2, 0]), i32([1, 2, 0, 1])), lambda: c.compact(refs.cpu()), lambda: c.compact(refs, table=p.table[:2]),
              lambda: c.compact(refs, refs_out=refs[:3]), lambda: c.compact(refs, n_used=past)):
        with pytest.raises(H.HawkError):
            f()
    p.check()


def test_a_captured_step_is_replayed(H):
    import torch
    p = Pool(H, 11, 4, 6, 30)
    new = i32([0] * 4)
    src, dst = i32([0, 0]), i32([2, 3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.cache.take(p.refs, p.n_past, new)
        torch.cuda.current_stream().synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            p.cache.fork(p.refs, p.n_past, src, dst)
            short = p.cache.take(p.refs, p.n_past, new)
    p.take([5, 3, 0, 0])
    p.write([5, 3, 0, 0])
    for step in range(3):
        mirror = Pool.__new__(Pool)
        mirror.__dict__.update({k: (v.clone() if torch.is_tensor(v) else v) for k, v in p.__dict__.items()})
        mirror.t, mirror.r, mirror.past = [list(x) for x in p.t], list(p.r), list(p.past)
        mirror.table, mirror.refs, mirror.n_past = p.table.clone(), p.refs.clone(), p.n_past.clone()
        mirror.cache = H.PagedCache(mirror.k, mirror.v, mirror.table)
        want = [1 + step, 0, 2, 7]
        mirror.fork([0, 0], [2, 3])
        out = mirror.take(want)
        new.copy_(i32(want))
        g.replay()
        torch.cuda.synchronize()
        assert short.cpu().tolist() == out
        p.t, p.r, p.past, p.hk, p.hv = mirror.t, mirror.r, mirror.past, mirror.hk, mirror.hv
        p.check()
        p.write([1, 0, 0, 0])
