"""The calls over a paged cache and the verification of chains without a GPU: where an entry lies, what is refused before any
launch, and what needs no buffers."""
import ctypes as C

import numpy as np
import pytest

from paper_2510_25739_amd import hawk

ONE = 4096      # an address: every call below fails, or has nothing to do, before anything is read through it


@pytest.fixture(scope="module")
def H():
    import os
    import paper_2510_25739_amd as H
    if not os.path.exists(H.lib_path()):
        from paper_2510_25739_amd import build
        build.build()
    return H


def cache(**kw):
    f = dict(k=ONE, v=ONE, layer_stride=1 << 20, page_stride=16 * 2 * 64, head_stride=16 * 64, entry_stride=64, table=ONE, table_stride=8,
             dtype=hawk.HAWK_FP16, n_layers=2, n_pages=10, page_size=16, n_heads=2, head_dim=64, n_seq=3, max_pages=8)
    f.update(kw)
    return hawk.HawkPagedCache(**f)


def rows(n=5, **kw):
    return hawk.HawkPagedRows(**{**dict(row_start=ONE, n_past=ONE, rows=n), **kw})


def heads(n, dtype=hawk.HAWK_FP16, **kw):
    return hawk.HawkHeads(**{**dict(data=ONE, row_stride=n * 64, head_stride=64, n_heads=n, dtype=dtype), **kw})


@pytest.mark.parametrize("page", [1, 2, 3, 5, 7, 16, 24, 100, 4096, 99991, 1 << 20])
def test_places_of_entries(H, page):
    # page and place by division for small and far entries, on either side of page borders
    L = H.load_library()
    max_pages = min(4000, (1 << 30) // page)
    c = cache(page_size=page, n_pages=max_pages, max_pages=max_pages, table_stride=max_pages, page_stride=1 << 40, entry_stride=72)
    table = np.random.RandomState(page).permutation(max_pages).astype(np.int32)
    p = table.ctypes.data_as(C.c_void_p)
    borders = [x * page + d for x in (0, 1, 2, max_pages // 2, max_pages - 1, max_pages) for d in (-2, -1, 0, 1, page // 2)]
    for e in borders + [2 ** 30, 2 ** 31 - 1, 2 ** 31, 2 ** 40, -2 ** 40]:
        want = (1 << 20) + int(table[e // page]) * (1 << 40) + e % page * 72 if 0 <= e < page * max_pages else -1
        assert L.hawk_paged_entry(C.byref(c), p, 1, e) == want, e


def test_entries_whose_page_is_outside_the_pool_do_not_exist(H):
    L = H.load_library()
    table = np.array([0, -1, 9, 10, 2 ** 31 - 1, -2 ** 31, 3, 3], dtype=np.int32)
    p = table.ctypes.data_as(C.c_void_p)
    c = cache()
    got = [L.hawk_paged_entry(C.byref(c), p, 0, 16 * i + 5) for i in range(9)]
    at = lambda page: page * 2048 + 5 * 64
    assert got == [at(0), -1, at(9), -1, -1, -1, at(3), at(3), -1]
    assert L.hawk_paged_entry(C.byref(c), p, 2, 0) == -1 and L.hawk_paged_entry(C.byref(c), None, 0, 0) == -1


BAD_CACHE = [dict(k=None), dict(v=None), dict(k=ONE + 8), dict(v=ONE + 2), dict(table=None), dict(dtype=3), dict(dtype=-1), dict(head_dim=0),
             dict(head_dim=60), dict(head_dim=264), dict(n_heads=0), dict(n_pages=0), dict(page_size=0), dict(n_seq=-1), dict(max_pages=0),
             dict(table_stride=7), dict(max_pages=1 << 27, table_stride=1 << 27), dict(page_stride=2044), dict(head_stride=1028),
             dict(entry_stride=68), dict(entry_stride=56), dict(head_stride=0), dict(page_stride=-2048), dict(layer_stride=-8), dict(layer_stride=4)]


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_bad_caches_are_refused(H, bad):
    L = H.load_library()
    c, r, q, k = cache(**bad), rows(), heads(4), heads(2)
    assert L.hawk_paged_append(C.byref(c), 0, C.byref(r), None, C.byref(k), C.byref(k), None, None, 0.0, None, 0, 0, 0, None, None, None) == -1
    assert L.hawk_paged_attention(C.byref(c), 0, C.byref(r), C.byref(q), None, 0.1, 0, C.byref(q), ONE, 1 << 40, None) == -1
    assert L.hawk_paged_attention_workspace_bytes(C.byref(c), 5, 4, 0) == 0
    assert L.hawk_paged_keep(C.byref(c), ONE, ONE, ONE, 2, None) == -1


def test_bad_appends_are_refused(H):
    L = H.load_library()

    def call(c=None, layer=0, r=None, q=None, k=None, v=None, qg=None, kg=None, eps=1e-5, rot=None, n_pos=0, rd=0, pairs=0, pos=None, qo=None):
        ref = lambda x: None if x is None else C.byref(x)
        return L.hawk_paged_append(ref(c or cache()), layer, ref(r or rows()), ref(q), ref(k or heads(2)), ref(v or heads(2)), qg, kg, eps, rot, n_pos,
                                   rd, pairs, pos, ref(qo), None)

    h4 = heads(4)
    bad = [dict(layer=2), dict(layer=-1), dict(r=rows(row_start=None)), dict(r=rows(n_past=None)), dict(r=rows(-1)), dict(k=heads(3)), dict(v=heads(1)),
           dict(k=heads(2, dtype=hawk.HAWK_BF16)), dict(k=heads(2, data=None)), dict(k=heads(2, data=ONE + 4)), dict(k=heads(2, row_stride=132)),
           dict(v=heads(2, head_stride=-64)), dict(q=h4), dict(qo=h4), dict(q=h4, qo=heads(3)), dict(q=h4, qo=heads(4, dtype=hawk.HAWK_BF16)),
           dict(q=heads(4, dtype=hawk.HAWK_BF16), qo=h4), dict(q=h4, qo=heads(4, row_stride=512)), dict(q=heads(4, data=1 << 20), qo=heads(4, row_stride=0)),
           dict(q=heads(4, data=1 << 20), qo=heads(4, head_stride=8)), dict(qg=ONE), dict(kg=ONE + 4), dict(kg=ONE, eps=float("nan")),
           dict(kg=ONE, eps=-1.0), dict(rot=ONE, n_pos=0, rd=64), dict(rot=ONE, n_pos=9, rd=0), dict(rot=ONE, n_pos=9, rd=60),
           dict(rot=ONE, n_pos=9, rd=72), dict(rot=ONE, n_pos=9, rd=64, pairs=2), dict(rot=ONE + 8, n_pos=9, rd=64), dict(pos=ONE), dict(r=rows(1 << 24))]
    for kw in bad:
        assert call(**kw) == -1, kw
    empty = hawk.HawkPagedRows(None, None, 0)
    none = heads(2, data=None)
    assert call(r=empty, k=none, v=none) == 0 and call(c=cache(n_seq=0, table=None)) == 0


def test_bad_attention_is_refused(H):
    L = H.load_library()

    def call(c=None, layer=0, r=None, q=None, tree=None, scale=0.125, max_len=0, out=None, ws=ONE, nws=1 << 40):
        return L.hawk_paged_attention(C.byref(c or cache()), layer, C.byref(r or rows()), C.byref(q or heads(4)), tree, scale, max_len,
                                      C.byref(out or heads(4, data=1 << 20)), ws, nws, None)

    for kw in (dict(layer=2), dict(r=rows(n_past=None)), dict(q=heads(3)), dict(q=heads(4, dtype=hawk.HAWK_FP32)), dict(out=heads(2)), dict(q=heads(4, data=None)),
               dict(out=heads(4, data=ONE + 8)), dict(out=heads(4, dtype=7)), dict(out=heads(4, row_stride=0)), dict(out=heads(4, head_stride=0)),
               dict(tree=ONE + 4), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(r=rows(1 << 28))):
        assert call(**kw) == -1, kw
    assert call(r=rows(0)) == 0 and call(c=cache(n_seq=0, table=None)) == 0
    # a long axis of few rows needs room for its parts
    long = cache(page_size=4096, page_stride=4096 * 2 * 64, head_stride=4096 * 64)
    need = L.hawk_paged_attention_workspace_bytes(C.byref(long), 5, 4, 0)
    assert need > 0 and call(c=long, nws=need - 1) == -3 and call(c=long, ws=None) == -1 and call(c=long, ws=ONE + 4) == -1
    assert L.hawk_paged_attention_workspace_bytes(C.byref(cache()), 5, 4, 0) == 0        # 128 entries at most
    assert L.hawk_paged_attention_workspace_bytes(C.byref(long), 5, 3, 0) == 0 and L.hawk_paged_attention_workspace_bytes(C.byref(long), -1, 4, 0) == 0


def test_bad_keeps_are_refused(H):
    L = H.load_library()
    for kw in (dict(n_past=None), dict(path=None), dict(n_keep=None), dict(depth=0), dict(depth=65)):
        a = {**dict(n_past=ONE, path=ONE, n_keep=ONE, depth=3), **kw}
        assert L.hawk_paged_keep(C.byref(cache()), a["n_past"], a["path"], a["n_keep"], a["depth"], None) == -1, kw
    assert L.hawk_paged_keep(C.byref(cache(n_seq=0)), ONE, ONE, ONE, 3, None) == 0
    assert L.hawk_rotary_table(None, 4, 8, 1e4, None) == -1 and L.hawk_rotary_table(ONE, 4, 7, 1e4, None) == -1
    assert L.hawk_rotary_table(ONE, 4, 8, 0.0, None) == -1 and L.hawk_rotary_table(ONE, -1, 8, 1e4, None) == -1
    assert L.hawk_rotary_table(ONE, 0, 8, 1e4, None) == 0 and L.hawk_rotary_table(None, 0, 8, 1e4, None) == 0


def test_bad_chains_are_refused(H):
    L = H.load_library()
    base = dict(p=ONE, ps=100, start=None, p_rows=9, q=ONE, qs=200, qr=100, d=ONE, nd=None, ua=ONE, uf=ONE, n_seq=3, k=2, n=100, t=1.0, top=5,
                on=ONE, ot=ONE, ws=ONE, nws=1 << 40, stream=None)
    call = lambda **kw: L.hawk_verify_chains(*{**base, **kw}.values())
    for kw in (dict(p=None), dict(d=None), dict(ua=None), dict(uf=None), dict(on=None), dict(ot=None), dict(ws=None), dict(ws=ONE + 8), dict(k=-1),
               dict(k=64), dict(n=0), dict(n=(1 << 20) + 1, ps=1 << 21, qr=1 << 21), dict(t=-0.5), dict(t=float("nan")), dict(top=0), dict(ps=99),
               dict(qr=99), dict(qs=-1), dict(p_rows=-1), dict(n_seq=-1), dict(n_seq=1 << 20)):
        assert call(**kw) == -1, kw
    need = L.hawk_verify_chains_workspace_bytes(3, 2, 100)
    assert need > 0 and call(nws=need - 1) == -3
    assert call(n_seq=0, p=None, d=None, ws=None) == 0
    for a in ((0, 2, 100), (3, -1, 100), (3, 64, 100), (3, 2, 0), (3, 2, (1 << 20) + 1)):
        assert L.hawk_verify_chains_workspace_bytes(*a) == 0


def test_a_keep_of_no_sequences_needs_no_buffers(H):
    L = H.load_library()
    assert L.hawk_paged_keep(C.byref(cache(n_seq=0, table=None)), None, None, None, 3, None) == 0
    assert L.hawk_paged_keep(C.byref(cache(n_seq=0)), None, None, None, 0, None) == -1


def test_a_keep_in_layers_that_share_memory_is_refused(H):
    """With no stride between layers every layer would move the same entries, one over the other's."""
    L = H.load_library()
    for stride in (0, 56):
        assert L.hawk_paged_keep(C.byref(cache(layer_stride=stride)), ONE, ONE, ONE, 3, None) == -1
    assert L.hawk_paged_keep(C.byref(cache(layer_stride=0, n_layers=1, n_seq=0)), None, None, None, 3, None) == 0


def test_host_tensors_are_refused(H):
    import torch
    with pytest.raises(hawk.HawkError):
        H.rotary_table(4, 8, device="cpu")
    f, i = torch.float32, torch.int32
    with pytest.raises(hawk.HawkError):
        H.verify_chains(torch.zeros(3, 9), None, torch.zeros(1, 2, dtype=i), torch.zeros(1, 2), torch.zeros(1), 1.0, 5)
    with pytest.raises(hawk.HawkError):
        H.verify_chains(torch.zeros(3, 9), None, torch.zeros(2, dtype=i), torch.zeros(1, 2), torch.zeros(1), 1.0, 5)
    with pytest.raises(hawk.HawkError):
        H.PagedCache(torch.zeros(2, 2, 2, 4, 8, dtype=f), torch.zeros(2, 2, 2, 4, 8, dtype=f), torch.zeros(1, 2, dtype=i))


def test_the_rule_of_the_cut_takes_any_sizes(H):
    L = H.load_library()
    for a in ((1, 3, 5, 0, 4, 64, 100, 0), (1, 3, 5, 2, 1, 64, 100, 0), (1, 0, 5, 2, 4, 64, 100, 0), (1, 3, -1, 2, 4, 64, 100, 0), (1, 3, 5, 2, 4, 64, 0, 0)):
        assert L.hawk_paged_attention_plan(*a) >= 0


def bad_starts():
    """Row starts as they must not be: descending, below 0, behind the rows, in any order; and one as it must."""
    rng = np.random.RandomState(7)
    far = [-2 ** 31, -1000, -1, 0, 5, 90, 99, 100, 101, 1000, 2 ** 31 - 1]
    for n_seq in (1, 3, 4, 70, 130):
        yield np.sort(rng.randint(0, 101, n_seq + 1))
        yield np.sort(rng.randint(0, 101, n_seq + 1))[::-1]
        for _ in range(3):
            yield rng.randint(-50, 160, n_seq + 1)
            yield rng.choice(far, n_seq + 1)
    yield np.array([0, 90, 0, 5])


@pytest.mark.parametrize("group,tile", [(1, 4), (4, 4), (3, 7), (8, 8)])
def test_no_row_starts_lead_a_tile_outside_the_buffers(H, group, tile):
    # Whichever sequence the search for a tile ends at, the rows of the tile are rows of that sequence and of the buffers.  (Of the last array,
    # 100 rows in groups of four, tile 2 taken as sequence 1's had row 2^30.)
    L, rows = H.load_library(), 100
    for starts in bad_starts():
        starts = np.ascontiguousarray(starts, dtype=np.int32)
        p, n_seq = starts.ctypes.data_as(C.c_void_p), len(starts) - 1
        tiles = (rows * group >> tile) + n_seq
        for s in sorted({0, 1, 2, n_seq // 2, n_seq - 1} & set(range(n_seq))):
            lo, hi = max(int(starts[s]), 0), min(int(starts[s + 1]), rows)
            for t in range(tiles):
                for r in {0, 1, group, (1 << tile) // 2, (1 << tile) - 1}:
                    row = L.hawk_paged_attention_row(p, 10, s, rows, group, 4096, tile, t, r)
                    assert row == -1 or lo <= row < hi, (starts, s, t, r, row)


@pytest.mark.parametrize("group,tile", [(1, 4), (4, 4), (3, 7), (8, 8)])
def test_tiles_hold_every_row_of_a_step_once(H, group, tile):
    L, rows = H.load_library(), 100
    starts = np.array([0, 0, 7, 8, 40, 40, 93], dtype=np.int32)
    p, n_seq = starts.ctypes.data_as(C.c_void_p), len(starts) - 1
    count = np.zeros(rows + 1, dtype=int)
    for s in range(n_seq):
        for t in range((rows * group >> tile) + n_seq):
            for r in range(1 << tile):
                count[L.hawk_paged_attention_row(p, 0, s, rows, group, 4096, tile, t, r)] += 1
    assert (count[:93] == group).all() and (count[93:rows] == 0).all()
