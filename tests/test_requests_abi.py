"""Pages, adapters and filtered draws without a GPU: what is refused before any launch, and what needs no buffers."""
import ctypes as C

import pytest

from paper_2510_25739_amd import hawk

ONE = 4096      # an address: every call below fails, or has nothing to do, before anything is read through it


@pytest.fixture(scope="module")
def L():
    import os
    import paper_2510_25739_amd as H
    if not os.path.exists(H.lib_path()):
        from paper_2510_25739_amd import build
        build.build()
    return H.load_library()


def cache(**kw):
    f = dict(k=ONE, v=ONE, layer_stride=1 << 20, page_stride=16 * 2 * 64, head_stride=16 * 64, entry_stride=64, table=ONE, table_stride=8,
             dtype=hawk.HAWK_FP16, n_layers=2, n_pages=10, page_size=16, n_heads=2, head_dim=64, n_seq=3, max_pages=8)
    f.update(kw)
    return hawk.HawkPagedCache(**f)


BAD_CACHE = [dict(k=None), dict(v=ONE + 8), dict(table=None), dict(dtype=3), dict(head_dim=60), dict(n_pages=0), dict(n_seq=-1), dict(table_stride=7),
             dict(entry_stride=56)]


def calls(L, c, refs=ONE, past=ONE, new=ONE, short=ONE, src=ONE, dst=ONE, n=2, out=ONE, stride=8, refs_out=ONE, used=ONE, ws=ONE, nws=1 << 30):
    r = C.byref(c)
    return dict(fork=L.hawk_paged_fork(r, refs, past, src, dst, n, None), take=L.hawk_paged_take(r, refs, past, new, short, ws, nws, None),
                trim=L.hawk_paged_trim(r, refs, past, None), compact=L.hawk_paged_compact(r, refs, out, stride, refs_out, used, ws, nws, None),
                copy=L.hawk_paged_copy(r, r, src, dst, n, None))


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_bad_caches_are_refused(L, bad):
    c = cache(**bad)
    assert set(calls(L, c).values()) == {-1}
    assert L.hawk_paged_pages_workspace_bytes(C.byref(c)) == 0


def test_bad_page_calls_are_refused(L):
    need = L.hawk_paged_pages_workspace_bytes(C.byref(cache()))
    assert need > 0 and need % 16 == 0

    def refused(which, code=-1, c=None, **kw):
        # the calls that are not asked about get a pool that refuses them
        c = c or cache()
        r = C.byref(c)
        a = dict(refs=ONE, past=ONE, new=ONE, short=ONE, src=ONE, dst=ONE, n=2, out=ONE, stride=8, refs_out=ONE, used=ONE, ws=ONE, nws=need)
        a.update(kw)
        got = {"fork": lambda: L.hawk_paged_fork(r, a["refs"], a["past"], a["src"], a["dst"], a["n"], None),
               "take": lambda: L.hawk_paged_take(r, a["refs"], a["past"], a["new"], a["short"], a["ws"], a["nws"], None),
               "trim": lambda: L.hawk_paged_trim(r, a["refs"], a["past"], None),
               "compact": lambda: L.hawk_paged_compact(r, a["refs"], a["out"], a["stride"], a["refs_out"], a["used"], a["ws"], a["nws"], None),
               "copy": lambda: L.hawk_paged_copy(r, r, a["src"], a["dst"], a["n"], None)}[which]()
        assert got == code, (which, kw, got)

    for which, names in dict(fork=("refs", "past", "src", "dst"), take=("refs", "past", "new", "short", "ws"), trim=("refs", "past"),
                             compact=("refs", "out", "refs_out", "used", "ws"), copy=("src", "dst")).items():
        for name in names:
            refused(which, **{name: None})
    refused("fork", n=-1)
    refused("fork", n=4)                # more pairs than sequences
    refused("fork", n=(1 << 23) + 1, c=cache(n_seq=1 << 24))
    refused("copy", n=-1)
    refused("copy", n=(1 << 20) + 1)
    refused("compact", stride=7)
    refused("compact", stride=9)         # in place, but rows that would be written over rows not yet read
    for which in ("take", "compact"):
        refused(which, ws=ONE + 8)
        refused(which, -3, nws=need - 1)
        refused(which, c=cache(layer_stride=0))                                              # layers in one another's place
        refused(which, c=cache(n_seq=1 << 24, max_pages=1 << 7, table_stride=1 << 7))        # more places than are counted
    refused("copy", c=cache(layer_stride=0))
    a, b = cache(), cache(n_layers=1)
    for kw in (dict(n_layers=1), dict(dtype=hawk.HAWK_BF16), dict(page_size=8, page_stride=2048), dict(n_heads=1), dict(head_dim=32)):
        b = cache(**kw)
        assert L.hawk_paged_copy(C.byref(a), C.byref(b), ONE, ONE, 2, None) == -1, kw


def test_page_calls_without_work_need_no_buffers(L):
    c = cache(n_seq=0, table=None)
    r = C.byref(c)
    assert L.hawk_paged_fork(r, None, None, None, None, 0, None) == 0 and L.hawk_paged_trim(r, None, None, None) == 0
    assert L.hawk_paged_take(r, None, None, None, None, None, 0, None) == 0 and L.hawk_paged_copy(r, r, None, None, 0, None) == 0


def test_plan_sizes(L):
    size = L.hawk_adapter_plan_bytes
    for rows, n in ((-1, 1), (1, -1), ((1 << 22) + 1, 1), (1, 8193)):
        assert size(rows, n) == 0
    for rows, n in ((0, 0), (0, 5), (1, 0), (1, 1), (16, 3), (17, 3), (4001, 8), (1 << 22, 8192)):
        # a tile of 16 rows and one more a class with rows, each with its adapter; two words a row
        tiles = rows // 16 + min(rows, n + 1)
        words = 4 + 17 * tiles
        assert size(rows, n) == 4 * ((words + 1) // 2 * 2 + 2 * rows)


def adapters(**kw):
    return hawk.HawkAdapters(**{**dict(a=ONE, b=ONE, a_adapter_stride=8 * 64, a_row_stride=64, b_adapter_stride=40 * 8, b_row_stride=8, scale=None,
                                       dtype=hawk.HAWK_BF16, n_adapters=3, rank=8, d_in=64, d_out=40), **kw})


def matrix(width, **kw):
    return hawk.HawkMatrix(**{**dict(data=ONE, row_stride=width, dtype=hawk.HAWK_BF16), **kw})


def test_bad_adapter_calls_are_refused(L):
    need = L.hawk_adapter_plan_bytes(5, 3)

    def plan(start=ONE, adapter=ONE, n_seq=2, rows=5, n=3, plan=ONE, nbytes=need):
        return L.hawk_adapter_plan(start, adapter, n_seq, rows, n, plan, nbytes, None)

    for kw in (dict(start=None), dict(adapter=None), dict(n_seq=-1), dict(rows=-1), dict(n=-1), dict(n=8193), dict(plan=None), dict(plan=ONE + 8)):
        assert plan(**kw) == -1, kw
    assert plan(nbytes=need - 1) == -3

    def apply(w=None, plan=ONE, nbytes=need, rows=5, x=None, base=None, out=None, **kw):
        ref = lambda m: None if m is None else C.byref(m)
        return L.hawk_adapter_apply(ref(w or adapters(**kw)), plan, nbytes, rows, ref(x or matrix(64)), ref(base), ref(out or matrix(40, data=1 << 20)), None, 0, None)

    for kw in (dict(rank=0), dict(rank=12), dict(rank=136, b_row_stride=136), dict(d_in=0), dict(d_in=60), dict(d_in=72), dict(d_out=44), dict(d_out=0),
               dict(dtype=5), dict(n_adapters=-1), dict(a=None), dict(b=None), dict(a=ONE + 2), dict(b=ONE + 8), dict(a_row_stride=68),
               dict(b_row_stride=0), dict(a_adapter_stride=-8), dict(b_adapter_stride=4), dict(plan=None), dict(plan=ONE + 4), dict(rows=-1),
               dict(x=matrix(64, dtype=hawk.HAWK_FP16)), dict(x=matrix(64, data=None)), dict(x=matrix(64, data=ONE + 8)), dict(x=matrix(64, row_stride=68)),
               dict(x=matrix(64, row_stride=-64)), dict(base=matrix(40, dtype=hawk.HAWK_FP32)), dict(base=matrix(40, data=None)),
               dict(base=matrix(40, data=1 << 20, row_stride=48)), dict(out=matrix(40, row_stride=32)), dict(out=matrix(40, dtype=9))):
        assert apply(**kw) == -1, kw
    assert apply(nbytes=need - 1) == -3
    assert apply(rows=0, a=None, b=None, n_adapters=0, plan=None, x=matrix(64, data=None)) == 0


def test_sums_shared_by_workgroups_need_a_workspace(L):
    def size(rows=5, **kw):
        return L.hawk_adapter_apply_workspace_bytes(C.byref(adapters(**kw)), rows)

    wide = dict(rank=128, d_in=4096, a_row_stride=4096, b_row_stride=128)
    need = size(**wide)
    assert need > 0 and need % 16 == 0
    assert size() == 0 and size(rank=128) == 0 and size(rows=4096, **wide) == 0      # a little to read, or many tiles
    assert size(rows=0, **wide) == 0 and size(rows=-1, **wide) == 0 and size(rows=5, **{**wide, "rank": 12}) == 0
    w, plan = C.byref(adapters(**wide)), L.hawk_adapter_plan_bytes(5, 3)
    x, out = matrix(4096), matrix(40, data=1 << 20)
    for ws, n, code in ((None, need, -1), (ONE + 8, need, -1), (ONE, need - 1, -3), (ONE, 0, -3)):
        assert L.hawk_adapter_apply(w, ONE, plan, 5, C.byref(x), None, C.byref(out), ws, n, None) == code
    assert L.hawk_adapter_apply(w, ONE, plan, 0, C.byref(x), None, C.byref(out), None, 0, None) == 0


def test_bad_filtered_draws_are_refused(L):
    def call(logits=ONE, dtype=0, stride=100, u=ONE, rows=3, n=100, token=ONE):
        return L.hawk_sample_filtered(logits, dtype, stride, None, u, None, None, None, None, rows, n, token, None, None, ONE, 1 << 40, None)

    for kw in (dict(logits=None), dict(logits=ONE + 2), dict(dtype=4), dict(dtype=-1), dict(stride=99), dict(u=None), dict(rows=-1), dict(rows=(1 << 22) + 1),
               dict(n=0), dict(n=(1 << 20) + 1, stride=1 << 21), dict(token=None), dict(dtype=1, logits=ONE + 1)):
        assert call(**kw) == -1, kw
    assert call(rows=0, logits=None, u=None, token=None) == 0


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    import torch
    import paper_2510_25739_amd as H
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(H.HawkError):
        H.AdapterPlan(i, i[:2], 4, 2)
    with pytest.raises(H.HawkError):
        H.sample_filtered(torch.zeros(2, 5), torch.zeros(2))
