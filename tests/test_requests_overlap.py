"""Buffers of the calls for many requests that lie over one another, without a GPU: what would race is refused, what is only interleaved is not.
Calls that are not refused for it are refused for their workspace, so that nothing is launched."""
import ctypes as C
import itertools

import pytest

from paper_2510_25739_amd import hawk

ROWS = 5


@pytest.fixture(scope="module")
def L():
    import os
    import paper_2510_25739_amd as H
    if not os.path.exists(H.lib_path()):
        from paper_2510_25739_amd import build
        build.build()
    return H.load_library()


def apply(L, x, out, base=None, rows=ROWS, d_in=64, d_out=40, tx=hawk.HAWK_BF16, tout=hawk.HAWK_BF16):
    """x, out, base: (address, row stride).  -1: refused; -3: the plan's memory is too small, which is looked at last."""
    w = hawk.HawkAdapters(a=1 << 30, b=1 << 30, a_adapter_stride=8 * d_in, a_row_stride=d_in, b_adapter_stride=8 * d_out, b_row_stride=8, scale=None, dtype=tx,
                          n_adapters=3, rank=8, d_in=d_in, d_out=d_out)
    m = lambda at, t: None if at is None else C.byref(hawk.HawkMatrix(data=at[0], row_stride=at[1], dtype=t))
    return L.hawk_adapter_apply(C.byref(w), 1 << 20, 16, rows, m(x, tx), m(base, tout), m(out, tout), None, 0, None)


def test_a_result_over_its_input_is_refused(L):
    at = 1 << 16
    assert apply(L, (at, 64), (at, 64), d_out=64) == -1                              # out = x
    assert apply(L, (at, 64), (at, 64), (at, 64), d_out=64) == -1                    # base = out = x
    assert apply(L, (at, 64), (at + 64 * 2, 64), d_out=64) == -1                     # a row further
    assert apply(L, (at, 64), (at + 16, 64)) == -1                                   # inside the rows
    assert apply(L, (at + (ROWS * 64 - 8) * 2, 64), (at, 64), d_out=64) == -1        # the last piece
    assert apply(L, (at, 0), (at + 3 * 128, 64)) == -3 and apply(L, (at + 3 * 128, 0), (at, 64)) == -1    # one row for all: beside the result, in it
    assert apply(L, (at, 64), (1 << 18, 40), (1 << 18, 40)) == -3                    # base = out
    assert apply(L, (at, 64), (1 << 18, 40), ((1 << 18) + 16, 40)) == -1             # shifted against one another
    assert apply(L, (at, 64), ((1 << 18) + 80, 40), (1 << 18, 40)) == -1
    assert apply(L, (at, 64), (1 << 18, 40), ((1 << 18) + 80 * 2, 0)) == -1          # one row for all, which is a row of the result


def test_interleaved_rows_are_not(L):
    at = 1 << 16
    assert apply(L, (at, 104), (at + 128, 104)) == -3                                # columns 0 .. 63 and 64 .. 103 of one buffer
    assert apply(L, (at + 80, 104), (at, 104)) == -3
    assert apply(L, (at + 80, 144), (at, 144), (at + 208, 144)) == -3                # out, x and base side by side
    assert apply(L, (at, 104), (at + 120 * 1, 104)) == -1                            # (a pointer that is not aligned)
    assert apply(L, (at, 104), (at + 112, 104)) == -1                                # eight columns too near
    assert apply(L, (at + ROWS * 128, 64), (at, 64), d_out=64) == -3                 # one behind the other
    assert apply(L, (at, 1 << 40), (at + 128, 1 << 40), rows=1) == -3                # the stride of one row is not used


def test_every_arrangement_of_a_few_rows(L):
    """Against sets of addresses, with strides that differ (32 and 16 bits) and that are the same."""
    at, width = 1 << 16, {hawk.HAWK_BF16: 2, hawk.HAWK_FP32: 4}
    for rows, sx, so, tout, shift in itertools.product((1, 2, 4), (0, 16, 24, 40), (8, 24, 40), width, range(-320, 321, 16)):
        d_in, d_out = 16, 8
        covered = lambda p, stride, n, es: {p + r * stride * es + b for r in range(rows) for b in range(0, n * es, 2)}
        meet = bool(covered(at, sx, d_in, 2) & covered(at + shift, so, d_out, width[tout]))
        assert apply(L, (at, sx), (at + shift, so), rows=rows, d_in=d_in, d_out=d_out, tout=tout) == (-1 if meet else -3), (rows, sx, so, tout, shift)


def cache(at, stride=8, **kw):
    return hawk.HawkPagedCache(**{**dict(k=1 << 30, v=1 << 31, layer_stride=1 << 20, page_stride=16 * 2 * 64, head_stride=16 * 64, entry_stride=64, table=at,
                                         table_stride=stride, dtype=hawk.HAWK_FP16, n_layers=2, n_pages=10, page_size=16, n_heads=2, head_dim=64, n_seq=3,
                                         max_pages=8), **kw})


def compact(L, table, out, refs=1 << 18, refs_out=1 << 19, n_seq=3):
    """table, out: (address, row stride).  -1: refused; -3: the workspace is too small, which is looked at last."""
    return L.hawk_paged_compact(C.byref(cache(*table, n_seq=n_seq)), refs, out[0], out[1], refs_out, 1 << 21, 1 << 22, 16, None)


def test_tables_and_counts_that_lie_over_one_another_in_part_are_refused(L):
    at = 1 << 16
    assert compact(L, (at, 8), (at, 8)) == -3                                        # in place
    assert compact(L, (at, 8), (at + 3 * 32, 8)) == -3                               # one behind the other
    assert compact(L, (at, 8), (at + 32, 8)) == -1                                   # a row further
    assert compact(L, (at + 4, 8), (at, 8)) == -1
    assert compact(L, (at, 16), (at + 32, 16)) == -3                                 # side by side in one array
    assert compact(L, (at, 16), (at + 28, 16)) == -1
    assert compact(L, (at, 16), (at, 8)) == -1 and compact(L, (at, 16), (at, 8), n_seq=1) == -3
    assert compact(L, (at, 8), (at, 8), refs=1 << 18, refs_out=1 << 18) == -3
    for by in (-36, -4, 4, 36):
        assert compact(L, (at, 8), (at, 8), refs_out=(1 << 18) + by) == -1
    for by in (-40, 40):
        assert compact(L, (at, 8), (at, 8), refs_out=(1 << 18) + by) == -3
