"""Tables whose rows are further apart than they are long, through the C calls: what the same life gives with rows behind one another, and nothing
written between the rows."""
import ctypes as C

import pytest

from test_gpu_pages import DEV, H, i32   # noqa: F401

pytestmark = pytest.mark.gpu

N_SEQ, COLS, PAGES, PAD = 5, 6, 24, 77


def life(H, stride, out_stride, in_place):   # noqa: F811
    """Table, counts and entries after takes, forks, a trim and a compaction; what lies between the rows is PAD."""
    import torch
    from paper_2510_25739_amd import hawk
    L = H.load_library()
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(2, PAGES, 2, 4, 8, generator=g).to(DEV) for _ in range(2))

    def rows(step):
        t = torch.full((N_SEQ * step,), PAD, dtype=torch.int32, device=DEV).view(N_SEQ, step)
        t[:, :COLS] = -1
        return t

    table, out, refs, past, short, used = rows(stride), rows(out_stride), i32([0] * PAGES), i32([0] * N_SEQ), i32([9] * N_SEQ), i32([0])
    c = hawk.HawkPagedCache(k=k.data_ptr(), v=v.data_ptr(), layer_stride=k.stride(0), page_stride=k.stride(1), head_stride=k.stride(2), entry_stride=8,
                            table=table.data_ptr(), table_stride=stride, dtype=hawk.HAWK_FP32, n_layers=2, n_pages=PAGES, page_size=4, n_heads=2, head_dim=8,
                            n_seq=N_SEQ, max_pages=COLS)
    n = L.hawk_paged_pages_workspace_bytes(C.byref(c))
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    seen = []

    def take(new):
        assert L.hawk_paged_take(C.byref(c), refs.data_ptr(), past.data_ptr(), i32(new).data_ptr(), short.data_ptr(), ws.data_ptr(), n, stream) == 0
        torch.cuda.synchronize()
        seen.append(short.tolist())
        past.add_(i32([x if x > 0 and not s else 0 for x, s in zip(new, seen[-1])]))

    take([9, 14, 0, 0, -1])
    a, b = i32([0, 1]), i32([3, 4])
    assert L.hawk_paged_fork(C.byref(c), refs.data_ptr(), past.data_ptr(), a.data_ptr(), b.data_ptr(), 2, stream) == 0
    take([0, 3, 2, 2, 5])
    past[1] = 0
    assert L.hawk_paged_trim(C.byref(c), refs.data_ptr(), past.data_ptr(), stream) == 0
    to = table if in_place else out
    assert L.hawk_paged_compact(C.byref(c), refs.data_ptr(), to.data_ptr(), to.stride(0), refs.data_ptr(), used.data_ptr(), ws.data_ptr(), n, stream) == 0
    torch.cuda.synchronize()
    for t in (table, out):
        assert bool((t[:, COLS:] == PAD).all())
    return seen, to[:, :COLS].tolist(), refs.tolist(), past.tolist(), used.tolist(), k.cpu(), v.cpu()


@pytest.mark.parametrize("stride,out_stride,in_place", [(6, 11, False), (9, 6, False), (9, 9, False), (64, 7, False), (9, 6, True)])
def test_rows_of_tables_apart(H, stride, out_stride, in_place):   # noqa: F811
    import torch
    want, got = life(H, COLS, COLS, False), life(H, stride, out_stride, in_place)
    assert got[:5] == want[:5]
    assert torch.equal(got[5], want[5]) and torch.equal(got[6], want[6])
    assert sum(n > 0 for n in got[2]) == got[4][0] and any(x > 0 for row in got[1] for x in row)
