"""The largest pools and forks that the page calls take, without a GPU: beyond them they are refused before any launch."""
import ctypes as C

from paper_2510_25739_amd import hawk
from test_requests_abi import ONE, L, cache   # noqa: F401


def test_pools_whose_page_numbers_would_wrap_are_refused(L):   # noqa: F811
    # lookups go through the counts in rounds of 16384: a round behind the last page has to have numbers of 31 bits as well
    most = (1 << 31) - (1 << 15)
    thin = dict(page_size=1, n_heads=1, head_dim=8, page_stride=8, head_stride=8, entry_stride=8, n_layers=1)
    for n, code in ((most, -3), (most + 1, -1), ((1 << 31) - 1, -1)):
        c = cache(n_pages=n, **thin)
        r = C.byref(c)
        assert (L.hawk_paged_pages_workspace_bytes(r) > 0) == (code == -3)
        assert L.hawk_paged_take(r, ONE, ONE, ONE, ONE, ONE, 16, None) == code          # (a workspace that is too small)
        assert L.hawk_paged_compact(r, ONE, ONE, 8, ONE, ONE, ONE, 16, None) == code
    assert L.hawk_paged_copy(r, r, ONE, ONE, 1, None) == -1


def test_forks_of_more_pairs_than_are_compared_in_a_moment_are_refused(L):   # noqa: F811
    r = C.byref(cache(n_seq=1 << 24))
    for n in ((1 << 18) + 1, 1 << 20, 1 << 23):
        assert L.hawk_paged_fork(r, ONE, ONE, ONE, ONE, n, None) == -1
