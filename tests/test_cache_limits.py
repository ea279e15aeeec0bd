"""The cache operators at the largest sizes: what the kernels' 32-bit positions
do not hold is refused on the host (no GPU needed)."""
import ctypes

import pytest

from paper_2607_20214_gb300 import build
from paper_2607_20214_gb300 import elsaa as E
from test_cache_abi import cache, calls

UNS, WS = E.ELSAA_ERR_UNSUPPORTED, E.ELSAA_ERR_WORKSPACE
MOST = 2 ** 31 - 2 ** 16


@pytest.fixture(scope="module")
def lib():
    build.build()
    return E.load_library()


@pytest.mark.parametrize("ps", [16, 32, 64, 128])
def test_tables_of_nearly_2_31_tokens_are_refused_everywhere(lib, ps):
    for pages in (2 ** 31 // ps - 1, MOST // ps + 1):
        c = cache(max_pages=pages, page_size=ps, H=2, H_kv=2, B=1)
        for name, call in calls(lib, c).items():
            assert call() == UNS, name
            assert "max_pages * page_size" in E.elsaa_last_error(), name
    # one page fewer: the next check speaks
    c = cache(max_pages=MOST // ps, page_size=ps, H=2, H_kv=2, B=1)
    for name, call in calls(lib, c, ws=None, keep=16).items():
        if name in ("select", "attention", "evict"):
            assert call() == WS, name
    assert calls(lib, c)["size"]() == E.ELSAA_OK


def test_eviction_to_nearly_2_31_tokens_is_refused(lib):
    for keep in (2 ** 31 - 1, MOST + 1):
        c = calls(lib, cache(), keep=keep, dst_pages=2 ** 31 - 1)
        for name in ("size", "evict"):
            assert c[name]() == UNS, name
            assert "keep" in E.elsaa_last_error(), name
    c = calls(lib, cache(), keep=MOST, dst_pages=2 ** 31 - 1, ws=None)
    assert c["size"]() == E.ELSAA_OK
    assert c["evict"]() == WS


@pytest.mark.parametrize("ps", [16, 128])
def test_selecting_nearly_2_31_pages_is_refused(lib, ps):
    for n_sel in (2 ** 31 - 1, MOST // ps + 1):
        c = calls(lib, cache(page_size=ps), n_sel=n_sel)
        assert c["select"]() == UNS
        assert "n_sel" in E.elsaa_last_error()
    c = calls(lib, cache(page_size=ps), n_sel=MOST // ps, ws=None)
    assert c["select"]() == WS


def test_appending_beyond_2_31_positions_is_refused(lib):
    """What the table holds and what the call may bring together: a sequence
    with fewer new rows than T may stand at its table's end."""
    for pages, ps, T in ((2 ** 24, 64, 2 ** 30), (4, 32, 2 ** 31 - 1),
                         (MOST // 128, 128, 128), (1, 16, MOST - 15)):
        c = cache(max_pages=pages, page_size=ps)
        assert calls(lib, c, T=T)["append"]() == UNS
        assert "T + max_pages * page_size" in E.elsaa_last_error()
    c = cache(max_pages=2 ** 24, page_size=64)
    assert calls(lib, c, T=2 ** 30 - 2 ** 16,
                 k=None)["append"]() == E.ELSAA_ERR_INVALID_ARG
