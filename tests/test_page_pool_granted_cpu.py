"""The refusals of dart_page_pool_reserve_rows, on the host."""
import ctypes as C

import pytest

from paper_2608_13524_gb300 import dart
from test_page_pool_cpu import P, pool_of


def reserve_rows(pool, **kw):
    f = dict(lens=P, n_rows=P, granted=P, pairs=P, max_pairs=5, count=P, ws=P, n=1 << 40, status=None)
    f.update(kw)
    return dart.lib().dart_page_pool_reserve_rows(C.byref(pool), *f.values(), None)


@pytest.mark.parametrize("bad", [dict(granted=None), dict(granted=P + 2), dict(lens=None), dict(n_rows=None), dict(n_rows=P + 1), dict(pairs=P + 4),
                                 dict(max_pairs=2), dict(count=None), dict(ws=P + 128), dict(n=100), dict(status=P + 1)], ids=str)
def test_bad_arguments_are_refused(bad):
    assert reserve_rows(pool_of(), **bad) == dart.DART_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(num_pages=0), dict(page_size=48), dict(nseq=0), dict(refs=None), dict(table=P + 2), dict(held=None)], ids=str)
def test_bad_pools_are_refused(bad):
    assert reserve_rows(pool_of(**bad)) == dart.DART_ERR_INVALID
