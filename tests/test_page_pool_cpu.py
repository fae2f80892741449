"""The pool of pages without a GPU: the plain form's own checks, and what the C
ABI and the binding refuse."""
import ctypes as C
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import pages
from paper_2608_13524_gb300 import dart

P = 1 << 20  # a pointer that is never followed: the refusals come before


def consistent(p):
    users = [0] * len(p.refs)
    for row in p.rows:
        assert len(set(row)) == len(row)
        for x in row:
            users[x] += 1
    assert users == p.refs


def test_the_plain_form_keeps_count():
    g = np.random.default_rng(0)
    for _ in range(30):
        nseq, page = int(g.integers(1, 8)), 16
        p, lens = pages.Pool(int(g.integers(4, 60)), page, nseq, 6), [0] * nseq
        for _ in range(20):
            op = g.integers(4)
            if op == 0:
                lens = p.select([int(x) for x in g.integers(-1, nseq, nseq)], lens)
            elif op == 1:
                rows = [int(x) for x in g.integers(-1, 40, nseq)]
                pairs, refused = p.reserve(lens, rows)
                assert len({b for _, b in pairs}) == len(pairs) and not {a for a, _ in pairs} & {b for _, b in pairs}
                lens = [n + max(r, 0) * (s not in refused) for s, (n, r) in enumerate(zip(lens, rows))]
                for s, row in enumerate(p.rows):  # the rows written now are on pages of their own
                    if s not in refused and rows[s] > 0:
                        assert all(p.refs[x] == 1 for x in row[(lens[s] - rows[s]) // page:])
            elif op == 2:
                lens = [int(g.integers(0, n + 1)) for n in lens]
                p.trim(lens)
            else:
                p.compact()
                assert all(r > 0 for r in p.refs[:sum(r > 0 for r in p.refs)])
            consistent(p)
            assert all(len(r) >= -(-n // page) for r, n in zip(p.rows, lens))


def pool_of(**kw):
    f = dict(num_pages=10, page_size=16, nseq=3, max_pages=4, refs=P, table=P, held=P)
    f.update(kw)
    return dart.DartPagePool(*f.values())


def calls(pool, lens=P, other=P, pairs=P, max_pairs=5, count=P, ws=P, n=1 << 40, status=None, parts=("select", "reserve", "trim", "compact")):
    L, p = dart.lib(), C.byref(pool)
    got = dict(select=lambda: L.dart_page_pool_select(p, other, lens, ws, n, status, None),
               reserve=lambda: L.dart_page_pool_reserve(p, lens, other, pairs, max_pairs, count, ws, n, status, None),
               trim=lambda: L.dart_page_pool_trim(p, lens, status, None),
               compact=lambda: L.dart_page_pool_compact(p, pairs, max_pairs, count, ws, n, status, None))
    return [got[m]() for m in parts]


@pytest.mark.parametrize("bad", [dict(num_pages=0), dict(num_pages=2 ** 30 + 1), dict(page_size=48), dict(page_size=8), dict(nseq=0), dict(max_pages=0),
                                 dict(nseq=2 ** 20, max_pages=2 ** 11), dict(max_pages=2 ** 27, page_size=16), dict(refs=None), dict(refs=P + 4),
                                 dict(table=None), dict(table=P + 2), dict(held=None)], ids=str)
def test_bad_pools_are_refused(bad):
    assert set(calls(pool_of(**bad))) == {dart.DART_ERR_INVALID}
    if not {"refs", "table", "held"} & set(bad):
        assert dart.lib().dart_page_pool_workspace(C.byref(pool_of(**bad))) == 0


@pytest.mark.parametrize("bad,parts", [(dict(lens=None), ("select", "reserve", "trim")), (dict(lens=P + 2), ("select", "reserve", "trim")),
                                       (dict(other=None), ("select", "reserve")), (dict(other=P + 1), ("select", "reserve")),
                                       (dict(pairs=None), ("reserve", "compact")), (dict(pairs=P + 4), ("reserve", "compact")),
                                       (dict(max_pairs=2), ("reserve", "compact")), (dict(max_pairs=4), ("compact",)), (dict(count=None), ("reserve", "compact")),
                                       (dict(ws=None), ("select", "reserve", "compact")), (dict(ws=P + 128), ("select", "reserve", "compact")),
                                       (dict(n=100), ("select", "reserve", "compact")), (dict(status=P + 1), ("select", "reserve", "trim", "compact"))], ids=str)
def test_bad_arguments_are_refused(bad, parts):
    assert set(calls(pool_of(), parts=parts, **bad)) == {dart.DART_ERR_INVALID}


def test_workspace_grows_with_the_pool():
    size = lambda **kw: dart.lib().dart_page_pool_workspace(C.byref(pool_of(**kw)))  # noqa: E731
    assert 0 < size() < size(num_pages=10 ** 6) and size() < size(nseq=1000) < size(nseq=1000, max_pages=1000)


@pytest.mark.parametrize("bad", [dict(pairs=None), dict(pairs=P + 4), dict(max_pairs=0), dict(count=None), dict(count=P + 2), dict(status=P + 2)], ids=str)
def test_bad_copies_are_refused(bad):
    f = dict(pairs=P, max_pairs=4, count=P, status=None)
    f.update(bad)
    c = dart.DartKvCache(4, 16, 2, 128, dart.DART_KV_E4M3, P, P, P, P, None, None)
    assert dart.lib().dart_cache_copy_pages(C.byref(c), *f.values(), None) == dart.DART_ERR_INVALID


def test_copies_of_pages_beyond_32_bits_are_refused():
    c = dart.DartKvCache(1, 128, 2 ** 23, 128, dart.DART_KV_BF16, P, P, None, None, None, None)
    assert dart.lib().dart_cache_copy_pages(C.byref(c), P, 4, P, None, None) == dart.DART_ERR_INVALID


def fake(shape, dtype=torch.int32, dev=0):
    return SimpleNamespace(shape=torch.Size(shape), dtype=dtype, get_device=lambda: dev, is_contiguous=lambda: True, data_ptr=lambda: P, device=dev)


def test_the_binding_refuses_other_tensors(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    monkeypatch.setattr(dart, "_empty", lambda shape, dtype, device: torch.empty(shape, dtype=dtype))
    p = dart.PagePool(10, 16, 3, 4)
    assert p.table.shape == (3, 4) and p.pairs.shape == (5, 2) and not p.refs.any() and not p.held.any()
    good = fake((3,))
    for t in (None, fake((2,)), fake((3,), torch.int64), fake((3,), dev=1)):
        for call in (lambda: p.select(t, good), lambda: p.select(good, t), lambda: p.reserve(t, good), lambda: p.reserve(good, t), lambda: p.trim(t)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        p.trim(good, status=fake((1,), torch.float32))
    with pytest.raises(ValueError):
        p.compact(status=fake((1,), torch.int64))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: p.select(good, good), lambda: p.reserve(good, good), lambda: p.trim(good), p.compact):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("shape", [(0, 16, 3, 4), (10, 15, 3, 4), (10, 16, 0, 4), (10, 16, 3, 0)], ids=str)
def test_the_binding_refuses_other_sizes(shape):
    with pytest.raises(dart.DartError):
        dart.PagePool(*shape)
