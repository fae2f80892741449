"""e2m1 pages without a GPU: the plain forms' own checks, and what the C ABI and
the binding refuse."""
import ctypes as C
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import four
from paper_2608_13524_gb300 import dart


def test_grids_and_ties():
    assert four.E4M3[-1] == 448.0 and len(four.E4M3) == 127 and (np.diff(four.E4M3) > 0).all()
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    assert four.nearest(four.E2M1, mids).tolist() == [0, 2, 2, 4, 4, 6, 6]
    eps = 2.0 ** -40
    assert four.nearest(four.E2M1, mids * (1 - eps)).tolist() == list(range(7))
    assert four.nearest(four.E2M1, mids * (1 + eps)).tolist() == list(range(1, 8))
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, four.E4M3)


def test_rows_that_lie_on_the_grid_come_back():
    g = np.random.default_rng(0)
    code = g.integers(0, 16, (50, 128)).astype(np.uint8)
    code[:, ::16] = 7  # (each block's largest is 6 of its scale)
    block = g.integers(0x68, 0x78, (50, 8)).astype(np.uint8)  # 64 .. 240
    block[:, 3] = 0x7A  # 320: the row's largest is in [1024, 2048)
    x = four.values(code, block, np.full(50, 2.0 ** -3))
    c, b, s = four.quantise(x)
    assert np.array_equal(four.values(c, b, s), x) and (s == 2.0 ** -3).all() and np.array_equal(b, block)
    assert np.array_equal(four.unpack(four.pack(c)), c)


def test_bounds_of_the_rounding():
    """An element is off by half a step of its block at most: a sixth of the
    block's largest magnitude, an eighth more where the block scale was rounded
    up to 2^-4 of itself."""
    g = np.random.default_rng(1)
    x = g.standard_normal((200, 128)) * np.exp(g.normal(0, 3, (200, 1)))
    c, b, s = four.quantise(x)
    assert b.max() <= four.nearest(four.E4M3, 342.0) and (np.frexp(np.abs(x).max(1) / s)[1] == 11).all()
    top = np.abs(x).reshape(200, 8, 16).max(-1, keepdims=True)
    off = np.abs(four.values(c, b, s) - x).reshape(200, 8, 16)
    assert (off <= top / 6 * (1 + 2.0 ** -4) + s[:, None, None] * 2.0 ** -10).all()


def test_nan_and_infinity_stay_in_their_block():
    x = np.ones((1, 128))
    x[0, 17], x[0, 70] = np.nan, -np.inf
    c, b, s = four.quantise(x)
    v = four.values(c, b, s)[0]
    assert np.isnan(v[16:32]).all() and np.isnan(v[64:80]).all() and s[0] == 2.0 ** -10
    assert (np.delete(v, np.r_[16:32, 64:80]) == four.values(*four.quantise(np.ones((1, 128))))[0, 0]).all()


def test_zero_rows():
    c, b, s = four.quantise(np.zeros((1, 128)))
    assert not c.any() and not b.any() and s[0] == 1.0


# ------------------------------------------------------------ refusals

P = 1 << 20  # a pointer that is never followed: the refusals come before


def cache_of(**kw):
    f = dict(num_pages=4, page_size=16, Hkv=2, dh=128, dtype=dart.DART_KV_E2M1, k=P, v=P, k_scale=P, v_scale=P, k_block=P, v_block=P)
    f.update(kw)
    return dart.DartKvCache(*f.values())


def read(cache, **kw):
    f = dict(nseq=1, max_pages=4, table=P, lens=P, R=2, k=P, ks=256, v=P, vs=256, n_rows=P, status=None)
    f.update(kw)
    return dart.lib().dart_cache_read(C.byref(cache), *f.values(), None)


def append(cache):
    return dart.lib().dart_cache_append(C.byref(cache), 1, 4, P, P, 2, P, 256, P, 256, None, P, 1.0e6, None, None)


BAD_CACHES = [dict(dtype=3), dict(dtype=-1), dict(k_scale=None), dict(v_scale=None), dict(k_block=None), dict(v_block=None), dict(k_block=P + 8),
              dict(v_block=P + 4), dict(k=P + 8), dict(v=None), dict(dh=64), dict(page_size=48), dict(num_pages=0), dict(Hkv=0),
              dict(num_pages=2 ** 30, Hkv=8)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(bad):
    c = cache_of(**bad)
    assert append(c) == read(c) == dart.DART_ERR_INVALID
    cfg = dart.DartPagedAttnConfig(1, 0, 4, 2, 1.0e6, 0.1)
    assert dart.lib().dart_paged_attention(C.byref(cfg), C.byref(c), P, P, P, 256, P, 256, P, 256, None, None, None, P, P, 1 << 40, None,
                                           None) == dart.DART_ERR_INVALID


@pytest.mark.parametrize("bad", [dict(nseq=0), dict(max_pages=0), dict(R=0), dict(table=None), dict(lens=P + 2), dict(n_rows=None), dict(k=P + 2),
                                 dict(v=None), dict(ks=255), dict(vs=248), dict(ks=260), dict(status=P + 1), dict(max_pages=2 ** 30),
                                 dict(R=2 ** 30, nseq=8)], ids=str)
def test_bad_reads_are_refused(bad):
    assert read(cache_of(), **bad) == dart.DART_ERR_INVALID


def fake(shape, dtype):
    return SimpleNamespace(shape=torch.Size(shape), dtype=dtype, dim=lambda: len(shape), get_device=lambda: 0, is_contiguous=lambda: True,
                           data_ptr=lambda: P, device="cuda:0")


def four_pool(**kw):
    F4, E4, F32 = torch.float4_e2m1fn_x2, torch.float8_e4m3fn, torch.float32
    f = dict(k=((4, 2, 16, 64), F4), v=((4, 2, 16, 64), F4), k_scale=((4, 2, 16), F32), v_scale=((4, 2, 16), F32),
             k_block=((4, 2, 16, 8), E4), v_block=((4, 2, 16, 8), E4))
    f.update(kw)
    return {m: None if x is None else fake(*x) for m, x in f.items()}


def test_the_binding_takes_four_bit_pages(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    c = dart.KVCache(**four_pool())
    assert (c.dh, c.page_size, c.Hkv, c.num_pages) == (128, 16, 2, 4)
    assert (c.c.dh, c.c.dtype, c.c.k_block) == (128, dart.DART_KV_E2M1, P)


E4 = torch.float8_e4m3fn


@pytest.mark.parametrize("bad", [dict(k_scale=None), dict(v_block=None), dict(k_block=((4, 2, 16, 16), E4)), dict(k_block=((4, 2, 16, 8), torch.uint8)),
                                 dict(v=((4, 2, 16, 128), torch.float4_e2m1fn_x2)), dict(k=((4, 2, 16, 64), torch.uint8)),
                                 dict(v=((4, 2, 16, 64), E4)), dict(v_scale=((4, 2, 8), torch.float32))], ids=str)
def test_the_binding_refuses_other_tensors(bad, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError):
        dart.KVCache(**four_pool(**bad))


def test_block_scales_belong_to_four_bits(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    k, b, s = ((4, 2, 16, 128), E4), ((4, 2, 16, 8), E4), ((4, 2, 16), torch.float32)
    with pytest.raises(ValueError):
        dart.KVCache(fake(*k), fake(*k), fake(*s), fake(*s), fake(*b), fake(*b))


def test_workspace_of_four_bit_pages():
    """Small trees stream the pages or convert them in the CTA; large ones have
    room for f16 tiles, as e4m3 pages have."""
    four_c, eight = cache_of(num_pages=1000, page_size=64, Hkv=8), cache_of(num_pages=1000, page_size=64, Hkv=8, dtype=dart.DART_KV_E4M3)
    for B in (0, 3, 31, 512):
        cfg = dart.DartPagedAttnConfig(8, B, 32, 32, 1.0e6, 0.1)
        a, b = (dart.lib().dart_paged_attention_workspace(C.byref(cfg), C.byref(c)) for c in (four_c, eight))
        assert a == b > 0
