"""Argument checks of the paged cache, its attention and the tree
verification: refused on the host before any CUDA call is made.  The oracle's
own checks are here too."""
import ctypes as C

import numpy as np
import pytest

from oracle import serve, tree_attn
from paper_2608_13524_gb300 import dart

INV = dart.DART_ERR_INVALID


def mem():
    buf = (C.c_uint8 * 2048)()
    return buf, (C.cast(buf, C.c_void_p).value + 255) & ~255


def cache(p, **kw):
    base = dict(num_pages=4, page_size=16, Hkv=2, dh=128, dtype=1, k=p, v=p, k_scale=p, v_scale=p)
    base.update(kw)
    return dart.DartKvCache(*base.values())


CACHE_BAD = [dict(num_pages=0), dict(num_pages=-1), dict(page_size=0), dict(page_size=8), dict(page_size=24), dict(page_size=256),
             dict(Hkv=0), dict(dh=64), dict(dtype=2), dict(dtype=-1), dict(num_pages=1 << 30), dict(k=None), dict(v=None),
             dict(k_scale=None), dict(v_scale=None), dict(dtype=0), "k+8", "v+8", "k_scale+4", "v_scale+4"]


def bad_cache(p, bad):
    return cache(p, **({bad.split("+")[0]: p + int(bad.split("+")[1])} if isinstance(bad, str) else bad))


@pytest.mark.parametrize("bad", CACHE_BAD, ids=str)
def test_caches_that_are_refused(bad):
    keep, p = mem()
    kv = bad_cache(p, bad)
    lib = dart.lib()
    assert lib.dart_cache_append(C.byref(kv), 1, 2, p, p, 4, p, 256, p, 256, None, p, 1e6, None, None) == INV
    cfg = dart.DartPagedAttnConfig(1, 0, 2, 4, 1e6, 0.1)
    assert lib.dart_paged_attention(C.byref(cfg), C.byref(kv), p, p, p, 512, p, 256, p, 256, None, None, None, p, p, 1 << 40,
                                    None, None) == INV


APPEND = dict(nseq=1, max_pages=2, table="p", lens="p", R=4, k="p", ks=256, v="p", vs=256, rows=None, n="p", theta=1e6, status=None)
APPEND_BAD = [dict(nseq=0), dict(max_pages=0), dict(R=0), dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")),
              dict(table=None), dict(lens=None), dict(k=None), dict(v=None), dict(n=None), dict(ks=255), dict(ks=248), dict(vs=260),
              dict(vs=0), dict(table="p+2"), dict(lens="p+1"), dict(k="p+8"), dict(v="p+2"), dict(rows="p+3"), dict(n="p+2"),
              dict(status="p+2"), dict(max_pages=1 << 28), dict(nseq=1 << 20, R=1 << 12)]


@pytest.mark.parametrize("bad", APPEND_BAD, ids=str)
def test_append_refuses(bad):
    keep, p = mem()
    a = dict(APPEND, **bad)
    ptr = {x: None if a[x] is None else p + int((a[x] + "+0").split("+")[1]) for x in ("table", "lens", "k", "v", "rows", "n", "status")}
    kv = cache(p)
    assert dart.lib().dart_cache_append(C.byref(kv), a["nseq"], a["max_pages"], ptr["table"], ptr["lens"], a["R"], ptr["k"], a["ks"],
                                        ptr["v"], a["vs"], ptr["rows"], ptr["n"], a["theta"], ptr["status"], None) == INV
    assert dart.lib().dart_cache_append(None, 1, 2, p, p, 4, p, 256, p, 256, None, p, 1e6, None, None) == INV


CFG = dict(nseq=1, B=3, max_pages=2, Hq=4, theta=1e6, scale=0.1)
CFG_BAD = [dict(nseq=0), dict(B=-1), dict(B=1025), dict(max_pages=0), dict(Hq=1), dict(Hq=5), dict(Hq=6), dict(Hq=64), dict(theta=1.0),
           dict(theta=float("inf")), dict(scale=0.0), dict(scale=float("nan")), dict(max_pages=1 << 27), dict(nseq=1 << 29)]


@pytest.mark.parametrize("bad", CFG_BAD, ids=str)
def test_attention_configurations_that_are_refused(bad):
    keep, p = mem()
    cfg, kv = dart.DartPagedAttnConfig(*dict(CFG, **bad).values()), cache(p)
    lib = dart.lib()
    assert lib.dart_paged_attention_workspace(C.byref(cfg), C.byref(kv)) == 0
    assert lib.dart_paged_attention(C.byref(cfg), C.byref(kv), p, p, p, 512, p, 256, p, 256, p, p, p, p, p, 1 << 40, None, None) == INV


def test_attention_refuses_pointers_strides_and_small_workspaces():
    keep, p = mem()
    lib = dart.lib()
    kv = cache(p)

    def call(cfg, table=p, lens=p, q=p, qs=512, k=p, ks=256, v=p, vs=256, depths=p, mask=p, n=p, out=p, ws=p, size=1 << 40, status=None):
        return lib.dart_paged_attention(C.byref(cfg), C.byref(kv), table, lens, q, qs, k, ks, v, vs, depths, mask, n, out, ws, size,
                                        status, None)

    cfg = dart.DartPagedAttnConfig(*CFG.values())
    need = lib.dart_paged_attention_workspace(C.byref(cfg), C.byref(kv))
    assert need > 0
    for name in ("table", "lens", "q", "k", "v", "depths", "mask", "n", "out", "ws"):
        assert call(cfg, **{name: None}) == INV, name
        assert call(cfg, **{name: p + 2}) == INV, name
    for name in ("q", "k", "v", "out"):
        assert call(cfg, **{name: p + 8}) == INV, name
    assert call(cfg, mask=p + 4) == INV and call(cfg, ws=p + 128) == INV and call(cfg, status=p + 1) == INV
    assert call(cfg, size=need - 1) == INV
    for name in ("qs", "ks", "vs"):
        assert call(cfg, **{name: 128}) == INV and call(cfg, **{name: 514}) == INV, name
    assert lib.dart_paged_attention(None, C.byref(kv), p, p, p, 512, p, 256, p, 256, p, p, p, p, p, 1 << 40, None, None) == INV


VER = dict(nseq=1, B=3, V=100, dtype=1, ld=100, T=1.0)
VER_BAD = [dict(nseq=0), dict(B=0), dict(B=1025), dict(V=0), dict(V=1 << 24, ld=1 << 24), dict(dtype=2), dict(ld=99), dict(T=-1.0),
           dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-7), dict(nseq=1 << 29)]


@pytest.mark.parametrize("bad", VER_BAD, ids=str)
def test_verification_configurations_that_are_refused(bad):
    keep, p = mem()
    cfg = dart.DartVerifyConfig(*dict(VER, **bad).values())
    assert dart.lib().dart_verify_tree(C.byref(cfg), p, p, p, p, p, p, p, p, p, p, None) == INV


def test_verification_refuses_pointers():
    keep, p = mem()
    cfg = dart.DartVerifyConfig(*VER.values())
    for i in range(10):
        for bad in (None, p + 2):
            a = [p] * 10
            a[i] = bad
            assert dart.lib().dart_verify_tree(C.byref(cfg), *a, None) == INV, (i, bad)
    assert dart.lib().dart_verify_tree(C.byref(cfg), p + 8, *[p] * 9, None) == INV
    assert dart.lib().dart_verify_tree(None, *[p] * 10, None) == INV


def test_binding_refuses_what_a_pointer_hides():
    import torch
    with pytest.raises(ValueError, match="float8"):
        dart.KVCache(torch.zeros(2, 1, 16, 128), torch.zeros(2, 1, 16, 128))
    z = torch.zeros(2, 1, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="scales"):
        dart.KVCache(z, z, torch.zeros(2, 1, 16), torch.zeros(2, 1, 16))
    with pytest.raises(ValueError, match="scales"):
        dart.KVCache(z.to(torch.float8_e4m3fn), z.to(torch.float8_e4m3fn))


def test_binding_refuses_another_device_and_a_status_on_the_host(monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="made on device 0"):
        dart._current(7, 0)
    assert dart._current(7, 1) == (1, 7)
    with pytest.raises(ValueError, match="status"):
        dart._status(torch.zeros(1, dtype=torch.int32), 1)
    assert dart._status(None, 1) is None


# ------------------------------------------------------------ the oracle

def test_oracle_attention_is_the_contiguous_oracle():
    """Row 0 as the last context token: the nodes' rows are those of the
    contiguous layer's oracle."""
    g = np.random.default_rng(1)
    B, C_, Hq, Hkv = 9, 13, 4, 2
    q, kt, vt = (g.standard_normal((1, B + 1, h, 128)) for h in (Hq, Hkv, Hkv))
    kc, vc = g.standard_normal((2, 1, C_, Hkv, 128))
    parents = np.array([[-1, -1, 0, 0, 1, 3, 5, 2, -1]])
    depths = np.array([[1, 1, 2, 2, 2, 3, 4, 3, 1]])
    n = np.array([8])
    out, mag, _ = serve.attention(q, kt, vt, [(kc[0], vc[0])], parents, depths, n, [C_], 1e4, 0.1)
    k2 = np.concatenate([kc, tree_attn.rope(kt[:, :1], C_, 1e4)], 1)
    v2 = np.concatenate([vc, vt[:, :1]], 1)
    old = tree_attn.tree_attention(q[:, 1:], kt[:, 1:], vt[:, 1:], k2, v2, parents, depths, n, C_, 1e4, 0.1)
    np.testing.assert_allclose(out[:, 1:], old, rtol=1e-10, atol=1e-12)
    assert (mag + 1e-12 >= np.abs(out)).all()
    # row 0 is one more decoding step
    x = tree_attn.rope(q[0, 0, 3], C_, 1e4)
    w = np.exp(0.1 * k2[0, :, 1] @ x)
    np.testing.assert_allclose(out[0, 0, 3], w @ v2[0, :, 1] / w.sum(), rtol=1e-10)


def test_oracle_verification_draws_from_the_target():
    """Over a fine grid of u, and the exact law of the noise, the first token
    has the target's probabilities."""
    V, T = 6, 0.7
    z = np.array([0.3, -1.0, 1.2, 0.0, 0.5, -0.2], np.float32)
    p = np.exp(z.astype(np.float64) / T)
    p /= p.sum()
    tokens, parents = np.array([[2, 4]], np.int32), np.array([[-1, -1]], np.int32)
    grid = (np.arange(4000) + 0.5) / 4000
    got = np.zeros(V)
    logits = np.tile(z, (1, 3, 1))
    left = [0, 1, 3, 5]
    for x in grid:
        u = np.full((1, 3), x, np.float32)
        first = [serve.verify(logits, tokens, parents, [2], T, u, np.where(np.arange(V) == j, 1e-6, 1.0)[None])[0][1][0] for j in left[:1]]
        if first[0] in (2, 4):
            got[first[0]] += 1 / len(grid)
        else:  # the noise picks among the rest in proportion to p (exponential races)
            got[left] += p[left] / p[left].sum() / len(grid)
    assert np.abs(got - p).max() < 1e-3
    # each of the rest wins when its noise is the smallest
    for j in left:
        noise = np.where(np.arange(V) == j, 1e-6, 1.0)[None]
        assert serve.verify(logits, tokens, parents, [2], T, np.full((1, 3), 0.9999), noise)[0][1][0] == j
