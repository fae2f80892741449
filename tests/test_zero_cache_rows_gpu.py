"""Rows of zeros in a cache of codes, whose scale is 1 as dart_cache_append
leaves it, beside keys or values far below 1: such a row has no part in what the
others are measured by.  Tolerances: see test_paged_attn_gpu.py and
test_four_bits_gpu.py; all of them are relative to the values."""
import numpy as np
import pytest
import torch

import four_data as fd
import serve_data as sd
import test_four_bits_gpu as four_test
import test_paged_attn_gpu as paged_test
from test_paged_attn_gpu import dart  # noqa: F401

pytestmark = pytest.mark.gpu

# (B, Hq, Hkv): one and two groups of 8 rows streamed, tiles converted in the CTA, tiles laid out as f16 first
SHAPES = [(0, 8, 2), (3, 16, 4), (20, 8, 2), (300, 4, 2)]
# which of a sequence's tokens are zero
PLACES = {"some": lambda p, n: p % 5 == 2, "first": lambda p, n: p < 140, "last": lambda p, n: p == n - 1, "one": lambda p, n: p == n // 2}


def data(kind, shape, lens, page, seed, which, magnitude, place):
    """Keys (which = 0) or values (1) of the cache and the tree times `magnitude`
    (queries by as much less), some rows of the cache zero."""
    B, Hq, Hkv = shape
    x = (fd.attn_data4 if kind == "e2m1" else lambda *a: sd.attn_data(*a[:4], True, *a[4:]))(len(lens), B, lens, page, Hq, Hkv, seed)
    x.pool[2 + which].mul_(magnitude)
    parts = [p * magnitude if i == 1 + which else p / magnitude if i == 0 and which == 0 else p for i, p in enumerate(x.dev)]
    x.dev = tuple(p.contiguous() for p in parts)
    if which == 0:
        x.q, x.kt = x.q / magnitude, x.kt * magnitude
    else:
        x.vt = x.vt * magnitude
    table = x.table.cpu().numpy()
    x.ctx = [tuple(a * magnitude if i == which else a for i, a in enumerate(c)) for c in x.ctx]
    for s, n in enumerate(lens):
        p = np.flatnonzero(PLACES[place](np.arange(n), n))
        x.ctx[s][which][p] = 0.0
        at, slot = torch.from_numpy(table[s][p // page].astype(np.int64)).cuda(), torch.from_numpy(p % page).cuda()
        x.pool[which].view(torch.uint8)[at, :, slot] = 0
        x.pool[2 + which][at, :, slot] = 1.0
        if kind == "e2m1":
            x.pool[4 + which].view(torch.uint8)[at, :, slot] = 0
    return x


@pytest.mark.parametrize("place", sorted(PLACES))
@pytest.mark.parametrize("magnitude", [2.0 ** -13, 2.0 ** -40])
@pytest.mark.parametrize("which", [0, 1], ids=["keys", "values"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_rows_of_zeros_among_small_ones(dart, kind, shape, which, magnitude, place):  # noqa: F811
    lens = [700, 129]
    x = data(kind, shape, lens, 32, 9700, which, magnitude, place)
    t = four_test if kind == "e2m1" else paged_test
    t.check(x, t.run(dart, x))


@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_a_cache_of_zeros_alone(dart, kind, shape):  # noqa: F811
    PLACES["all"] = lambda p, n: p >= 0
    try:
        x = data(kind, shape, [300, 128], 32, 9701, 1, 2.0 ** -20, "all")
    finally:
        del PLACES["all"]
    t = four_test if kind == "e2m1" else paged_test
    t.check(x, t.run(dart, x))


@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_zeros_that_the_cache_writes_itself(dart, kind):  # noqa: F811
    """Values of 2^-16 with zero rows among them, written by append: the output is
    that of a cache in which the zero rows have the scale of their neighbours."""
    dtype = dict(e4m3=sd.E4M3, e2m1=fd.F4)[kind]
    g, n, page, Hkv = torch.Generator(device="cuda").manual_seed(3), 200, 16, 2
    k, v = (torch.randn((1, n, Hkv, 128), generator=g, device="cuda") for _ in range(2))
    v *= 2.0 ** -16
    v[:, ::3] = 0.0
    k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    up = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    most = -(-n // page)
    table, lens = up([list(range(most))]), up([n])
    q, kt, vt = (torch.randn((1, 1, h, 128), generator=g, device="cuda").to(torch.bfloat16) for h in (8, Hkv, Hkv))
    vt = (vt.float() * 2.0 ** -16).to(torch.bfloat16)
    got = []
    for small in (False, True):
        cache = dart.KVCache.new(most, page, Hkv, dtype=dtype)
        cache.append(k, v, table, up([0]), up([n]))
        p = torch.arange(0, n, 3, device="cuda")
        assert (cache.v_scale[p // page, :, p % page] == 1.0).all()
        if small:
            cache.v_scale[p // page, :, p % page] = 2.0 ** -27
        got.append(dart.PagedTreeAttention(cache, 1, 0, most, 8)(q, kt, vt, table, lens).double())
    # (both are within half a step of bf16 and a few f16 roundings of one another)
    assert float((got[0] - got[1]).norm() / got[1].norm()) <= 2.0 ** -8
