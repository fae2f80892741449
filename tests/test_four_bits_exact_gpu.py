"""Codes of rotated keys are those of the definition, also where 2^-20 of the
row decides one: the oracle rotates in 64 bits."""
import numpy as np
import pytest
import torch

import four_data as fd
import serve_data as sd
from oracle import four, serve

pytestmark = pytest.mark.gpu
THETA = 1.0e6


@pytest.fixture(scope="module")
def dart():
    from paper_2608_13524_gb300 import dart as d
    return d


def wrong_codes(dart, kv, lens, Hkv, page=32):
    """Elements of keys and of values whose stored value is not the definition's."""
    nseq, R = kv.shape[:2]
    most = -(-(max(lens) + R) // page)
    table = np.random.default_rng(5).permutation(nseq * most).astype(np.int32).reshape(nseq, most)
    shape = (nseq * most, Hkv, page)
    pool = [torch.zeros(shape + (64,), dtype=torch.uint8, device="cuda").view(fd.F4) for _ in range(2)]
    pool += [torch.zeros(shape, device="cuda") for _ in range(2)]
    pool += [torch.zeros(shape + (8,), dtype=torch.uint8, device="cuda").view(sd.E4M3) for _ in range(2)]
    cache = dart.KVCache(*pool)
    dev = kv.to(torch.bfloat16).cuda()
    up = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
    cache.append(dev[:, :, :Hkv], dev[:, :, Hkv:], up(table), up(lens), up([R] * nseq), rope_theta=THETA)
    got = [t.view(torch.uint8).cpu().numpy() if t.dtype != torch.float32 else t.cpu().numpy() for t in pool]
    k, v = (x.double().numpy() for x in (kv[:, :, :Hkv], kv[:, :, Hkv:]))
    wrong = 0
    for (s, pos), (wk, wv) in serve.append(k, v, lens, [R] * nseq, None, THETA).items():
        at, slot = int(table[s][pos // page]), pos % page
        for i, w in enumerate((wk, wv)):
            code, block, scale = four.quantise(w)
            assert np.array_equal(got[2 + i][at, :, slot], scale) and np.array_equal(got[4 + i][at, :, slot], block), (s, pos, i)
            wrong += int((four.values(code, block, scale) != four.values(four.unpack(got[i][at, :, slot]), block, scale)).sum())
    return wrong


@pytest.mark.parametrize("lens,R,Hkv", [([0, 0], 40, 3), ([0, 70000, 999990], 900, 8), ([3] * 5, 2000, 4), ([524280, 0], 1400, 5)], ids=str)
def test_random_rows(dart, lens, R, Hkv):
    """Some 400 in 100000 of these rows have an element that 32 bits leave open."""
    g = np.random.default_rng(len(lens) + R)
    kv = torch.from_numpy(g.standard_normal((len(lens), R, 2 * Hkv, 128)).astype(np.float32)).to(torch.bfloat16).float()
    assert wrong_codes(dart, kv, lens, Hkv) == 0


@pytest.mark.parametrize("first", [0, 1, 5, 100])
def test_rows_made_of_ties(dart, first):
    """Few bits in every element: at position 0 halves between codes are met
    exactly, and near it missed by what the slow frequencies turn."""
    g = np.random.default_rng(first)
    kv = torch.from_numpy(g.integers(-24, 25, (2, 30, 4, 128)).astype(np.float32) / 4)
    kv[..., 0] = 24.0
    assert wrong_codes(dart, kv, [first, first + 1], 2) == 0


def test_powers_of_two_and_small_rows(dart):
    """Largest elements at powers of two, rows of 2^-100 to 2^100, rows of zeros."""
    g = np.random.default_rng(3)
    kv = torch.from_numpy(g.standard_normal((2, 64, 4, 128)).astype(np.float32))
    kv = kv / kv.abs().amax(-1, keepdim=True) * torch.exp2(torch.from_numpy(g.integers(-100, 101, (2, 64, 4, 1))).float())
    kv[:, ::7] = 0.0
    assert wrong_codes(dart, kv.to(torch.bfloat16).float(), [0, 4000], 2) == 0


def test_infinities_at_position_zero(dart):
    """A row of ties with an infinity: its block and its pair's are NaN, the others exact."""
    g = np.random.default_rng(4)
    kv = torch.from_numpy(g.integers(-24, 25, (1, 1, 2, 128)).astype(np.float32) / 4)
    kv[..., 0] = 24.0
    kv[0, 0, 0, 20] = np.inf
    kv[0, 0, 1, 100] = np.nan
    page = 16
    pool = [torch.zeros((1, 1, page, 64), dtype=torch.uint8, device="cuda").view(fd.F4) for _ in range(2)]
    pool += [torch.zeros((1, 1, page), device="cuda") for _ in range(2)]
    pool += [torch.zeros((1, 1, page, 8), dtype=torch.uint8, device="cuda").view(sd.E4M3) for _ in range(2)]
    cache = dart.KVCache(*pool)
    dev = kv.to(torch.bfloat16).cuda()
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    cache.append(dev[:, :, :1], dev[:, :, 1:], 0 * one[None], 0 * one, one, rope_theta=THETA)
    x, y = kv[0, 0].double().numpy().copy()
    x[84] = np.nan  # the pair of element 20
    for i, want in enumerate((x, y)):
        code, block, scale = four.quantise(want)
        assert np.array_equal(pool[4 + i].view(torch.uint8).cpu().numpy()[0, 0, 0], block) and float(pool[2 + i][0, 0, 0]) == scale
        got = four.values(four.unpack(pool[i].view(torch.uint8).cpu().numpy()[0, 0, 0]), block, scale)
        assert np.array_equal(got, four.values(code, block, scale), equal_nan=True)
