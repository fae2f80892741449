"""Paged tree attention at the edges of its contract, against the fp64 oracle:
zero queries and keys, products below the floats, mask bits of later rows.
Tolerances: see test_paged_attn_gpu.py."""
import numpy as np
import pytest
import torch

import serve_data as sd
from test_paged_attn_gpu import check, dart, run  # noqa: F401

pytestmark = pytest.mark.gpu


def scaled(x, q=1.0, k=1.0):
    """The rows' queries and keys times powers of two (or zero), in the data and on the device."""
    rows = [(s, r) for s in range(len(x.lens)) for r in range(int(x.n_nodes[s]) + 1)]
    for s, r in rows:
        x.q[s, r] *= q
        x.kt[s, r] *= k
    x.dev = (bf16_of(x.q), bf16_of(x.kt), x.dev[2])


def bf16_of(a):
    return torch.from_numpy(np.ascontiguousarray(a)).float().to(torch.bfloat16).cuda()


# (B, Hq, Hkv): rows streamed, one and two query tiles, tiles of e4m3 pages laid out as f16 first
SHAPES = [(3, 8, 2), (20, 8, 2), (60, 8, 2), (130, 8, 2), (300, 4, 2)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("lens", [[0, 0], [128, 256], [0, 37], [384, 5]], ids=str)
def test_zero_queries_and_keys(dart, lens, shape, fp8):  # noqa: F811
    """Every visible key has the same weight: a first pass with zeroed tensors."""
    B, Hq, Hkv = shape
    x = sd.attn_data(2, B, lens, 16, fp8, Hq, Hkv, 7200, fill=0.9)
    scaled(x, 0.0, 0.0)
    check(x, run(dart, x))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_some_zero_rows(dart, shape, fp8):  # noqa: F811
    """Zero queries among others, and zero keys among others."""
    B, Hq, Hkv = shape
    x = sd.attn_data(2, B, [128, 0], 16, fp8, Hq, Hkv, 7201)
    x.q[:, ::3] = 0.0
    x.kt[:, 1::2] = 0.0
    scaled(x)
    check(x, run(dart, x))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("q,k", [(2.0 ** -80, 2.0 ** -80), (2.0 ** -100, 2.0 ** -30), (2.0 ** -40, 2.0 ** -110)], ids=str)
def test_products_below_the_floats(dart, q, k, shape, fp8):  # noqa: F811
    B, Hq, Hkv = shape
    x = sd.attn_data(2, B, [0, 256], 32, fp8, Hq, Hkv, 7202)
    scaled(x, q, k)
    check(x, run(dart, x))


@pytest.mark.parametrize("fp8", [False, True])
def test_a_new_pool_without_scales(dart, fp8):  # noqa: F811
    """A pool straight from KVCache.new (e4m3: scales of zero) read as it is:
    zero keys and zero values."""
    for B in (0, 3, 20, 130):
        x = sd.attn_data(2, B, [130, 256], 16, fp8, 8, 2, 7203)
        cache = dart.KVCache.new(x.pool[0].shape[0], 16, 2, dtype=x.pool[0].dtype)
        x.ctx = [(np.zeros_like(k), np.zeros_like(v)) for k, v in x.ctx]
        scaled(x, 0.0, 0.0)
        check(x, run(dart, x, cache))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_mask_bits_of_later_rows_are_not_used(dart, shape, fp8):  # noqa: F811
    """Ancestors come before their descendants; bits beyond a row's own are
    garbage in every kernel, in the same 128 keys as the row's own or not."""
    B, Hq, Hkv = shape
    x = sd.attn_data(2, B, [100, 0], 16, fp8, Hq, Hkv, 7204, fill=0.9)
    plain = run(dart, x).clone()
    depths, mask, n = x.tree
    words = mask.cpu().numpy().view(np.uint64).copy()
    bits = np.unpackbits(words.view(np.uint8).reshape(2, B, -1), axis=-1, bitorder="little")
    for i in range(B):
        bits[:, i, i + 1:] = 1
    later = np.packbits(bits, axis=-1, bitorder="little").view(np.int64)
    x.tree = (depths, torch.from_numpy(np.ascontiguousarray(later.reshape(mask.shape))).cuda(), n)
    assert torch.equal(run(dart, x), plain)
    check(x, plain)
