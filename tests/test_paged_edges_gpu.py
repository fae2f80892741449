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


@pytest.mark.parametrize("fp8", [False, True])
def test_one_unit_over_all_sms(dart, fp8):  # noqa: F811
    """One kv head and a long context: more than 32 CTAs share a unit of the tiles."""
    x = sd.attn_data(1, 17, [30011], 128, fp8, 4, 1, 7205)
    check(x, run(dart, x), [(0, r) for r in (0, 1, 9, 17)])


@pytest.mark.parametrize("fp8", [False, True])
def test_largest_tree_of_sixteen_heads(dart, fp8):  # noqa: F811
    """129 query tiles of one kv head."""
    x = sd.attn_data(1, 1024, [333], 64, fp8, 16, 1, 7206, fill=0.99)
    n = int(x.n_nodes[0])
    check(x, run(dart, x), [(0, r) for r in (0, 7, 8, 500, n - 1, n)])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("B", [0, 1, 3, 20, 80])
def test_another_base_and_scale(dart, B, fp8, monkeypatch):  # noqa: F811
    """Heads in groups of 8, a rotary base of 1e4 and a softmax scale of 0.05."""
    import test_paged_attn_gpu as base
    x = sd.attn_data(2, B, [77, 260], 32, fp8, 8, 1, 7207)
    att = dart.PagedTreeAttention(dart.KVCache(*x.pool), 2, B, x.max_pages, 8, rope_theta=1.0e4, scale=0.05)
    out = att(*x.dev, x.table, x.d_lens, *x.tree)
    torch.cuda.synchronize()
    monkeypatch.setattr(base, "THETA", 1.0e4)
    monkeypatch.setattr(base, "SCALE", 0.05)
    check(x, out)


def test_verifications_and_writes_at_once(dart):  # noqa: F811
    """Two verifiers, and two writes into one cache, on four streams with nothing
    between them: what each gives alone."""
    from test_cache_append_gpu import setup, up as up32
    from test_verify_tree_gpu import data, up
    calls, outs = [], []
    for seed in (0, 1):
        z, dev, tokens, parents, n, u, noise = data(2, 40, 5000, 1.0, True, 9600 + seed)
        ver = dart.TreeVerifier(2, 40, 5000, 1.0)
        args = [dev, up(tokens), up(parents), up(n), up(u), up(noise)]
        calls.append(lambda st=None, ver=ver, args=args: ver(*args, stream=st))
        outs += list(ver.out.values())
    cache, _, table, dk, dv, *_ = setup(dart, 2, 300, [0, 0], [300, 300], 32, True, 2, 8300)
    for s in (0, 1):
        args = [dk[s:s + 1], dv[s:s + 1], up32(table[s:s + 1]), up32([0]), up32([300])]
        calls.append(lambda st=None, args=args: cache.append(*args, stream=st))
    pools = [cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale]
    pos = torch.arange(300).cuda()
    at = torch.from_numpy(table.astype(np.int64)).cuda()[:, pos // 32]  # [sequence][token]

    def result():
        torch.cuda.synchronize()
        return [t.clone() for t in outs] + [t[at, :, pos % 32] for t in pools]

    for c in calls:
        c()
    alone = result()
    for t in outs + pools:
        t.zero_()
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for c, st in zip(calls, streams):
        c(st)
    assert all(torch.equal(a, b) for a, b in zip(alone, result()))
