"""Writing rows into the paged cache, against the fp64 oracle.

Tolerances.  A rotated key is two products and a sum in fp32 with angles and
their sines to 2^-21: off by at most r = |x| 2^-20, |x| the pair's length.
bf16 slots: r + half a step of bf16 (2^-8 of the value).  e4m3 slots: the scale
is within 2^-20 of max |x| / 448; an element is off by half a step of e4m3
(2^-4 of its value, or half of 2^-9 steps of the scale below the normal range)
plus r, and one more 2^-20 for the quotient.  Values are not rotated: bf16
slots hold them exactly."""
import numpy as np
import pytest
import torch

import serve_data as sd
from oracle import serve

pytestmark = pytest.mark.gpu

THETA = 1.0e6
DH = 128


@pytest.fixture(scope="module")
def dart():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13524_gb300 import dart as d
    d.lib()
    return d


def setup(dart, nseq, R, lens, n_rows, page, fp8, Hkv, seed, path=False, scale=1.0):
    g = np.random.default_rng(seed)
    need = max(int(a) + int(b) for a, b in zip(lens, n_rows))
    max_pages = max(1, -(-need // page))
    num = nseq * max_pages + 2
    table = g.permutation(num)[:nseq * max_pages].astype(np.int32).reshape(nseq, max_pages)
    dt = sd.E4M3 if fp8 else torch.bfloat16
    pool = [torch.from_numpy(g.integers(0, 255, (num, Hkv, page, DH * (1 if fp8 else 2)), dtype=np.uint8)).cuda().view(dt) for _ in range(2)]
    pool += [torch.from_numpy(g.random((num, Hkv, page), dtype=np.float32)).cuda() for _ in range(2)] if fp8 else [None, None]
    cache = sd.guarded_cache(dart, pool)
    kv = sd.bf16(g, (nseq, R, 2 * Hkv + 1, DH), scale)
    dev = kv.to(torch.bfloat16).cuda()
    rows = None
    if path:
        rows = g.integers(0, R, (nseq, R)).astype(np.int32)  # the same row twice, too
        for s in range(nseq):
            rows[s, int(n_rows[s]):] = 10 ** 8
    return cache, pool, table, dev[:, :, :Hkv], dev[:, :, Hkv + 1:], kv[:, :, :Hkv].double().numpy(), kv[:, :, Hkv + 1:].double().numpy(), rows


def up(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def check(cache, pool, table, k, v, lens, n_rows, rows, page, fp8):
    want = serve.append(k, v, lens, n_rows, rows, THETA)
    touched = torch.zeros(pool[0].shape[0], page, dtype=torch.bool)
    got = [x.view(torch.uint8).cpu() if x is not None and x.dtype != torch.float32 else (None if x is None else x.cpu())
           for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    val = [(cache.k, cache.v)[i].cpu().double().numpy() for i in range(2)]
    for (s, pos), (wk, wv) in want.items():
        pg, slot = int(table[s][pos // page]), pos % page
        touched[pg, slot] = True
        pair = np.hypot(wk[:, :64], wk[:, 64:])
        r = np.concatenate([pair, pair], 1) * 2.0 ** -20
        for i, (w, off) in enumerate(((wk, r), (wv, 0.0 * r))):
            have = val[i][pg, :, slot]
            if fp8:
                sc = got[2 + i][pg, :, slot].double().numpy()
                amax = np.abs(w).max(1)
                exact = np.where(amax > 0, np.maximum(amax / 448, 2.0 ** -120), 1.0)
                assert (np.abs(sc / exact - 1) <= 2.0 ** -19).all()
                have = have * sc[:, None]
                step = np.maximum(np.abs(w) * 2.0 ** -4, sc[:, None] * 2.0 ** -10)
                assert (np.abs(have - w) <= step * (1 + 2.0 ** -4) + off + np.abs(w) * 2.0 ** -19).all()
            elif i == 0:
                assert (np.abs(have - w) <= np.abs(w) * 2.0 ** -8 + off * (1 + 2.0 ** -8)).all()
            else:
                assert np.array_equal(have, w)
    torch.cuda.synchronize()
    for i, x in enumerate(got):  # every other slot as it was
        if x is None:
            continue
        old = pool[i].view(torch.uint8).cpu() if i < 2 else pool[i].cpu()
        same = (x == old).all(-1) if i < 2 else x == old
        assert bool((same | touched[:, None, :]).all())


CASES = [
    # lens, n_rows, R, page, e4m3, Hkv, path
    ([0], [1], 1, 16, False, 1, False),
    ([0], [1], 1, 16, True, 1, False),
    ([15, 16, 17, 0], [3, 0, 2, 40], 40, 16, True, 2, False),
    ([15, 16, 17, 0], [3, 0, 2, 40], 40, 32, False, 2, False),
    ([100, 7], [9, 17], 33, 64, True, 8, True),
    ([100, 7], [9, 17], 33, 64, False, 8, True),
    ([1, 127, 128], [300, 1, 129], 300, 128, True, 5, False),
    ([60000], [70], 70, 128, True, 3, False),
    ([0, 5], [1500, 1201], 1500, 64, False, 8, False),
    ([0, 5], [1500, 1201], 1500, 64, True, 8, False),
    ([3], [700], 700, 16, True, 6, True),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_the_oracle(dart, i):
    lens, n_rows, R, page, fp8, Hkv, path = CASES[i]
    nseq = len(lens)
    cache, pool, table, dk, dv, k, v, rows = setup(dart, nseq, R, lens, n_rows, page, fp8, Hkv, 8000 + i, path)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.append(dk, dv, up(table), up(lens), up(n_rows), rows=None if rows is None else up(rows), rope_theta=THETA, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    check(cache, pool, table, k, v, lens, n_rows, rows, page, fp8)


@pytest.mark.parametrize("scale", [0.0, 1e-38, 1e-34, 1e30])
def test_magnitudes(dart, scale):
    cache, pool, table, dk, dv, k, v, _ = setup(dart, 1, 20, [5], [20], 16, True, 2, 8100, scale=scale)
    cache.append(dk, dv, up(table), up([5]), up([20]), rope_theta=THETA)
    torch.cuda.synchronize()
    if scale > 1e-37:
        check(cache, pool, table, k, v, [5], [20], None, 16, True)
    else:  # fp32 products of the smallest floats lose bits: finite and tiny is all that is asked
        at = up(table)[0, (torch.arange(20) + 5).cuda() // 16].long()
        slot = (torch.arange(20) + 5).cuda() % 16
        x = cache.k[at, :, slot].float() * cache.k_scale[at, :, slot][..., None]
        assert bool(torch.isfinite(x).all()) and float(x.abs().max()) < 1e-36


def test_nonfinite_elements_stay_in_their_head(dart):
    cache, pool, table, dk, dv, *_ = setup(dart, 1, 4, [0], [4], 16, True, 3, 8101)
    dv = dv.clone()
    dv[0, 1, 1, 5] = float("nan")
    dv[0, 2, 2, 7] = float("inf")
    cache.append(dk, dv, up(table), up([0]), up([4]), rope_theta=THETA)
    torch.cuda.synchronize()
    pg = int(table[0][0])
    x = cache.v[pg, :, :4].float().cpu() * cache.v_scale[pg, :, :4].cpu()[..., None]
    bad = ~torch.isfinite(x)
    want = torch.zeros_like(bad)
    want[1, 1, 5] = True
    want[2, 2] = True
    assert torch.equal(bad, want)


def test_what_cannot_be_written_is_reported(dart):
    """Positions past the table, pages outside the pool and rows outside the
    input: skipped, status 4, everything else as usual."""
    for what in ("past", "page", "row", "negative"):
        cache, pool, table, dk, dv, k, v, rows = setup(dart, 2, 20, [10, 10], [20, 20], 16, True, 2, 8102, path=True)
        t, r, n = table.copy(), rows.copy(), [20, 20]
        gone = []
        if what == "past":
            t = np.ascontiguousarray(t[:, :1])  # one page: positions 16.. do not exist
            gone = [(s, p) for s in range(2) for p in range(16, 30)]
        elif what == "page":
            t[0, 1] = pool[0].shape[0]
            gone = [(0, p) for p in range(16, 30)]
        else:
            r[1, 3] = 20 if what == "row" else -1
            gone = [(1, 13)]
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        cache.append(dk, dv, up(t), up([10, 10]), up(n), rows=up(r), rope_theta=THETA, status=status)
        torch.cuda.synchronize()
        assert int(status) == 4, what
        r[1, 3] = 0 if what in ("row", "negative") else r[1, 3]
        want = serve.append
        try:
            serve.append = lambda *a: {key: w for key, w in want(*a).items() if key not in gone}
            check(cache, pool, table, k, v, [10, 10], n, r, 16, True)
        finally:
            serve.append = want


def test_lengths_and_counts_are_clamped(dart):
    cache, pool, table, dk, dv, k, v, _ = setup(dart, 2, 8, [0, 0], [8, 0], 16, False, 1, 8103)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.append(dk, dv, up(table), up([-7, 0]), up([100, -2]), rope_theta=THETA, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    check(cache, pool, table, k, v, [0, 0], [8, 0], None, 16, False)


def test_on_another_stream_and_captured(dart):
    cache, pool, table, dk, dv, k, v, _ = setup(dart, 1, 10, [3], [10], 16, True, 2, 8104)
    t, n, at = up(table), up([10]), up([0])
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        cache.append(dk, dv, t, at, n, rope_theta=THETA)
    at.copy_(up([3]))
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    check(cache, pool, table, k, v, [3], [10], None, 16, True)
