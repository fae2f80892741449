"""e2m1 pages on the GPU, against the fp64 oracle.

Attention.  An element code * block is exact in f16; what is rounded: the output
(bf16), the rotated queries (f16, 2^-11; against tree rows of the streaming
kernel to bf16 once more), tree keys (bf16), in the tiles a key's or value's
scale over the tile's power of two (f16) and its product with the code (f16), and
the probabilities (f16, or bf16 at the streaming kernel's tree rows).  All of it
lies below the roundings that test_paged_attn_gpu.py counts for pages whose
elements may be rounded to bf16 (2^-8) once more, so its bound holds:
  e = a_cache (2^-7 + 2^-11) + a_tree (2^-7 + 2^-11 + 2^-15) + (a_cache + a_tree) 2^-18
  |err| <= 2^-8 |out| + M ((e^2e - 1) + e^2e (2^-7 + 2^-16) + 2^-18)
and the relative 2-norm: output, and at the tree rows three more, of 2^-8 /
sqrt(3) each: 4.6e-3; asked for 5.5e-3.

Cache writes.  Values: every code, block scale and scale as the oracle has them.
Keys: off by half a step of the code (0.25, 0.5 or 1 block scales; 1 at the top
where a block scale was rounded down) or by what a block scale of 0 hides (6 *
2^-10 of the scale), plus the rotation's 2^-20 of the pair."""
import numpy as np
import pytest
import torch

import canary
import four_data as fd
import serve_data as sd
from oracle import four, serve

pytestmark = pytest.mark.gpu

THETA = 1.0e6
SCALE = 128 ** -0.5
RMS = 5.5e-3


@pytest.fixture(scope="module")
def dart():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13524_gb300 import dart as d
    d.lib()
    return d


def up(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


# ------------------------------------------------------------ attention

def run(dart, x, status=None, stream=None):
    att = dart.PagedTreeAttention(dart.KVCache(*x.pool), len(x.lens), x.B, x.max_pages, x.Hq, rope_theta=THETA)
    out = att(*x.dev, x.table, x.d_lens, *x.tree, status=status, stream=stream)
    torch.cuda.synchronize()
    return out


def check(x, got, rows=None, rms=RMS):
    got = got.double().cpu().numpy()
    want, mag, grow = serve.attention(x.q, x.kt, x.vt, x.ctx, x.parents, x.depths, x.n_nodes, x.lens, THETA, SCALE, rows)
    if rows is None:
        for s, n in enumerate(x.n_nodes):
            assert not got[s, n + 1:].any()
        rows = [(s, r) for s in range(len(x.lens)) for r in range(x.B + 1)]
    a_c, a_t = grow[..., 0:1], grow[..., 1:2]
    e = a_c * (2 ** -7 + 2 ** -11) + a_t * (2 ** -7 + 2 ** -11 + 2 ** -15) + (a_c + a_t) * 2 ** -18
    bound = 2 ** -8 * np.abs(want) + mag * (np.expm1(2 * e) + np.exp(2 * e) * (2 ** -7 + 2 ** -16) + 2 ** -18) + 1e-30
    s, r = np.array(rows).T
    d = (got - want)[s, r]
    assert np.isfinite(d).all()
    assert (np.abs(d) <= bound[s, r]).all(), float((np.abs(d) / bound[s, r]).max())
    rel = float(np.linalg.norm(d) / np.linalg.norm(want[s, r]))
    print(f"rel {rel:.2e}, {float((np.abs(d) / bound[s, r]).max()):.2f} of the bound")
    assert rel <= rms


CASES = [
    # name, B, lens, page, Hq, Hkv, further
    ("token-empty-cache", 0, [0], 16, 8, 2, {}),
    ("token-one", 0, [1, 0, 2], 16, 4, 1, {}),
    ("token-chunk-edges", 0, [15, 16, 17, 31, 32, 33, 48, 63, 64, 65], 16, 16, 8, {}),
    ("token-page-edges", 0, [31, 32, 33, 63, 64, 65, 127], 32, 8, 2, {}),
    ("token-page-edges-128", 0, [127, 128, 129, 255, 256, 257], 128, 32, 8, {}),
    ("token-heads-16", 0, [70, 5], 32, 16, 1, {}),
    ("token-heads-1", 0, [70, 300], 64, 3, 3, {}),
    ("token-heads-8", 0, [1000], 64, 16, 2, {}),
    ("token-many-ragged", 0, [int(7 * i * i % 901) for i in range(40)], 32, 8, 2, {}),
    ("token-long", 0, [9001], 16, 4, 1, {}),
    ("token-unfused", 0, [50, 60], 16, 8, 2, dict(fused=False)),
    ("node-1", 1, [40, 0], 16, 8, 2, {}),
    ("rows-16", 3, [64, 100, 47], 16, 8, 2, {}),
    ("rows-17", 16, [200, 33], 32, 4, 4, {}),
    ("no-cache", 40, [0, 0], 16, 8, 2, dict(fill=0.7)),
    ("words-63-64-65", 64, [63, 64, 65], 64, 8, 2, dict(fill=0.98)),
    ("tile-edges", 127, [127, 128, 129, 1], 128, 4, 1, {}),
    ("tile-edges-16", 31, [127, 128, 129, 383], 16, 4, 1, dict(fill=0.9)),
    ("tree-300", 300, [500, 77], 16, 4, 2, dict(fill=0.9)),
    ("heads-16-tree", 20, [300, 0, 11], 32, 16, 1, dict(fill=0.8)),
    ("heads-1-tree", 200, [260], 64, 2, 2, dict(fill=0.8)),
    ("long-tree", 33, [5000], 128, 4, 1, {}),
    ("many-tiles", 40, [3000, 1, 2000], 64, 8, 2, dict(fill=0.9)),
    ("widened-ragged", 200, [700, 0, 129, 900], 32, 8, 2, dict(fill=0.9)),
    ("large", 0, [300], 32, 4, 1, dict(magnitude=2.0 ** 12)),
    ("small-tree", 20, [300], 32, 4, 1, dict(magnitude=2.0 ** -20)),
    ("sharp", 20, [400, 90], 16, 8, 2, dict(q_scale=8.0)),
    ("sharp-token", 0, [400, 90], 16, 8, 2, dict(q_scale=8.0)),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: c[0])
def test_attention(dart, case):
    name, B, lens, page, Hq, Hkv, more = case
    x = fd.attn_data4(len(lens), B, lens, page, Hq, Hkv, 9000 + CASES.index(case), **more)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = run(dart, x, status=status)
    assert int(status) == 0
    # logits of deviation 8, or 2^12 in the one case whose keys are that large: the rounded queries act as strongly
    check(x, out, rms=RMS * 8 if "q_scale" in more else 1.0 if name == "large" else RMS)


def test_large_tree_sampled(dart):
    x = fd.attn_data4(2, 1024, [700, 2000], 64, 8, 2, 9101, fill=0.97)
    g = np.random.default_rng(1)
    rows = [(s, int(r)) for s in range(2) for r in {0, 1, int(x.n_nodes[s]), *g.integers(0, x.n_nodes[s] + 1, 24)}]
    check(x, run(dart, x), rows)


@pytest.mark.parametrize("B", [0, 33, 300])
def test_the_same_bits_every_time(dart, B):
    x = fd.attn_data4(3, B, [1500, 40, 700], 32, 8, 2, 9102 + B)
    first = run(dart, x).clone()
    for _ in range(5):
        assert torch.equal(run(dart, x), first)


@pytest.mark.parametrize("B", [0, 33, 300])
def test_zero_rows_and_block_scales(dart, B):
    """All of the cache 0: every visible key of it has the same weight."""
    x = fd.attn_data4(2, B, [200, 90], 32, 8, 2, 9110 + B)
    for t in x.pool[:2]:
        t.view(torch.uint8).zero_()
    x.ctx = [tuple(0.0 * a for a in c) for c in x.ctx]
    check(x, run(dart, x))


def test_pages_outside_the_pool_are_reported(dart):
    for B in (0, 33, 300):
        x = fd.attn_data4(2, B, [200, 90], 32, 8, 2, 9120 + B)
        good = run(dart, x).clone()
        for bad in (-1, 10 ** 9, x.pool[0].shape[0]):
            t = x.table.clone()
            t[1, 1] = bad
            keep, x.table = x.table, t
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            got = run(dart, x, status=status)
            x.table = keep
            assert int(status) == 4 and torch.equal(got[0], good[0])


# ------------------------------------------------------------ writes and reads

def filled(dart, num, Hkv, page, seed):
    g = np.random.default_rng(seed)
    raw = [g.integers(0, 256, (num, Hkv, page, 64), dtype=np.uint8) for _ in range(2)]
    raw += [g.random((num, Hkv, page), dtype=np.float32) for _ in range(2)] + [g.integers(0, 127, (num, Hkv, page, 8), dtype=np.uint8) for _ in range(2)]
    return raw, dart.KVCache(*[fd.guarded(a, t) for a, t in zip(raw, (fd.F4, fd.F4, torch.float32, torch.float32, sd.E4M3, sd.E4M3))])


def host(cache):
    pool = (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_block, cache.v_block)
    return [t.cpu().numpy() if t.dtype == torch.float32 else t.view(torch.uint8).cpu().numpy() for t in pool]


def setup(dart, nseq, R, lens, n_rows, page, Hkv, seed, path=False, magnitude=1.0):
    g = np.random.default_rng(seed)
    most = max(1, -(-max(int(a) + int(b) for a, b in zip(lens, n_rows)) // page))
    num = nseq * most + 2
    table = g.permutation(num)[:nseq * most].astype(np.int32).reshape(nseq, most)
    raw, cache = filled(dart, num, Hkv, page, seed + 1)
    kv = sd.bf16(g, (nseq, R, 2 * Hkv + 1, 128), magnitude)
    kv *= torch.from_numpy(np.exp2(g.integers(-6, 7, (nseq, R, 2 * Hkv + 1, 8, 1))).astype(np.float32)).expand(-1, -1, -1, -1, 16).flatten(-2)
    kv = kv.to(torch.bfloat16).float()
    dev = kv.to(torch.bfloat16).cuda()
    rows = None
    if path:
        rows = g.integers(0, R, (nseq, R)).astype(np.int32)
        for s in range(nseq):
            rows[s, int(n_rows[s]):] = 10 ** 8
    return raw, cache, table, dev[:, :, :Hkv], dev[:, :, Hkv + 1:], kv[:, :, :Hkv].double().numpy(), kv[:, :, Hkv + 1:].double().numpy(), rows


def check_rows(raw, cache, table, k, v, lens, n_rows, rows, page):
    got, want = host(cache), serve.append(k, v, lens, n_rows, rows, THETA)
    touched = np.zeros((raw[0].shape[0], page), bool)
    wrong = total = 0
    for (s, pos), (wk, wv) in want.items():
        pg, slot = int(table[s][pos // page]), pos % page
        touched[pg, slot] = True
        code, block, scale = four.quantise(wv)
        assert np.array_equal(four.unpack(got[1][pg, :, slot]), code) and np.array_equal(got[5][pg, :, slot], block)
        assert np.array_equal(got[3][pg, :, slot], scale)
        code, block, scale = four.unpack(got[0][pg, :, slot]), got[4][pg, :, slot], got[2][pg, :, slot]
        of = np.repeat(four.E4M3[block], 16, -1) * scale[:, None]
        z = four.E2M1[code & 7]
        half = of * np.where(z > 3, 1.0, np.where(z > 1.5, 0.5, 0.25)) + scale[:, None] * 6 * 2.0 ** -10
        pair = np.hypot(wk[:, :64], wk[:, 64:])
        off = np.abs(four.values(code, block, scale) - wk)
        assert (off <= half * (1 + 2.0 ** -20) + np.concatenate([pair, pair], 1) * 2.0 ** -20).all()
        c, b, sc = four.quantise(wk)
        assert (np.frexp(scale)[0] == 0.5).all() and (np.abs(np.log2(scale / sc)) <= 1).all()
        wrong += int((four.values(c, b, sc) != four.values(code, block, scale)).sum())
        total += code.size
    # a rotated key within 2^-20 of a border of two codes (or of two block scales, which its 16 share): far below one in 1000
    assert wrong <= 2 + total // 1000 + 32 * (total > 0)
    for i, (a, b) in enumerate(zip(raw, got)):
        keep = ~touched
        assert np.array_equal(a.transpose(0, 2, 1, *range(3, a.ndim))[keep], b.transpose(0, 2, 1, *range(3, b.ndim))[keep]), i


WRITES = [
    # lens, n_rows, R, page, Hkv, path
    ([0], [1], 1, 16, 1, False),
    ([0, 5, 30], [40, 0, 7], 40, 16, 2, False),
    ([17, 0], [3, 3], 20, 64, 8, True),
    ([100, 1], [65, 64], 70, 128, 3, False),
    ([0] * 3, [700, 500, 699], 700, 32, 5, False),
    ([0] * 4, [1500, 1499, 1, 1400], 1500, 64, 8, False),
]


@pytest.mark.parametrize("case", WRITES, ids=str)
def test_append(dart, case):
    lens, n_rows, R, page, Hkv, path = case
    raw, cache, table, dk, dv, k, v, rows = setup(dart, len(lens), R, lens, n_rows, page, Hkv, 9200 + WRITES.index(case), path)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.append(dk, dv, up(table), up(lens), up(n_rows), rows=None if rows is None else up(rows), rope_theta=THETA, status=status)
    assert int(status) == 0
    check_rows(raw, cache, table, k, v, lens, n_rows, rows, page)


@pytest.mark.parametrize("magnitude", [2.0 ** -130, 2.0 ** -110, 2.0 ** -60, 2.0 ** 60, 2.0 ** 118])
def test_append_of_any_magnitude(dart, magnitude):
    raw, cache, table, dk, dv, k, v, rows = setup(dart, 2, 30, [3, 0], [30, 30], 16, 4, 9230, magnitude=magnitude)
    cache.append(dk, dv, up(table), up([3, 0]), up([30, 30]), rope_theta=THETA)
    got, want = host(cache), serve.append(k, v, [3, 0], [30, 30], None, THETA)
    for (s, pos), (_, wv) in want.items():
        pg, slot = int(table[s][pos // 16]), pos % 16
        code, block, scale = four.quantise(wv)
        assert np.array_equal(got[3][pg, :, slot], scale) and np.array_equal(got[5][pg, :, slot], block)
        assert np.array_equal(four.values(four.unpack(got[1][pg, :, slot]), got[5][pg, :, slot], scale), four.values(code, block, scale))


def test_ties_of_codes_and_block_scales(dart):
    """bf16 values that lie between two codes, and largest values that lie
    between two block scales: the even one."""
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    rows = np.zeros((1, 127, 1, 128))
    for i in range(127):
        m = (four.E4M3[min(i, 125)] + four.E4M3[min(i, 125) + 1]) / 2 if i % 2 else four.E4M3[i]
        rows[0, i, 0, 0] = 6 * four.E4M3[100]  # (fixes the row's scale: 2^-10 of it and below)
        rows[0, i, 0, 16:32] = 6 * m if 6 * m < 6 * four.E4M3[100] else 0
        b = four.E4M3[40 + i % 60]
        rows[0, i, 0, 32] = 6 * b
        rows[0, i, 0, 33:40] = mid * b
        rows[0, i, 0, 40:47] = -mid * b
    x = torch.from_numpy(rows).to(torch.bfloat16)
    exact = x.double().numpy()
    raw, cache = filled(dart, 8, 1, 16, 9240)
    cache.append(x.cuda(), x.cuda(), up(np.arange(8).reshape(1, 8)), up([0]), up([127]), rope_theta=THETA)
    got = host(cache)
    code, block, scale = four.quantise(exact[0, :, 0])
    at = lambda a: a[:, 0].reshape(128, *a.shape[3:])[:127]  # noqa: E731
    assert np.array_equal(at(got[3]), scale) and np.array_equal(at(got[5]), block) and np.array_equal(four.unpack(at(got[1])), code)


def test_nan_and_infinity(dart):
    g = np.random.default_rng(9250)
    v = sd.bf16(g, (1, 4, 2, 128)).numpy().astype(np.float64)
    v[0, 0, 0, 5], v[0, 1, 1, 127], v[0, 2, 0, 64], v[0, 2, 0, 3] = np.nan, np.inf, -np.inf, np.nan
    v[0, 3, 0] = np.nan
    raw, cache = filled(dart, 1, 2, 16, 9251)
    d = torch.from_numpy(v).to(torch.bfloat16).cuda()
    cache.append(torch.zeros_like(d), d, up([[0]]), up([0]), up([4]), rope_theta=THETA)
    got = host(cache)
    code, block, scale = four.quantise(v[0].transpose(1, 0, 2))
    assert np.array_equal(got[3][0, :, :4], scale) and np.array_equal(got[5][0, :, :4], block)
    have, want = (four.values(four.unpack(got[1][0, :, :4]), got[5][0, :, :4], scale), four.values(code, block, scale))
    assert np.array_equal(np.isnan(have), np.isnan(want)) and np.array_equal(have[~np.isnan(want)], want[~np.isnan(want)])


def pools(dart, kind, num, Hkv, page, seed):
    """A cache of each type with numbers in it, and what they stand for (fp64)."""
    g = np.random.default_rng(seed)
    if kind == "e2m1":
        raw, cache = filled(dart, num, Hkv, page, seed)
        return cache, [four.values(four.unpack(raw[i]), raw[4 + i], raw[2 + i]) for i in range(2)]
    if kind == "bf16":
        x = [sd.bf16(g, (num, Hkv, page, 128)) for _ in range(2)]
        return sd.guarded_cache(dart, [t.to(torch.bfloat16).cuda() for t in x] + [None, None]), [t.double().numpy() for t in x]
    x = [sd.bf16(g, (num, Hkv, page, 128)).to(sd.E4M3) for _ in range(2)]
    s = [torch.from_numpy(g.random((num, Hkv, page), dtype=np.float32)) for _ in range(2)]
    return sd.guarded_cache(dart, [t.cuda() for t in x + s]), [a.double().numpy() * b.double().numpy()[..., None] for a, b in zip(x, s)]


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("case", [([0], [1], 1, 16, 1), ([5, 0, 16], [20, 0, 33], 33, 16, 2), ([100, 3], [300, 299], 310, 64, 8)], ids=str)
def test_read(dart, case, kind, fused):
    """Rows of tokens, rounded once to bf16; rows behind and between as they were."""
    lens, n_rows, R, page, Hkv = case
    nseq, most = len(lens), -(-max(a + b for a, b in zip(lens, n_rows)) // page)
    table = np.random.default_rng(9300).permutation(nseq * most + 1)[:nseq * most].astype(np.int32).reshape(nseq, most)
    cache, vals = pools(dart, kind, nseq * most + 1, Hkv, page, 9301)
    wide = canary.empty((nseq, R, 2 * Hkv + 1, 128), dtype=torch.bfloat16)
    wide.fill_(7.0)
    out = (wide[:, :, :Hkv], wide[:, :, Hkv + 1:]) if fused else tuple(canary.empty((nseq, R, Hkv, 128), dtype=torch.bfloat16).fill_(7.0) for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.read(*out, up(table), up(lens), up(n_rows), status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for i in range(2):
        got = out[i].double().cpu().numpy()
        for s in range(nseq):
            pos = lens[s] + np.arange(n_rows[s])
            # (a product of two fp32 numbers, rounded to fp32 and then to bf16, as torch rounds it)
            exact = vals[i][table[s][pos // page], :, pos % page]
            want = torch.from_numpy(exact).float().to(torch.bfloat16).double().numpy()
            assert np.array_equal(got[s, :n_rows[s]], want) and (got[s, n_rows[s]:] == 7.0).all()
    if fused:
        assert (wide[:, :, Hkv] == 7.0).all()


def test_reads_and_writes_out_of_range_are_reported(dart):
    for kind in ("bf16", "e4m3", "e2m1"):
        cache, vals = pools(dart, kind, 3, 2, 16, 9310)
        out = [canary.empty((2, 40, 2, 128), dtype=torch.bfloat16).fill_(7.0) for _ in range(2)]
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        cache.read(*out, up([[0, 2], [1, 3]]), up([10, 0]), up([40, 20]), status=status)  # past the table; page 3 of 3
        torch.cuda.synchronize()
        assert int(status) == 4
        for i in range(2):
            got = out[i].cpu().float().numpy()
            assert (got[0, 22:] == 7.0).all() and (got[1, 16:] == 7.0).all() and not (got[0, :22] == 7.0).all()
        status.zero_()
        cache.read(*out, up([[0, 2], [1, 9]]), up([-5, 33]), up([-1, 0]), status=status)
        assert int(status) == 0


def test_write_then_read_is_the_oracles_round_trip(dart):
    raw, cache, table, dk, dv, k, v, _ = setup(dart, 3, 200, [0, 40, 7], [200, 150, 199], 32, 4, 9320)
    lens, n_rows = up([0, 40, 7]), up([200, 150, 199])
    cache.append(dk, dv, up(table), lens, n_rows, rope_theta=THETA)
    out = [canary.empty((3, 200, 4, 128), dtype=torch.bfloat16).zero_() for _ in range(2)]
    cache.read(*out, up(table), lens, n_rows)
    want = four.values(*four.quantise(v))
    got = out[1].double().cpu().numpy()
    for s, n in enumerate([200, 150, 199]):
        assert np.array_equal(got[s, :n], torch.from_numpy(want[s, :n]).to(torch.bfloat16).double().numpy())
