"""Tree attention over the paged cache against the fp64 oracle.

Tolerance.  Let w be a row's exact probabilities, M = sum w |v| per element and
a the largest scale * sum |q||k| of its keys.  Rounded to bf16 (at most 2^-8
relative each): the output, the probabilities, tree keys, and the queries
(2^-8 + 2^-11 where they pass through f16 first); a cache key or value in e4m3
may be rounded to bf16 once more.  A logit is then off by
  e = a_cache (2^-7 + 2^-11) + a_tree (2^-7 + 2^-11 + 2^-15) + (a_cache + a_tree) 2^-18
(the last term: fp32 sums, exponentials and angles), which moves normalised
weights by a factor within e^(+-2e), so
  |err| <= 2^-8 |out| + M ((e^2e - 1) + e^2e (2^-7 + 2^-16) + 2^-18).
That is the worst case, in which all roundings conspire; they are independent,
each 2^-8 / sqrt(3) rms at most, and for N(0, 1) data (logits of deviation 1)
four of them act (output, probabilities, query, key): the relative 2-norm of
the error is below sqrt(4) * 2^-8 / sqrt(3) = 4.6e-3, a fifth (e4m3 values
rounded again) makes it 5.1e-3.  Asked for: 5.5e-3.
"""
import numpy as np
import pytest
import torch

import canary
import serve_data as sd
from oracle import serve, tree_attn

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


def run(dart, x, cache=None, status=None, stream=None):
    cache = cache or dart.KVCache(*x.pool)
    att = dart.PagedTreeAttention(cache, len(x.lens), x.B, x.max_pages, x.Hq, rope_theta=THETA)
    out = att(*x.dev, x.table, x.d_lens, *x.tree, status=status, stream=stream)
    torch.cuda.synchronize()
    return out


def check(x, got, rows=None):
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
    assert rel <= RMS


CASES = [
    # name, B, lens, page, e4m3, Hq, Hkv, further
    ("token-empty-cache", 0, [0], 16, False, 8, 2, {}),
    ("token-one", 0, [1, 0, 2], 16, True, 4, 1, {}),
    ("token-chunk-edges", 0, [15, 16, 17, 31, 32, 33], 16, False, 16, 8, {}),
    ("token-page-edges", 0, [127, 128, 129, 255, 256, 257], 128, True, 32, 8, {}),
    ("token-heads-16", 0, [70, 5], 32, False, 16, 1, {}),
    ("token-heads-1", 0, [70, 300], 64, True, 3, 3, {}),
    ("token-heads-2-8", 0, [1000], 64, False, 16, 2, {}),
    ("token-many-ragged", 0, [int(7 * i * i % 901) for i in range(40)], 32, True, 8, 2, {}),
    ("token-long", 0, [9001], 16, True, 4, 1, {}),
    ("token-unfused", 0, [50, 60], 16, False, 8, 2, dict(fused=False)),
    ("node-1", 1, [40, 0], 16, False, 8, 2, {}),
    ("rows-16", 3, [64, 100], 16, True, 8, 2, {}),
    ("rows-17", 16, [200, 33], 32, False, 4, 4, {}),
    ("no-cache", 40, [0, 0], 16, True, 8, 2, dict(fill=0.7)),
    ("words-63-64-65", 64, [63, 64, 65], 64, False, 8, 2, dict(fill=0.98)),
    ("tile-edges", 127, [127, 128, 129, 1], 128, False, 4, 1, {}),
    ("tile-edges-e4m3", 128, [127, 128, 129, 383], 64, True, 4, 1, dict(fill=0.9)),
    ("tree-300", 300, [500, 77], 16, True, 4, 2, dict(fill=0.9)),
    ("heads-16-tree", 20, [300, 0, 11], 32, True, 16, 1, dict(fill=0.8)),
    ("heads-8-tree", 50, [129], 16, False, 16, 2, {}),
    ("heads-1-tree", 200, [260], 64, False, 2, 2, dict(fill=0.8)),
    ("long-tree", 33, [5000], 128, False, 4, 1, {}),
    ("sharp", 20, [400, 90], 16, False, 8, 2, dict(q_scale=8.0)),
    ("sharp-e4m3", 20, [400, 90], 16, True, 8, 2, dict(q_scale=8.0)),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: c[0])
def test_against_the_oracle(dart, case):
    name, B, lens, page, fp8, Hq, Hkv, more = case
    x = sd.attn_data(len(lens), B, lens, page, fp8, Hq, Hkv, 7000 + CASES.index(case), **more)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = run(dart, x, status=status)
    assert int(status) == 0
    if "q_scale" in more:  # logits of deviation 8: the rounded queries and keys act eight times as strongly
        global RMS
        keep, RMS = RMS, RMS * 8
        try:
            check(x, out)
        finally:
            RMS = keep
    else:
        check(x, out)


def test_large_tree_sampled(dart):
    x = sd.attn_data(2, 1024, [700, 2000], 64, True, 8, 2, 7101, fill=0.97)
    g = np.random.default_rng(1)
    rows = [(s, int(r)) for s in range(2) for r in {0, 1, int(x.n_nodes[s]), *g.integers(0, x.n_nodes[s] + 1, 24)}]
    check(x, run(dart, x), rows)


def test_far_positions(dart):
    """A position of 500000 in a table that repeats one page: angles keep their
    precision, offsets stay in range."""
    n, page, Hkv = 500_001, 128, 1
    x = sd.attn_data(1, 2, [page], page, False, 2, Hkv, 7102)
    table = torch.full((1, -(-n // page)), int(x.table[0, 0]), dtype=torch.int32, device="cuda")
    cache = dart.KVCache(*x.pool)
    att = dart.PagedTreeAttention(cache, 1, 2, table.shape[1], 2, rope_theta=THETA)
    out = att(*x.dev, table, torch.tensor([n], dtype=torch.int32, device="cuda"), *x.tree)
    torch.cuda.synchronize()
    kc, vc = x.ctx[0]
    reps = -(-n // page)
    x.ctx = [(np.tile(kc, (reps, 1, 1))[:n], np.tile(vc, (reps, 1, 1))[:n])]
    x.lens = np.array([n], np.int32)
    check(x, out)


def test_agrees_with_the_contiguous_layer(dart):
    """The rows of the nodes equal dart_tree_attention's over a context that
    ends with row 0's rotated key: both within their tolerance of one another."""
    B, C = 60, 200
    x = sd.attn_data(1, B, [C], 16, False, 8, 2, 7103)
    out = run(dart, x)
    k0 = torch.from_numpy(tree_attn.rope(x.kt[0, 0], C, THETA)).float().to(torch.bfloat16).cuda()
    bf = lambda a: torch.from_numpy(a).float().to(torch.bfloat16).cuda()  # noqa: E731
    kc, vc = (bf(a)[None] for a in x.ctx[0])
    kc, vc = torch.cat([kc, k0[None, None]], 1), torch.cat([vc, bf(x.vt[0, 0])[None, None]], 1)
    q, kt, vt = (t[:, 1:].contiguous() for t in x.dev)
    att = dart.TreeAttention(1, B, C + 1, 8, 2, 128, THETA)
    old = att(q, kt, vt, kc.contiguous(), vc.contiguous(), (x.tree[0] + C).int(), x.tree[1], x.tree[2])
    torch.cuda.synchronize()
    d = (out[:, 1:].float() - old).double()
    assert float(d.norm() / old.double().norm()) <= 2 * RMS


def test_every_call_gives_the_same_bits(dart):
    for B, lens in ((0, [4000, 17, 900]), (100, [1500, 0, 300])):
        x = sd.attn_data(3, B, lens, 32, True, 8, 2, 7104)
        assert torch.equal(run(dart, x), run(dart, x))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("B", [0, 3, 20, 130])
def test_powers_of_two_pass_through(dart, B, fp8):
    """Keys times 2^60, queries times 2^-60 and values times 2^50: every rounding
    is relative to a power of two, so the bits are those of the plain call."""
    x = sd.attn_data(2, B, [300, 900], 64, fp8, 8, 2, 7106)
    plain = run(dart, x).clone()
    k, v, ks, vs = x.pool
    x.pool = [k, v, ks * 2.0 ** 60, vs * 2.0 ** 50] if fp8 else [k * 2.0 ** 60, v * 2.0 ** 50, None, None]
    x.dev = tuple((t.float() * 2.0 ** e).to(torch.bfloat16) for t, e in zip(x.dev, (-60, 60, 50)))
    assert torch.equal(run(dart, x).float(), plain.float() * 2.0 ** 50)


@pytest.mark.parametrize("fp8", [False, True])
def test_many_calls_give_the_same_bits(dart, fp8):
    """Hundreds of calls of a shape whose shares switch from cache tiles to tree
    tiles early, where a slot freed too soon would be refilled under its reader."""
    x = sd.attn_data(2, 1024, [700, 2000], 64, fp8, 8, 2, 7101, fill=0.97)
    att = dart.PagedTreeAttention(dart.KVCache(*x.pool), 2, x.B, x.max_pages, 8, rope_theta=THETA)
    first = None
    for _ in range(300):
        out = att(*x.dev, x.table, x.d_lens, *x.tree)
        torch.cuda.synchronize()
        first = out.clone() if first is None else first
        assert torch.equal(out, first)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("B", [2, 5])
def test_more_sequences_than_lanes(dart, B, fp8):
    """Ragged sequences (every seventh empty) beyond a warp's lanes, few rows and tiles."""
    lens = [0 if i % 7 == 3 else 5 + (53 * i) % 300 for i in range(75)]
    x = sd.attn_data(len(lens), B, lens, 16, fp8, 8, 2, 7107, fill=0.8)
    rows = [(s, r) for s in (0, 3, 31, 32, 33, 63, 64, 74) for r in range(int(x.n_nodes[s]) + 1)]
    check(x, run(dart, x), rows)


def test_two_calls_at_once(dart):
    """Two handles over one cache, on two streams with nothing between them: each
    has its own workspace, so each gives what it gives alone."""
    x = sd.attn_data(2, 90, [3000, 1500], 64, True, 8, 2, 7108)
    y = sd.attn_data(2, 0, [3000, 1500], 64, True, 8, 2, 7108)
    cache = dart.KVCache(*x.pool)
    tree = dart.PagedTreeAttention(cache, 2, 90, x.max_pages, 8, rope_theta=THETA)
    token = dart.PagedTreeAttention(cache, 2, 0, x.max_pages, 8, rope_theta=THETA)
    calls = [lambda st=None: tree(*x.dev, x.table, x.d_lens, *x.tree, stream=st),
             lambda st=None: token(*y.dev, x.table, x.d_lens, stream=st)]
    alone = [c().clone() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        got = [c(st) for c, st in zip(calls, streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, got))


def test_split_does_not_show(dart):
    """One sequence alone (its keys shared by all SMs) and among 60 others
    (many sequences to an SM): the same result within two roundings."""
    lens = [700 + 13 * i for i in range(60)]
    x = sd.attn_data(60, 0, lens, 64, False, 8, 2, 7105)
    many = run(dart, x)
    att = dart.PagedTreeAttention(dart.KVCache(*x.pool), 1, 0, x.max_pages, 8, rope_theta=THETA)
    for s in (0, 31, 59):
        one = att(*(t[s:s + 1] for t in x.dev), x.table[s:s + 1].contiguous(), x.d_lens[s:s + 1])
        torch.cuda.synchronize()
        d = (one - many[s:s + 1]).double()
        assert float(d.norm() / one.double().norm()) <= 2 * RMS


@pytest.mark.parametrize("B", [0, 70])
def test_bad_pages_and_lengths(dart, B):
    """A page number outside the pool is reported and not used; a length beyond
    the table counts as its end, a negative one as zero; the other sequences
    are untouched by either."""
    x = sd.attn_data(4, B, [100, 64, 0, 48], 16, True, 8, 2, 7106)
    full = x.table.clone()
    full[1, 4:] = full[1, 0]  # sequence 1: a whole table of pages
    x.table = full
    n = x.max_pages * 16
    kc, vc = x.ctx[1]
    x.ctx[1] = tuple(np.concatenate([a, np.tile(a[:16], (x.max_pages - 4, 1, 1))]) for a in (kc, vc))
    x.lens[1] = n
    x.d_lens = torch.tensor([100, n + 5, -3, 48], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = run(dart, x, status=status)
    assert int(status) == 0
    check(x, good)
    for bad in (-1, 10 ** 9, x.pool[0].shape[0]):
        x.table = full.clone()
        x.table[0, 3] = bad
        status.zero_()
        out = run(dart, x, status=status)
        assert int(status) == 4
        assert torch.equal(out[2:], good[2:])


def test_captured_and_replayed_for_other_lengths(dart):
    """A captured call reads lengths, pages and rows anew on every replay; a
    second graph with its own workspace runs on another stream meanwhile."""
    xs = [sd.attn_data(3, 20, lens, 16, True, 8, 2, 7107 + i) for i, lens in enumerate(([90, 1, 33], [5, 200, 64]))]
    pages = max(x.max_pages for x in xs)
    runs = []
    for x in xs:
        table = torch.full((3, pages), -1, dtype=torch.int32, device="cuda")
        table[:, :x.max_pages] = x.table
        att = dart.PagedTreeAttention(dart.KVCache(*x.pool), 3, 20, pages, 8, rope_theta=THETA)
        stream = torch.cuda.Stream()
        args = [t.clone() for t in x.dev] + [table, x.d_lens.clone()] + [t.clone() for t in x.tree]
        args[0], args[1], args[2] = (torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").copy_(t) for t in x.dev)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            att(*args)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            att(*args)
        runs.append((att, stream, graph, args))
    for _ in range(3):
        for att, stream, graph, _ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for x, (att, _, _, _) in zip(xs, runs):
        check(x, att.out)
    # other lengths and rows in the same buffers
    att, stream, graph, args = runs[0]
    x = sd.attn_data(3, 20, [17, 80, 0], 16, True, 8, 2, 7109, fill=0.6)
    pad = torch.full((3, pages), -1, dtype=torch.int32, device="cuda")
    pad[:, :x.max_pages] = x.table
    with torch.cuda.stream(stream):
        for dst, src in zip(args, list(x.dev) + [pad, x.d_lens] + list(x.tree)):
            dst.copy_(src)
        for dst, src in zip((att.cache.k, att.cache.v, att.cache.k_scale, att.cache.v_scale), x.pool):
            dst[:len(src)].view(torch.uint8).copy_(src.view(torch.uint8))
        graph.replay()
    torch.cuda.synchronize()
    check(x, att.out)


def test_calls_on_an_idle_gpu_give_up_no_wait(dart):
    """Single calls with nothing before them and cold caches: no bounded wait
    runs out (the issuing thread of the tiles may be late by more than a tile)."""
    x = sd.attn_data(1, 16, [20000], 128, False, 8, 2, 7112)
    cold = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first = None
    for i in range(6):
        cold.fill_(i)
        torch.cuda.synchronize()
        out = run(dart, x, status=status)
        assert int(status) == 0
        first = out if first is None else first
        assert torch.equal(out, first)


def test_nothing_else_is_written(dart):
    x = sd.attn_data(2, 30, [100, 3], 16, True, 8, 2, 7110)
    cache = sd.guarded_cache(dart, x.pool)
    before = [t.view(torch.uint8).clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    run(dart, x, cache)
    for b, t in zip(before, (cache.k, cache.v, cache.k_scale, cache.v_scale)):
        assert torch.equal(b, t.view(torch.uint8))
    canary.check()


def test_tolerance_detects_a_planted_mask_error(dart, monkeypatch):
    """An oracle that forgets each row's parent is far outside the tolerance."""
    x = sd.attn_data(1, 40, [20], 16, False, 4, 1, 7111)
    out = run(dart, x)
    check(x, out)
    honest = serve.root_path
    monkeypatch.setattr(serve, "root_path", lambda p, i: [j for j in honest(p, i) if j != int(p[i])])
    with pytest.raises(AssertionError):
        check(x, out)
