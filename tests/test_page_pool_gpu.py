"""The pool of pages on the GPU against the plain form: everything equal, in
runs of random calls; and what pages hold after the copies."""
import numpy as np
import pytest
import torch

import canary
import four_data as fd
import serve_data as sd
from oracle import pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dart():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13524_gb300 import dart as d
    d.lib()
    return d


def up(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def same(p, want, garbage):
    """The pool equals the plain form's; entries behind a sequence's pages are not looked at."""
    assert p.refs.tolist() == want.refs
    held = p.held.tolist()
    assert held == [len(r) for r in want.rows]
    table = p.table.cpu().numpy()
    for s, row in enumerate(want.rows):
        assert table[s, :held[s]].tolist() == row, s


def start(dart, num, page, nseq, most):
    p = dart.PagePool(num, page, nseq, most)
    p.table.fill_(10 ** 9)  # (what stands behind a sequence's pages is no page number)
    return p, pages.Pool(num, page, nseq, most)


RUNS = [
    # num_pages, page, nseq, max_pages, calls, tokens of a call
    (1, 16, 1, 1, 12, 20),
    (40, 16, 5, 6, 60, 40),
    (300, 16, 33, 40, 40, 100),
    (4099, 32, 70, 129, 25, 900),
    (9001, 16, 3, 4000, 20, 30000),
    (40000, 16, 300, 257, 12, 3000),
    (33000, 128, 1500, 20, 10, 1000),
    (4096, 16, 60, 120, 25, 900),
    (4000, 32, 16, 400, 25, 5000),
]


@pytest.mark.parametrize("run", RUNS, ids=str)
def test_random_calls(dart, run):
    num, page, nseq, most, n, rows_to = run
    g = np.random.default_rng(num)
    p, want = start(dart, num, page, nseq, most)
    lens, d_lens = [0] * nseq, up([0] * nseq)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for i in range(n):
        op = int(g.choice([0, 1, 1, 2, 3])) if i else 1
        status.zero_()
        if op == 0:
            parents = np.where(g.random(nseq) < 0.6, np.arange(nseq), g.integers(-1, nseq, nseq))
            p.select(up(parents), d_lens, status=status)
            lens = want.select(parents.tolist(), lens)
            assert int(status) == 0
        elif op == 1:
            rows = np.where(g.random(nseq) < 0.3, g.integers(-2, 1, nseq), g.integers(1, rows_to + 1, nseq)).tolist()
            got = p.reserve(d_lens, up(rows), status=status)
            pairs, refused = want.reserve(lens, rows)
            count = int(got[1])
            assert got[0][:count].tolist() == [list(x) for x in pairs]
            assert int(status) == (8 if refused else 0)
            lens = [a + max(b, 0) * (s not in refused) for s, (a, b) in enumerate(zip(lens, rows))]
        elif op == 2:
            lens = [int(g.integers(0, a + 1)) if g.random() < 0.5 else a for a in lens]
            p.trim(up(lens), status=status)
            want.trim(lens)
            assert int(status) == 0
        else:
            got = p.compact(status=status)
            moves = want.compact()
            assert int(got[1]) == len(moves) and got[0][:len(moves)].tolist() == [list(x) for x in moves]
            assert int(status) == 0
        if op != 0:
            d_lens = up(lens)
        assert d_lens.tolist() == lens
        same(p, want, None)


def test_exchange_and_chain(dart):
    """Sequences that take each other's place, and chains: all from the state before."""
    p, want = start(dart, 60, 16, 6, 8)
    rows = [5, 20, 40, 70, 0, 100]
    p.reserve(up([0] * 6), up(rows))
    want.reserve([0] * 6, rows)
    for parents in ([1, 0, 3, 2, 4, 5], [5, 0, 1, 2, 3, 4], [0, 0, 0, 0, 0, 0], [0, -1, -1, 1, -1, 5]):
        lens = up(rows)
        p.select(up(parents), lens)
        rows = want.select(parents, rows)
        assert lens.tolist() == rows
        same(p, want, None)


def test_bad_values_are_reported(dart):
    p, want = start(dart, 30, 16, 3, 5)
    lens = [20, 40, 0]
    p.reserve(up([0] * 3), up(lens))
    want.reserve([0] * 3, lens)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = up(lens)
    p.select(up([-2, 3, 10 ** 9]), d, status=status)  # none of them a parent: all stay
    assert int(status) == 4 and d.tolist() == lens
    same(p, want, None)
    status.zero_()
    p.reserve(up(lens), up([2 ** 31 - 1, 1, 81]), status=status)  # rows that the table does not have
    assert int(status) == 8
    want.reserve(lens, [0, 1, 0])
    same(p, want, None)
    # page numbers outside the pool: counted nowhere, moved nowhere
    for bad in (-1, 30, 2 ** 31 - 1):
        q, _ = start(dart, 30, 16, 3, 5)
        q.reserve(up([0] * 3), up(lens))
        refs = q.refs.clone()
        q.table[1, 1] = bad
        for call in (lambda: q.select(up([0, 1, 1]), up(lens), status=status), lambda: q.reserve(up([20, 20, 0]), up([0, 5, 0]), status=status),
                     lambda: q.trim(up([20, 10, 0]), status=status), lambda: q.compact(status=status)):
            status.zero_()
            q.held.copy_(up([2, 3, 0]))
            call()
            assert int(status) == 4, bad
        assert int(q.refs.min()) >= 0 and int(q.refs.sum()) <= int(refs.sum()) + 3
    # lengths and counts outside their range count as the nearer end
    q, w = start(dart, 30, 16, 2, 5)
    q.reserve(up([0, 0]), up([80, 30]))
    w.reserve([0, 0], [80, 30])
    q.held.copy_(up([10 ** 9, 2]))
    q.trim(up([2 ** 31 - 1, -7]))
    w.trim([80, 0])
    same(q, w, None)


def test_streams_and_graphs(dart):
    """Captured once, replayed for other lengths and parents."""
    p, want = start(dart, 200, 16, 8, 10)
    parents, lens, rows = up(range(8)), up([0] * 8), up([0] * 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.trim(lens)  # (the first call of each is made before the capture)
        p.select(parents, lens)
        p.reserve(lens, rows)
        p.compact()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.trim(lens)
        p.select(parents, lens)
        p.reserve(lens, rows)
        pairs = p.pairs.clone()
        count = p.count.clone()
        p.compact()
    g = np.random.default_rng(3)
    now = [0] * 8
    for _ in range(12):
        par, n = g.integers(-1, 8, 8).tolist(), g.integers(0, 30, 8).tolist()
        parents.copy_(up(par))
        rows.copy_(up(n))
        lens.copy_(up(now))
        graph.replay()
        want.trim(now)
        now = want.select(par, now)
        copies, refused = want.reserve(now, n)
        assert pairs[:int(count)].tolist() == [list(x) for x in copies]
        moves = want.compact()
        assert p.pairs[:int(p.count)].tolist() == [list(x) for x in moves]
        assert lens.tolist() == now
        same(p, want, None)
        now = [a + b * (s not in refused) for s, (a, b) in enumerate(zip(now, n))]
        now = [int(g.integers(0, a + 1)) for a in now]


def test_two_pools_on_two_streams(dart):
    runs = []
    for i in range(2):
        p, want = start(dart, 3000, 16, 64, 40)
        runs.append((p, want, torch.cuda.Stream(), up([0] * 64), up([100 + i] * 64), up([0] * 64 if i else range(64))))
    torch.cuda.synchronize()
    for _ in range(30):
        for p, _, st, lens, rows, parents in runs:
            p.reserve(lens, rows, stream=st)
            p.select(parents, rows, stream=st)
            p.compact(stream=st)
            p.trim(lens, stream=st)
    torch.cuda.synchronize()
    for p, want, *_ in runs:
        same(p, want, None)


# ------------------------------------------------------------ copies

def caches(dart, kind, num, Hkv, page):
    g = np.random.default_rng(num)
    if kind == "bf16":
        shapes = [((num, Hkv, page, 256), torch.bfloat16)] * 2
    elif kind == "e4m3":
        shapes = [((num, Hkv, page, 128), sd.E4M3)] * 2 + [((num, Hkv, page, 4), torch.float32)] * 2
    else:
        shapes = [((num, Hkv, page, 64), fd.F4)] * 2 + [((num, Hkv, page, 4), torch.float32)] * 2 + [((num, Hkv, page, 8), sd.E4M3)] * 2
    raw = [g.integers(0, 256, s, dtype=np.uint8) for s, _ in shapes]
    dev = [fd.guarded(a, t) for a, (_, t) in zip(raw, shapes)]
    dev = [t.view(num, Hkv, page) if t.dtype == torch.float32 else t for t in dev]
    return dart.KVCache(*dev), raw, dev


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("case", [(2, 1, 16, [(0, 1)]), (50, 3, 32, [(7, 1), (7, 2), (49, 0)]), (300, 8, 64, [(i, 299 - i) for i in range(140)]),
                                  (20, 5, 128, [])], ids=lambda c: str(c[:3]))
def test_copies(dart, case, kind):
    num, Hkv, page, pairs = case
    cache, raw, dev = caches(dart, kind, num, Hkv, page)
    d = up(pairs + [(1, 0), (0, 1)])  # (pairs behind the count are not copied)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.copy_pages(d, up([len(pairs)]), status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for a, t in zip(raw, dev):
        for x, y in pairs:
            a[y] = a[x]
        assert np.array_equal(t.contiguous().view(torch.uint8).cpu().numpy().reshape(a.shape), a)


def test_copies_out_of_range(dart):
    cache, raw, dev = caches(dart, "e2m1", 6, 2, 16)
    for pairs, count, done, told in (([(0, 6), (-1, 2), (3, 4)], 3, [(3, 4)], 4), ([(0, 1), (2, 3)], 10 ** 9, [(0, 1), (2, 3)], 0),
                                     ([(0, 1)], -3, [], 0)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        cache.copy_pages(up(pairs), up([count]), status=status)
        assert int(status) == told
        for a, t in zip(raw, dev):
            for x, y in done:
                a[y] = a[x]
            assert np.array_equal(t.contiguous().view(torch.uint8).cpu().numpy().reshape(a.shape), a)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
def test_continuations_of_a_prompt(dart, kind):
    """The calls as they are used: a prompt, continuations of it that share its
    pages, rows of their own, a branch that wins, compaction; every sequence's
    tokens read back are those that were written, bit for bit what a cache
    without sharing gives."""
    dtype = dict(bf16=torch.bfloat16, e4m3=sd.E4M3, e2m1=fd.F4)[kind]
    nseq, page, Hkv, num, most, R = 5, 16, 2, 64, 8, 40
    g = np.random.default_rng(77)
    pool, cache = dart.PagePool(num, page, nseq, most), dart.KVCache.new(num, page, Hkv, dtype=dtype)
    alone, table = dart.KVCache.new(nseq * most, page, Hkv, dtype=dtype), up(np.arange(nseq * most).reshape(nseq, most))
    lens, story = up([0] * nseq), [[] for _ in range(nseq)]  # story: the rows of every sequence
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(rows):
        kv = [sd.bf16(g, (nseq, R, Hkv, 128)).to(torch.bfloat16).cuda() for _ in range(2)]
        n = up(rows)
        cache.copy_pages(*pool.reserve(lens, n, status=status), status=status)
        cache.append(*kv, pool.table, lens, n, status=status)
        for s in range(nseq):
            story[s] = story[s] + [(kv[0][s, i], kv[1][s, i]) for i in range(rows[s])]
        lens.add_(n)
        check()

    def check():
        n = [len(x) for x in story]
        assert lens.tolist() == n and int(status) == 0
        ks, vs = (torch.zeros((nseq, most * page, Hkv, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for s in range(nseq):
            for i, (k, v) in enumerate(story[s]):
                ks[s, i], vs[s, i] = k, v
        alone.append(ks, vs, table, up([0] * nseq), lens)
        got, want = ([torch.zeros_like(ks) for _ in range(2)] for _ in range(2))
        cache.read(*got, pool.table, up([0] * nseq), lens, status=status)
        alone.read(*want, table, up([0] * nseq), lens)
        assert int(status) == 0 and all(torch.equal(a, b) for a, b in zip(got, want))

    def become(parents):
        pool.select(up(parents), lens, status=status)
        old = list(story)
        for s, p in enumerate(parents):
            story[s] = old[p] if p >= 0 else []
        check()

    step([37, 20, 0, 0, 0])
    become([0, 1, 0, 0, 1])
    step([3, 0, 12, 30, 1])
    become([2, 2, 3, -1, 4])
    step([1, 1, 1, 5, 0])
    for s in range(nseq):
        story[s] = story[s][:max(0, len(story[s]) - 9)]
    lens.copy_(up([len(x) for x in story]))
    pool.trim(lens, status=status)
    check()
    cache.copy_pages(*pool.compact(status=status), status=status)
    check()
    used = int((pool.refs > 0).sum())
    assert int(pool.refs[:used].min()) > 0 and not pool.refs[used:].any()
    step([20, 2, 17, 40, 33])
