"""What a reservation grants: rows that append takes as they are, so that a
sequence without room is written nowhere and no other sequence's pages change."""
import numpy as np
import pytest
import torch

import four_data as fd
import serve_data as sd
from oracle import pages
from test_page_pool_gpu import dart, start, up  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = dict(bf16=torch.bfloat16, e4m3=sd.E4M3, e2m1=fd.F4)


@pytest.mark.parametrize("run", [(40, 16, 5, 6, 60, 40), (300, 16, 33, 40, 40, 100), (9001, 16, 3, 4000, 20, 30000), (40000, 16, 300, 257, 12, 3000),
                                 (33000, 128, 2500, 20, 10, 1000)], ids=str)
def test_granted_rows_are_the_plain_forms(dart, run):  # noqa: F811
    num, page, nseq, most, n, rows_to = run
    g = np.random.default_rng(num)
    p, want = start(dart, num, page, nseq, most)
    lens = [0] * nseq
    some = 0
    for i in range(n):
        rows = np.where(g.random(nseq) < 0.3, g.integers(-2, 1, nseq), g.integers(1, rows_to + 1, nseq)).tolist()
        d = up(rows)
        p.reserve(up(lens), d)
        _, refused = want.reserve(lens, rows)
        granted = [max(r, 0) * (s not in refused) for s, r in enumerate(rows)]
        assert p.granted.tolist() == granted and d.tolist() == rows
        some += bool(refused)
        lens = [a + b for a, b in zip(lens, granted)]
        if i % 3 == 2:
            parents = np.where(g.random(nseq) < 0.6, np.arange(nseq), g.integers(-1, nseq, nseq)).tolist()
            p.select(up(parents), up(lens))
            lens = want.select(parents, lens)
    assert some > 0


def test_granted_may_be_the_rows_asked_for(dart):  # noqa: F811
    p, _ = start(dart, 4, 16, 3, 4)
    p.granted.copy_(up([40, 16, 16]))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    p.reserve(up([0, 0, 0]), p.granted, status=status)
    assert p.granted.tolist() == [40, 16, 0] and int(status) == 8


def bytes_of(cache):
    pool = (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_block, cache.v_block)
    return [t.view(torch.uint8).clone() for t in pool if t is not None]


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("kind", sorted(TYPES))
def test_a_full_pool_is_written_nowhere_else(dart, kind, captured):  # noqa: F811
    """Sequences that get no room (no free page for a new page or for a copy of a
    shared one, no place in the table's row): their tokens go nowhere, lengths
    stay, and all bytes of the cache but those of granted rows are as before."""
    page, Hkv, R, nseq, most = 16, 2, 64, 5, 4
    cache, pool = dart.KVCache.new(6, page, Hkv, dtype=TYPES[kind]), dart.PagePool(6, page, nseq, most)
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn((nseq, R, Hkv, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    lens, rows = up([0] * nseq), up([0] * nseq)

    def step():
        cache.copy_pages(*pool.reserve(lens, rows))
        cache.append(k, v, pool.table, lens, pool.granted)
        lens.add_(pool.granted)

    step()  # (the first call of each is made before the capture)
    torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        lens.zero_()
    do = graph.replay if captured else step

    # 64 tokens take four pages, 16 more one; then 20 find one page of two and get none
    rows.copy_(up([64, 16, 20, 0, 0]))
    do()
    assert pool.granted.tolist() == [64, 16, 0, 0, 0] and lens.tolist() == [64, 16, 0, 0, 0]
    # sequence 3 goes on where 0 is, 4 where 1 is; both share, and one page is free
    pool.select(up([0, 1, 2, 0, 1]), lens)
    before = bytes_of(cache)
    rows.copy_(up([1, 0, 16, 5, 20]))  # 0 and 3: the row is full; 2: the last free page; 4: none left
    do()
    assert pool.granted.tolist() == [0, 0, 16, 0, 0] and lens.tolist() == [64, 16, 16, 64, 16]
    new = int(pool.table[2, 0])
    for a, b in zip(before, bytes_of(cache)):
        same = (a == b).flatten(1).all(1)
        assert not bool(same[new]) and bool(same[torch.arange(6, device="cuda") != new].all())
    # a page that two share, with room in it, and no page for the copy
    lens.copy_(up([64, 10, 16, 64, 10]))
    before = bytes_of(cache)
    rows.copy_(up([0, 3, 0, 0, 3]))
    do()
    assert pool.granted.tolist() == [0] * 5 and lens.tolist() == [64, 10, 16, 64, 10]
    assert all(torch.equal(a, b) for a, b in zip(before, bytes_of(cache)))
    # one of the sharers ends: its page is the other's alone
    pool.select(up([0, 1, 2, 3, -1]), lens)
    do()
    assert pool.granted.tolist() == [0, 3, 0, 0, 0] and lens.tolist() == [64, 13, 16, 64, 0]
