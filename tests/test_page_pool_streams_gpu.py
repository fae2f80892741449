"""Two pools at work on two streams: each ends as the plain form does."""
import numpy as np
import pytest
import torch

from test_page_pool_gpu import dart, same, start, up  # noqa: F401

pytestmark = pytest.mark.gpu


def test_two_pools_side_by_side(dart):  # noqa: F811
    g = np.random.default_rng(41)
    runs = []
    for num, nseq, most in ((3000, 64, 40), (5000, 90, 60)):
        p, want = start(dart, num, 16, nseq, most)
        steps, lens = [], [0] * nseq
        for i in range(12):
            rows = g.integers(0, 60, nseq).tolist()
            parents = np.where(g.random(nseq) < 0.7, np.arange(nseq), g.integers(-1, nseq, nseq)).tolist()
            pairs, refused = want.reserve(lens, rows)
            granted = [r * (s not in refused) for s, r in enumerate(rows)]
            after = [a + b for a, b in zip(lens, granted)]
            chosen = want.select(parents, after)
            cut = [int(g.integers(0, n + 1)) if g.random() < 0.4 else n for n in chosen]
            want.trim(cut)
            moves = want.compact() if i % 4 == 3 else None
            steps.append([up(lens), up(rows), up(parents), up(after), up(cut), pairs, granted, chosen, moves])
            lens = cut
        runs.append((p, want, torch.cuda.Stream(), steps))
    torch.cuda.synchronize()
    kept = [[], []]
    for i in range(12):  # (nothing waits for the host between them)
        for j, (p, _, st, steps) in enumerate(runs):
            lens, rows, parents, after, cut, *_ = steps[i]
            with torch.cuda.stream(st):
                p.reserve(lens, rows)
                got = [p.pairs.clone(), p.count.clone(), p.granted.clone()]
                p.select(parents, after)
                p.trim(cut)
                if i % 4 == 3:
                    p.compact()
                    got += [p.pairs.clone(), p.count.clone()]
                kept[j].append(got)
    torch.cuda.synchronize()
    for (p, want, _, steps), seen in zip(runs, kept):
        for (_, _, _, after, _, pairs, granted, chosen, moves), got in zip(steps, seen):
            assert got[0][:int(got[1])].tolist() == [list(x) for x in pairs] and got[2].tolist() == granted
            assert after.tolist() == chosen
            if moves is not None:
                assert got[3][:int(got[4])].tolist() == [list(x) for x in moves]
        same(p, want, None)
        assert sum(want.refs) > 0 and max(want.refs) > 1
