"""Pages rewritten and attended over again and again, with nothing between the
calls but the stream's order: what was written last is what is read, whichever
kernels start early."""
import numpy as np
import pytest
import torch

import four_data as fd
import serve_data as sd
from test_paged_attn_gpu import dart  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv", [(0, 8, 2), (3, 16, 4), (20, 8, 2), (150, 16, 4)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
def test_what_was_written_last_is_read(dart, kind, B, Hq, Hkv, captured):  # noqa: F811
    nseq, page, R, rounds = 3, 64, 700, 12
    g = torch.Generator(device="cuda").manual_seed(B)
    up = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
    most = -(-R // page)
    cache = dart.KVCache.new(nseq * most, page, Hkv, dtype=dict(bf16=torch.bfloat16, e4m3=sd.E4M3, e2m1=fd.F4)[kind])
    table = up(np.random.default_rng(1).permutation(nseq * most).reshape(nseq, most))
    lens, zero = up([R, R - 61, 130]), up([0] * nseq)
    att = dart.PagedTreeAttention(cache, nseq, B, most, Hq)
    rows = [torch.randn((nseq, B + 1, h, 128), generator=g, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv)]
    tree = (None, None, None)
    if B:
        words = torch.zeros((nseq, B, (B + 63) // 64), dtype=torch.int64, device="cuda")
        for i in range(B):
            words[:, i, i // 64] = 1 << (i % 64) if i % 64 < 63 else -(1 << 63)
        tree = (torch.ones((nseq, B), dtype=torch.int32, device="cuda"), words, up([B] * nseq))
    kv = [torch.randn((rounds, nseq, R, Hkv, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]

    def step(i):
        cache.append(kv[0][i], kv[1][i], table, zero, lens)
        return att(*rows, table, lens, *tree)

    want = []
    for i in range(rounds):
        cache.append(kv[0][i], kv[1][i], table, zero, lens)
        torch.cuda.synchronize()
        want.append(att(*rows, table, lens, *tree).clone())
        torch.cuda.synchronize()
    assert not torch.equal(want[0], want[1])
    if captured:
        got = [torch.empty_like(want[0]) for _ in range(rounds)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for i in range(rounds):
                got[i].copy_(step(i))
        for _ in range(4):
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    else:
        for _ in range(4):
            got = [step(i).clone() for i in range(rounds)]
            assert all(torch.equal(a, b) for a, b in zip(got, want))
