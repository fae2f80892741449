"""A round's serving step (attention over the cache, verification, the kept rows
into the cache, lengths advanced) captured once and replayed for other trees,
rows, logits and lengths: what the same calls give eagerly, bit by bit."""
import numpy as np
import pytest
import torch

import serve_data as sd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("B", [3, 40, 130])
def test_a_captured_round_is_replayed(B, fp8):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13524_gb300 import dart
    from test_verify_tree_gpu import data
    nseq, V, page, Hq, Hkv, pages = 2, 3001, 16, 8, 2, 40
    g = np.random.default_rng(7300 + B)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    table = up(g.permutation(nseq * pages).astype(np.int32).reshape(nseq, pages))

    def inputs(seed):
        """One round's: rows of q, k, v; tree and logits."""
        t = sd.bf16(np.random.default_rng(seed), (nseq, B + 1, Hq + 2 * Hkv, 128)).to(torch.bfloat16).cuda()
        _, z, tokens, parents, n, u, noise = data(nseq, B, V, 1.0, True, seed, fill=0.9)
        depths, mask = np.zeros((nseq, B), np.int32), np.zeros((nseq, B, (B + 63) // 64), np.int64)
        for s in range(nseq):
            for i in range(n[s]):
                depths[s, i] = 1 if parents[s, i] < 0 else depths[s, parents[s, i]] + 1
            mask[s] = sd.mask_words(parents[s], n[s], B, np.random.default_rng(seed + s))
        return [t, z] + [up(x) for x in (tokens, parents, n, depths, mask, u, noise)]

    class Server:
        def __init__(self):
            self.cache = dart.KVCache.new(nseq * pages, page, Hkv, dtype=sd.E4M3 if fp8 else torch.bfloat16)
            self.lens = torch.zeros(nseq, dtype=torch.int32, device="cuda")
            self.att = dart.PagedTreeAttention(self.cache, nseq, B, pages, Hq)
            self.ver = dart.TreeVerifier(nseq, B, V, 1.0)
            prompt = sd.bf16(np.random.default_rng(7400), (nseq, 90, 2 * Hkv, 128)).to(torch.bfloat16).cuda()
            n = up(np.array([90, 33], np.int32))
            self.cache.append(prompt[:, :, :Hkv], prompt[:, :, Hkv:], table, self.lens, n)
            self.lens += n

        def round(self, t, z, tokens, parents, n, depths, mask, u, noise):
            q, k, v = t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:]
            self.att(q, k, v, table, self.lens, depths, mask, n)
            kept = self.ver(z, tokens, parents, n, u, noise)
            self.cache.append(k, v, table, self.lens, kept["n_rows"], kept["rows"])
            self.lens += kept["n_rows"]

        def state(self):
            torch.cuda.synchronize()
            pools = [x for x in (self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale) if x is not None]
            return [x.clone() for x in [self.att.out, self.lens, *self.ver.out.values()] + [x.view(torch.uint8) for x in pools]]

    eager, replayed = Server(), Server()
    static = inputs(7500)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        replayed.round(*static)
    kept = []
    for seed in (7501, 7502, 7503, 7504):
        x = inputs(seed)
        eager.round(*x)
        with torch.cuda.stream(stream):
            for dst, src in zip(static, x):
                dst.copy_(src)
            graph.replay()
        a, b = eager.state(), replayed.state()
        assert all(torch.equal(p, q) for p, q in zip(a, b)), seed
        kept.append(a[2].tolist())
    assert max(max(k) for k in kept) > 1, kept  # (some rounds keep a node)
