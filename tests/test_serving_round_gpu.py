"""The operators as a server runs them: prompts into the cache, a tree from
dart.Dart, its rows through the paged attention, the branch that the target
keeps, that branch into the cache, and the next pass over what is there now."""
import numpy as np
import pytest
import torch

import serve_data as sd
from oracle import serve

pytestmark = pytest.mark.gpu

THETA = 1.0e6


@pytest.mark.parametrize("fp8", [False, True])
def test_two_rounds(fp8):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13524_gb300 import dart
    from parity import to_device
    from workloads import Config, make_inputs
    cfg = Config("serve", 2, 2003, 256, 5, 6, 6, 20, "bf16", 1.0, 77)
    x = make_inputs(cfg)
    dx = to_device(cfg, x)
    eng = dart.Dart(cfg, dx["Wi"], dx["Wo"], dx["E"])
    g = np.random.default_rng(78)
    nseq, B, R, Hq, Hkv, page = 2, cfg.B, cfg.B + 1, 8, 2, 16
    cache = dart.KVCache.new(24, page, Hkv, dtype=sd.E4M3 if fp8 else torch.bfloat16)
    table = torch.from_numpy(g.permutation(24)[:16].astype(np.int32).reshape(nseq, 8)).cuda()
    lens = torch.zeros(nseq, dtype=torch.int32, device="cuda")

    def rows_of(length):
        t = sd.bf16(g, (nseq, length, Hq + 2 * Hkv, 128)).to(torch.bfloat16).cuda()
        return t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:]

    def read(s):
        """What the cache holds of sequence s, as the attention has to see it."""
        n = int(lens[s])
        pos = torch.arange(n, device="cuda")
        at, slot = table[s, pos // page].long(), pos % page
        got = []
        for v, sc in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
            y = v.view(torch.uint8)[at, :, slot].view(v.dtype).double() if fp8 else v[at, :, slot].double()
            got.append((y * sc[at, :, slot][..., None].double() if fp8 else y).cpu().numpy())
        return tuple(got)

    prompt = np.array([37, 5], np.int32)
    _, k, v = rows_of(37)
    cache.append(k, v, table, lens, torch.from_numpy(prompt).cuda(), rope_theta=THETA)
    lens += torch.from_numpy(prompt).cuda()
    att = dart.PagedTreeAttention(cache, nseq, B, 8, Hq, rope_theta=THETA)
    ver = dart.TreeVerifier(nseq, B, cfg.V, 1.0)
    for rnd in range(2):
        tree = eng.build_tree(dx["Dlog"], dx["h0"])
        q, k, v = rows_of(R)
        out = att(q, k, v, table, lens, tree["depths"], tree["mask"], tree["n_nodes"])
        torch.cuda.synchronize()
        parents = tree["parents"].cpu().numpy()
        want, _, _ = serve.attention(*(t.double().cpu().numpy() for t in (q, k, v)), [read(s) for s in range(nseq)], parents,
                                     tree["depths"].cpu().numpy(), tree["n_nodes"].cpu().numpy(), lens.cpu().numpy(), THETA, 128 ** -0.5)
        d = out.double().cpu().numpy() - want
        assert np.linalg.norm(d) <= 5.5e-3 * np.linalg.norm(want)  # (see test_paged_attn_gpu.py)
        z = torch.from_numpy(g.standard_normal((nseq, R, cfg.V)).astype(np.float32)).cuda()
        tok = tree["tokens"].long()
        for s in range(nseq):  # the target agrees with the first child of every node
            for i in reversed(range(int(tree["n_nodes"][s]))):
                z[s, parents[s, i] + 1, tok[s, i]] = 12.0
        u = torch.rand((nseq, R), device="cuda")
        noise = torch.empty((nseq, cfg.V), device="cuda").exponential_()
        got = ver(z, tree["tokens"], tree["parents"], tree["n_nodes"], u=u, noise=noise)
        torch.cuda.synchronize()
        exp = serve.verify(z.cpu().numpy(), tree["tokens"].cpu().numpy(), parents, tree["n_nodes"].cpu().numpy(), 1.0,
                           u.cpu().numpy(), noise.cpu().numpy())
        for s in range(nseq):
            n = int(got["n_rows"][s])
            assert got["rows"][s, :n].tolist() == exp[s][0] and got["tokens"][s, :n].tolist() == exp[s][1]
        before = lens.clone()
        cache.append(k, v, table, lens, got["n_rows"], rows=got["rows"], rope_theta=THETA)
        lens += got["n_rows"]
        torch.cuda.synchronize()
        new = serve.append(k.double().cpu().numpy(), v.double().cpu().numpy(), before.cpu().numpy(), got["n_rows"].cpu().numpy(),
                           got["rows"].cpu().numpy(), THETA)
        for s in range(nseq):
            have = read(s)
            for pos in range(int(before[s]), int(lens[s])):
                for a, b in zip((have[0][pos], have[1][pos]), new[s, pos]):
                    top = np.abs(b).max(-1, keepdims=True)
                    assert (np.abs(a - b) <= np.maximum(np.abs(b) * 2.0 ** -4, top * 2.0 ** -18) * 1.07 + 1e-6).all()
    eng.close()
