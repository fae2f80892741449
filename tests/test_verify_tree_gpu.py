"""Verification of the tree against the fp64 oracle.

Rows and tokens have to be equal: the inputs keep u and the noise away from
the borders (the oracle is asked for the gap).  log p is a difference of two
fp32 numbers below 2^7, each with a relative error of 2^-22 and a sum of
exponentials off by at most 2^-19 of itself: within 2^-14."""
import math

import numpy as np
import pytest
import torch

from oracle import serve

pytestmark = pytest.mark.gpu

LOGP = 2.0 ** -14


@pytest.fixture(scope="module")
def dart():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_13524_gb300 import dart as d
    d.lib()
    return d


def up(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def data(nseq, B, V, T, bf16, seed, fill=1.0, follow=0.8, ld=None):
    """Trees of random shape; most rows' mass lies on one of their children."""
    g = np.random.default_rng(seed)
    parents = np.full((nseq, B), -2, np.int32)
    n_nodes = np.array([max(0, int(round(fill * B)) - (s if fill < 1 else 0)) for s in range(nseq)], np.int32)
    tokens = np.stack([g.permutation(V)[:B] if V >= B else g.integers(0, V, B) for _ in range(nseq)]).astype(np.int32)
    z = g.standard_normal((nseq, B + 1, V)).astype(np.float32) * 2
    for s in range(nseq):
        for i in range(n_nodes[s]):
            parents[s, i] = int(g.integers(max(-1, i - 6), i)) if i else -1
        for r in range(B + 1):
            kids = [i for i in range(n_nodes[s]) if parents[s, i] + 1 == r]
            if kids and g.random() < 0.9:
                z[s, r, tokens[s, kids[int(g.integers(len(kids)))]]] = math.log(V) + 2 + math.log(follow / (1 - follow))
    z *= T or 1.0
    zt = torch.from_numpy(z).to(torch.bfloat16 if bf16 else torch.float32)
    u = g.random((nseq, B + 1), dtype=np.float32)
    noise = np.maximum(g.exponential(size=(nseq, V)), 1e-12).astype(np.float32)
    dev = zt.cuda()
    if ld:
        wide = torch.full((nseq, B + 1, ld), 1e30, dtype=zt.dtype, device="cuda")
        wide[..., :V] = dev
        dev = wide[..., :V]
    return zt.float().numpy(), dev, tokens, parents, n_nodes, u, noise


def check(out, want, R):
    n = out["n_rows"].cpu().numpy()
    for s, (rows, toks, logp) in enumerate(want):
        assert n[s] == len(rows)
        pad = R - len(rows)
        assert out["rows"][s].tolist() == rows + [-1] * pad
        assert out["tokens"][s].tolist() == toks + [-1] * pad
        got = out["logp"][s].double().cpu().numpy()
        assert np.abs(got[:len(rows)] - logp).max() <= LOGP, np.abs(got[:len(rows)] - logp).max()
        assert not got[len(rows):].any()


def run(dart, z, tokens, parents, n_nodes, T, u, noise, **kw):
    nseq, R, V = z.shape
    ver = dart.TreeVerifier(nseq, R - 1, V, T)
    return ver(z, up(tokens), up(parents), up(n_nodes), u=up(u) if T else None, noise=up(noise) if T else None, **kw)


CASES = [
    # nseq, B, V, T, bf16, fill, ld
    (1, 1, 1, 1.0, False, 1.0, None),
    (1, 1, 2, 0.0, True, 1.0, None),
    (2, 5, 7, 1.0, True, 1.0, None),
    (3, 16, 1000, 0.7, False, 0.8, None),
    (3, 16, 1001, 0.7, True, 0.8, None),
    (2, 40, 999, 0.0, True, 1.0, 1013),
    (2, 40, 999, 1.3, False, 1.0, 1001),
    (1, 64, 4097, 0.0, False, 1.0, None),
    (9, 33, 5003, 1.0, True, 0.7, None),
    (2, 300, 20011, 1.0, True, 1.0, 20016),
    (1, 1024, 3001, 1.0, True, 1.0, None),
    (1, 20, 151936, 1.0, True, 1.0, None),
    (1, 6, 70001, 0.05, False, 1.0, None),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_the_oracle(dart, i):
    nseq, B, V, T, bf16, fill, ld = CASES[i]
    for again in range(3):
        z, dev, tokens, parents, n_nodes, u, noise = data(nseq, B, V, T, bf16, 9000 + 10 * i + again, fill, ld=ld)
        out = run(dart, dev, tokens, parents, n_nodes, T, u, noise)
        torch.cuda.synchronize()
        check(out, serve.verify(z, tokens, parents, n_nodes, T, u, noise), B + 1)


def test_a_whole_branch_and_none(dart):
    """A chain that is kept to its end, and one whose first node is not."""
    B, V = 30, 500
    z = np.zeros((2, B + 1, V), np.float32)
    tokens = np.stack([np.arange(B), np.arange(B)]).astype(np.int32)
    parents = np.stack([np.arange(B) - 1] * 2).astype(np.int32)
    for i in range(B):
        z[0, i, i] = 60.0
    z[1, 0, 77] = 60.0
    u, noise = np.full((2, B + 1), 0.5, np.float32), np.ones((2, V), np.float32)
    n = np.array([B, B], np.int32)
    for T in (0.0, 1.0):
        out = run(dart, up(z), tokens, parents, n, T, u, noise)
        check(out, serve.verify(z, tokens, parents, n, T, u, noise), B + 1)
        assert out["n_rows"].tolist() == [B + 1, 1] and int(out["tokens"][1, 0]) == 77


@pytest.mark.parametrize("T", [0.0, 1.0])
def test_odd_logits(dart, T):
    """Masked tokens, NaN, infinities, rows without a finite logit, rows whose
    children hold all of the mass, repeated and bad tokens and parents."""
    V, B = 300, 8
    inf = np.inf
    g = np.random.default_rng(3)
    z = g.standard_normal((9, B + 1, V)).astype(np.float32)
    parents = np.tile(np.array([-1, -1, -1, 0, 1, 2, 4, -1], np.int32), (9, 1))
    tokens = np.tile(np.array([5, 9, 5, 1, 2, 3, 4, 8], np.int32), (9, 1))
    z[0] = -inf                                # nothing anywhere
    z[1, 0, :] = -inf; z[1, 0, [5, 9]] = 1.0   # noqa: E702  only the children are left
    z[2, 0, 9] = inf                           # an infinite logit is the largest
    z[3, 0, 10:] = np.nan                      # NaN tokens are never taken
    z[4, 0, :] = -3.4028235e38                 # the type's lowest value everywhere
    z[5, 0, :] = -inf; z[5, 0, 9] = 2.0        # noqa: E702  one child alone
    z[6, 0, :] = np.nan
    tokens[7, :3] = [-1, V, 10 ** 9]           # no tokens of the vocabulary
    parents[8, :3] = [-1, 1, 7]                # parents that do not come before
    u = np.full((9, B + 1), 0.999999, np.float32)
    u[8] = 0.0
    noise = np.maximum(g.exponential(size=(9, V)), 1e-9).astype(np.float32)
    n = np.array([8] * 9, np.int32)
    out = run(dart, up(z), tokens, parents, n, T, u, noise)
    torch.cuda.synchronize()
    check(out, serve.verify(z, tokens, parents, n, T, u, noise), B + 1)


def test_ties_go_to_the_lowest_token(dart):
    V = 4000
    z = np.zeros((1, 2, V), np.float32)
    z[0, 0, [77, 78, 1999, 3999]] = 5.0
    z[0, 1, :] = 1.0
    tok, par, n = np.array([[78]], np.int32), np.array([[-1]], np.int32), np.array([1], np.int32)
    out = run(dart, up(z, torch.bfloat16), tok, par, n, 0.0, None, None)
    assert out["tokens"][0].tolist() == [77, -1]
    u, noise = np.zeros((1, 2), np.float32) + 0.9999, np.ones((1, V), np.float32)
    out = run(dart, up(z, torch.bfloat16), tok, par, n, 1.0, u, noise)
    assert out["tokens"][0].tolist() == [77, -1]


def test_the_tokens_follow_the_target(dart):
    """200000 draws of the first token from a distribution over 12 tokens, five
    of them children: chi-square with 11 degrees of freedom below 45 (the
    probability of more is 5e-6)."""
    g = np.random.default_rng(11)
    V, B, N = 12, 5, 20000
    z = np.tile(g.standard_normal(V).astype(np.float32), (N, B + 1, 1))
    tokens = np.tile(np.array([3, 7, 0, 11, 5], np.int32), (N, 1))
    parents = np.tile(np.array([-1, -1, -1, -1, 0], np.int32), (N, 1))
    n = np.full(N, B, np.int32)
    ver = dart.TreeVerifier(N, B, V, 0.8)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    count = np.zeros(V)
    args = [up(z), up(tokens), up(parents), up(n)]
    for _ in range(10):
        u = torch.rand((N, B + 1), generator=gen, device="cuda")
        noise = torch.empty((N, V), device="cuda").exponential_(generator=gen)
        first = ver(*args, u=u, noise=noise)["tokens"][:, 0]
        count += np.bincount(first.cpu().numpy(), minlength=V)
    p = np.exp(z[0, 0].astype(np.float64) / 0.8)
    p /= p.sum()
    chi = float(((count - 10 * N * p) ** 2 / (10 * N * p)).sum())
    assert chi < 45, chi


def test_every_call_gives_the_same_bits_captured_or_not(dart):
    z, dev, tokens, parents, n_nodes, u, noise = data(3, 40, 5000, 1.0, True, 9500)
    ver = dart.TreeVerifier(3, 40, 5000, 1.0)
    args = [dev, up(tokens), up(parents), up(n_nodes), up(u), up(noise)]
    first = {k: v.clone() for k, v in ver(*args).items()}
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        ver(*args)
    for v in ver.out.values():
        v.fill_(-7)
    graph.replay()
    torch.cuda.synchronize()
    for k, v in first.items():
        assert torch.equal(v, ver.out[k])
    check(ver.out, serve.verify(z, tokens, parents, n_nodes, 1.0, u, noise), 41)
