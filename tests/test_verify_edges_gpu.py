"""Verification of the tree at the edges of its contract, against the fp64
oracle: infinite logits in both types, children without a share of their own,
masked tokens, rows with many children, and rows longer than a thread's
registers hold.  Tolerance of log p: see test_verify_tree_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import serve
from test_verify_tree_gpu import LOGP, check, dart, data, run, up  # noqa: F401

pytestmark = pytest.mark.gpu

F32_MAX = 3.4028235e38
TYPES = [torch.float32, torch.bfloat16]


def device_logits(z, dtype, ld=None):
    """z [nseq][R][V] as dtype on the GPU (its values have to be of that type),
    rows `ld` apart, and what the oracle takes."""
    t = torch.from_numpy(z).to(dtype)
    d = t.cuda()
    if ld:
        wide = torch.full((*z.shape[:2], ld), 1e30, dtype=dtype, device="cuda")
        wide[..., :z.shape[2]] = d
        d = wide[..., :z.shape[2]]
    return t.float().numpy(), d


@pytest.mark.parametrize("ld", [None, 301, 305])
@pytest.mark.parametrize("T", [0.0, 1.0, 0.7])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_infinite_logits(dart, dtype, T, ld):  # noqa: F811
    """+inf counts as the largest number of the type wherever it stands: on a child,
    beside the children, on both, among the elements that no 16-byte vector holds."""
    V, B, inf = 300, 4, np.inf
    g = np.random.default_rng(21)
    z = g.standard_normal((12, B + 1, V)).astype(np.float32)
    tokens = np.tile(np.array([5, 9, 1, 2], np.int32), (12, 1))
    parents = np.tile(np.array([-1, -1, 0, 1], np.int32), (12, 1))
    u = np.full((12, B + 1), 0.25, np.float32)
    z[0, 0, 9] = inf                                       # a child
    z[1, 0, 77] = inf                                      # no child
    z[2, 0, [9, 77]] = inf                                 # both: half of the mass each
    z[3, 0, [9, 77]] = inf; u[3] = 0.75                    # noqa: E702
    z[4, 0, [5, 9]] = inf                                  # two children
    z[5, 0, [5, 9]] = inf; u[5] = 0.75                     # noqa: E702
    z[6, 0, [77, 299]] = inf                               # the last element of the row
    z[7, 0, [0, 77]] = inf                                 # the first
    z[8, 0, 20] = float(torch.finfo(dtype).max); z[8, 0, 77] = inf   # noqa: E702  (equal: a tie)
    z[9, 0, 9] = inf; z[9, 2] = z[9, 0]; z[9, 4, 298] = inf          # noqa: E702  further down a branch
    z[10, 0, [1, 296, 299]] = inf; u[10] = 0.9             # noqa: E702
    z[11, 0, :] = inf; u[11] = 0.999                       # noqa: E702  everywhere
    zf, d = device_logits(torch.from_numpy(z).to(dtype).float().numpy(), dtype, ld)
    zf = np.minimum(zf, float(torch.finfo(dtype).max))
    noise = np.maximum(g.exponential(size=(12, V)), 1e-9).astype(np.float32)
    n = np.full(12, B, np.int32)
    out = run(dart, d, tokens, parents, n, T, u, noise)
    torch.cuda.synchronize()
    check(out, serve.verify(zf, tokens, parents, n, T, u, noise), B + 1)


def test_a_child_without_a_share_is_not_kept(dart):  # noqa: F811
    """Four children before one whose token an earlier sibling has and one with
    p = 0: whatever u is, on the border between their neighbours too, neither
    is kept."""
    factors, steps = np.linspace(1.02, 1.98, 16), np.arange(-64, 64)
    nseq, V, B = len(factors) * len(steps), 16, 5
    z = np.full((nseq, B + 1, V), -300.0, np.float32)
    z[:, :, 0] = z[:, :, 15] = 0.0
    z[:, :, [1, 2]] = (np.log(np.repeat(factors, len(steps))) - 24 * np.log(2)).astype(np.float32)[:, None, None]
    tokens = np.tile(np.array([0, 1, 2, 1, 3], np.int32), (nseq, 1))
    parents = np.full((nseq, B), -1, np.int32)
    u = np.zeros((nseq, B + 1), np.float32)
    u[:, 0] = np.tile(0.5 + steps * 2.0 ** -24, len(factors))
    out = run(dart, up(z), tokens, parents, np.full(nseq, B, np.int32), 1.0, u, np.ones((nseq, V), np.float32))
    kept = out["rows"][:, 1].cpu().numpy()
    assert set(kept.tolist()) <= {-1, 1, 2, 3}, np.unique(kept, return_counts=True)
    assert (kept == -1).any() and (kept == 1).any()


@pytest.mark.parametrize("low", [-F32_MAX, -1e30, -300.0], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_a_masked_token_is_never_drawn(dart, dtype, low):  # noqa: F811
    """The children hold all of the mass, the other tokens are masked by a low
    logit instead of -inf, and u is the last number below 1: rounding may put it
    past the children, but a token of p = 0 does not follow."""
    nseq, V, B = 512, 600, 20
    g = np.random.default_rng(22)
    low = float(torch.tensor(low).to(dtype)) if low > -1e38 else float(torch.finfo(dtype).min)
    z = np.full((nseq, B + 1, V), low, np.float32)
    z[:, :, :B] = g.standard_normal((nseq, B + 1, B)) * 3
    zf, d = device_logits(torch.from_numpy(z).to(dtype).float().numpy(), dtype)
    tokens, parents = np.tile(np.arange(B, dtype=np.int32), (nseq, 1)), np.full((nseq, B), -1, np.int32)
    u = np.full((nseq, B + 1), 1 - 2.0 ** -24, np.float32)
    noise = np.maximum(g.exponential(size=(nseq, V)), 1e-9).astype(np.float32)
    out = run(dart, d, tokens, parents, np.full(nseq, B, np.int32), 1.0, u, noise)
    first = out["tokens"][:, 0].cpu().numpy()
    assert ((first >= 0) & (first < B)).all(), np.unique(first[first >= B])
    want = zf[np.arange(nseq), 0, first]
    lp = want - np.log(np.exp(zf[:, 0, :B].astype(np.float64)).sum(1))
    assert np.abs(out["logp"][:, 0].cpu().numpy() - lp).max() <= LOGP


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("T", [0.0, 1.0])
@pytest.mark.parametrize("kids", [31, 32, 33, 64, 200])
def test_many_children_of_one_row(dart, kids, T, dtype):  # noqa: F811
    """Repeated tokens on both sides of the 32nd child, u in the middle of the
    first, the last and the border children's shares, and beyond all of them."""
    V, B = 400, 210
    g = np.random.default_rng(23)
    picks = sorted({0, 1, kids // 2, kids - 1} | ({31, 32, 33} & set(range(kids))))
    nseq = len(picks) + 1
    row = torch.from_numpy(g.standard_normal(V).astype(np.float32)).to(dtype).float().numpy()
    toks = g.permutation(V)[:B].astype(np.int32)
    for a, b in ((2, 0), (28, 5), (35, 3), (40, 36), (100, 30)):  # child a repeats child b
        if a < kids and a not in picks:
            toks[a] = toks[b]
    z = np.tile(row, (nseq, B + 1, 1))
    parents = np.full((nseq, B), 0, np.int32)  # the others: children of the first node
    parents[:, :kids] = -1
    tokens = np.tile(toks, (nseq, 1))
    p = np.exp(row.astype(np.float64))
    p /= p.sum()
    share = np.array([0.0 if toks[i] in toks[:i] else p[toks[i]] for i in range(kids)])
    upto = np.cumsum(share)
    u = np.full((nseq, B + 1), 0.9999, np.float32)
    for s, i in enumerate(picks):
        u[s, 0] = upto[i] - share[i] / 2
        if T == 0:
            z[s, 0, toks[i]] = 10.0
    u[nseq - 1, 0] = (upto[-1] + 1) / 2
    noise = np.maximum(g.exponential(size=(nseq, V)), 1e-9).astype(np.float32)
    zf, d = device_logits(z, dtype)
    n = np.full(nseq, B, np.int32)
    out = run(dart, d, tokens, parents, n, T, u, noise)
    want = serve.verify(zf, tokens, parents, n, T, u, noise)
    assert [w[0][1] for w in want[:-1]] == [i + 1 for i in picks]  # (the oracle keeps the children that were meant)
    check(out, want, B + 1)


@pytest.mark.parametrize("T", [0.0, 0.9])
@pytest.mark.parametrize("nseq,V,dtype", [(1, 151936, torch.float32), (24, 70001, torch.float32), (24, 20011, torch.bfloat16),
                                          (24, 150000, torch.bfloat16)], ids=str)
def test_long_rows_and_many_sequences(dart, nseq, V, dtype, T):  # noqa: F811
    """Rows beyond the vectors that a thread holds, with children, the largest
    logit and the token that follows among the elements behind them, and the
    clusters of many sequences."""
    B = 6
    g = np.random.default_rng(24)
    ctas = 16 if nseq == 1 else 8
    width = 4 if dtype == torch.float32 else 8
    share = V // width // ctas
    behind = np.concatenate([np.arange(min(512 * 4, share - 1), share) + r * share for r in range(ctas)]) * width
    behind = behind[behind < V - width]
    z = g.standard_normal((nseq, B + 1, V)).astype(np.float32)
    tokens = np.zeros((nseq, B), np.int32)
    parents = np.tile(np.array([-1, -1, -1, 0, 1, 3], np.int32), (nseq, 1))
    last = g.choice(behind, nseq)
    for s in range(nseq):
        tokens[s] = g.choice(np.setdiff1d(behind, last[s]), B, replace=False) + g.integers(0, width, B)
        z[s, 0, tokens[s, s % 3]] = 16.0
        for r in range(1, B + 1):
            z[s, r, last[s] + 1] = 16.0
    zf, d = device_logits(torch.from_numpy(z).to(dtype).float().numpy(), dtype)
    u = np.full((nseq, B + 1), 0.5, np.float32)
    noise = np.maximum(g.exponential(size=(nseq, V)), 1e-3).astype(np.float32)
    n = np.full(nseq, B, np.int32)
    out = run(dart, d, tokens, parents, n, T, u, noise)
    want = serve.verify(zf, tokens, parents, n, T, u, noise)
    assert any(len(w[0]) > 1 for w in want)
    check(out, want, B + 1)
