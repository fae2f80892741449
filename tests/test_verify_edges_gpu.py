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
    """+inf counts as the largest float wherever it stands: on a child, beside
    the children, on both, among the elements that no 16-byte vector holds."""
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
    z[8, 0, 20] = float(torch.finfo(dtype).max); z[8, 0, 77] = inf   # noqa: E702  (fp32: equal, so a tie)
    z[9, 0, 9] = inf; z[9, 2] = z[9, 0]; z[9, 4, 298] = inf          # noqa: E702  further down a branch
    z[10, 0, [1, 296, 299]] = inf; u[10] = 0.9             # noqa: E702
    z[11, 0, :] = inf; u[11] = 0.999                       # noqa: E702  everywhere
    zf, d = device_logits(torch.from_numpy(z).to(dtype).float().numpy(), dtype, ld)
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
