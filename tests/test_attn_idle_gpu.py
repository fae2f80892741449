"""Single calls of the contiguous tree attention on an idle GPU with cold caches:
no bounded wait gives up (the thread that issues the products may be late by more
than a key tile, so the softmax's arrivals are counted per P buffer), and every
call gives the same bits."""
import numpy as np
import pytest
import torch

import canary
from workloads import AttnConfig, make_attn_inputs
from test_attn_gpu import bf_dev, dart  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nseq,B,C,tiles", [(1, 16, 20000, 1), (24, 32, 2048, 1), (4, 64, 2048, 1), (8, 512, 2048, 2)])
def test_cold_calls_give_up_no_wait(dart, nseq, B, C, tiles):  # noqa: F811
    cfg = AttnConfig("idle", nseq, B, C, 16, 64, 4600)
    x = make_attn_inputs(cfg)
    assert dart.dart_tree_attention_tiles(dart.make_attn_config(nseq, B, C, cfg.Hq, cfg.Hkv, cfg.dh, cfg.rope_theta, cfg.scale), 152) == tiles
    par, n = torch.from_numpy(x["parents"]).cuda(), torch.from_numpy(x["n_nodes"]).cuda()
    mask = canary.empty((nseq, B, (B + 63) // 64), dtype=torch.int64, device="cuda")
    dart.dart_ancestor_mask(par, n, mask)
    dep = torch.from_numpy(x["depths"]).cuda()
    pos = torch.where(dep > 0, dep + cfg.offset, torch.full_like(dep, -1)).to(torch.int32)
    att = dart.TreeAttention(nseq, B, C, cfg.Hq, cfg.Hkv, cfg.dh, cfg.rope_theta, cfg.scale)
    args = [bf_dev(x[k]) for k in ("q", "k_tree", "v_tree", "k_ctx", "v_ctx")] + [pos, mask, n]
    cold = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    first = None
    for i in range(6):
        cold.fill_(i)
        torch.cuda.synchronize()
        out = att(*args, status)
        torch.cuda.synchronize()
        assert not status.any()
        first = out.clone() if first is None else first
        assert torch.equal(out, first)
    assert np.isfinite(first.cpu().numpy()).all()
