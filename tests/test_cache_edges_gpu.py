"""Cache writes: e4m3 codes and scales bit by bit."""
import numpy as np
import pytest
import torch

import serve_data as sd
from test_cache_append_gpu import THETA, dart, setup, up  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.0, 1e-30, 1e-33, 3e-36, 1e36])
def test_codes_and_scales_are_those_of_the_definition(dart, scale):  # noqa: F811
    """Values (not rotated): scale = max |x| / 448 (at least 2^-120) and x / scale,
    each rounded once to fp32, the quotient then to e4m3: the same bits."""
    R, Hkv = 600, 4
    cache, pool, table, dk, dv, k, v, _ = setup(dart, 1, R, [0], [R], 64, True, Hkv, 8210, scale=scale)
    dv = dv.clone()
    g = torch.Generator().manual_seed(1)
    # halves of the heads in few bits, whose quotients often lie between two codes
    few = (torch.randint(-9, 10, (1, R, 2, 128), generator=g).float() * scale).to(torch.bfloat16)
    dv[:, :, :2] = few.cuda()
    cache.append(dk, dv, up(table), up([0]), up([R]), rope_theta=THETA)
    torch.cuda.synchronize()
    x = dv[0].float().cpu()
    amax = x.abs().amax(-1)
    want = torch.where(amax > 0, torch.clamp(amax / 448.0, min=2.0 ** -120), torch.ones_like(amax))
    codes = (x / want[..., None]).to(sd.E4M3).view(torch.uint8)
    pos = torch.arange(R)
    page, slot = torch.from_numpy(table[0].astype(np.int64))[pos // 64], pos % 64
    assert torch.equal(cache.v_scale.cpu()[page, :, slot], want)
    got = cache.v.view(torch.uint8).cpu()[page, :, slot]
    assert torch.equal(got, codes), int((got != codes).sum())
