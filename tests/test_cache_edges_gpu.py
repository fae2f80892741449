"""Cache writes: the form for many tokens (four heads a group of threads), and
e4m3 codes and scales bit by bit.  Tolerances: see test_cache_append_gpu.py."""
import numpy as np
import pytest
import torch

import serve_data as sd
from test_cache_append_gpu import THETA, check, dart, setup, up  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hkv,R,path", [(5, 2500, False), (6, 2500, True), (8, 2449, False), (4, 4900, False)])
def test_many_tokens(dart, Hkv, R, path, fp8):  # noqa: F811
    """At least 9728 groups, heads that do not fill the last group of four among them."""
    lens, n_rows = [3, 130], [R, R - 600]
    cache, pool, table, dk, dv, k, v, rows = setup(dart, 2, R, lens, n_rows, 64, fp8, Hkv, 8200 + Hkv, path)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.append(dk, dv, up(table), up(lens), up(n_rows), rows=None if rows is None else up(rows), rope_theta=THETA, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    check(cache, pool, table, k, v, lens, n_rows, rows, 64, fp8)


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
