"""Inputs of the e2m1 pages' tests: the arrays of serve_data over a pool of
codes whose unused slots hold NaN block scales and scales."""
import numpy as np
import torch

import canary
import serve_data as sd
from oracle import four

F4 = torch.float4_e2m1fn_x2


def guarded(a, dtype):
    """A numpy array in guarded device memory, as `dtype`."""
    raw = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    d = canary.empty(tuple(raw.shape), dtype=raw.dtype)
    d.copy_(raw)
    return d.view(dtype)


def pool4(tables, lens, page, Hkv, num_pages, g, magnitude=1.0):
    """Codes, block scales (zeros and the largest among them) and scales that are
    no powers of two for the sequences' tokens, garbage and NaN elsewhere.
    Returns [k, v, k_scale, v_scale, k_block, v_block] (numpy) and ctx."""
    shape = (num_pages, Hkv, page)
    code = [g.integers(0, 256, shape + (sd.DH // 2,), dtype=np.uint8) for _ in range(2)]
    block = [np.full(shape + (8,), 0x7F, np.uint8) for _ in range(2)]
    scale = [np.full(shape, np.nan, np.float32) for _ in range(2)]
    ctx = []
    for s, n in enumerate(lens):
        pos = np.arange(n)
        at, slot = tables[s][pos // page].astype(np.int64), pos % page
        both = []
        for i in range(2):
            b = g.integers(0x48, 0x60, (n, Hkv, 8), dtype=np.uint8)  # 4 .. 30
            odd = g.random((n, Hkv, 8))
            b[odd < 0.02] = 0
            b[odd > 0.99] = 0x7E
            sc = (magnitude * 2.0 ** -6 * g.uniform(0.7, 1.4, (n, Hkv))).astype(np.float32)
            sc[b.max(-1) == 0x7E] *= 2.0 ** -4
            block[i][at, :, slot], scale[i][at, :, slot] = b, sc
            both.append(four.values(four.unpack(code[i][at, :, slot]), b, sc))
        ctx.append(tuple(both))
    return code + scale + block, ctx


def attn_data4(nseq, B, lens, page, Hq, Hkv, seed, magnitude=1.0, **more):
    x = sd.attn_data(nseq, B, lens, page, False, Hq, Hkv, seed, **more)
    pool, x.ctx = pool4(x.table.cpu().numpy(), lens, page, Hkv, x.pool[0].shape[0], np.random.default_rng(seed + 1), magnitude)
    x.pool = [guarded(a, t) for a, t in zip(pool, (F4, F4, torch.float32, torch.float32, sd.E4M3, sd.E4M3))]
    return x
