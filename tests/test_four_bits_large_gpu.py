"""Attention over e2m1 pages whose elements are of 2^12: with logits of an
ordinary size against the oracle at ordinary tolerances (test_four_bits_gpu.py),
and with logits that leave one key its whole weight against that key's value.

There the output is the value row of the largest logit, where it leads by more
than 40 + 2 e (e: what test_paged_attn_gpu.py allows a logit to be off by), so
that all others weigh less than 2^-57 each: off by its rounding to bf16 (2^-8),
and of a cache value by the roundings of the probability, the scale over the tile's
power of two and its product with the code to f16 (2^-11 each), of a tree value by the probability's to bf16 (2^-8)."""
import numpy as np
import pytest
import torch

import four_data as fd
import test_four_bits_gpu as four_test
from oracle.tree_attn import root_path, rope
from test_paged_attn_gpu import dart  # noqa: F401

pytestmark = pytest.mark.gpu
SHAPES = [(0, 8, 2), (3, 16, 4), (20, 8, 2), (300, 4, 2)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_large_elements(dart, shape):  # noqa: F811
    B, Hq, Hkv = shape
    m = 2.0 ** 12
    x = fd.attn_data4(2, B, [400, 130], 32, Hq, Hkv, 9800 + B, magnitude=m)
    q, k, v = x.dev
    x.dev = ((q / m).contiguous(), (k * m).contiguous(), (v * m).contiguous())
    x.q, x.kt, x.vt = x.q / m, x.kt * m, x.vt * m
    four_test.check(x, four_test.run(dart, x))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_key_alone(dart, shape):  # noqa: F811
    B, Hq, Hkv = shape
    x = fd.attn_data4(2, B, [400, 130], 32, Hq, Hkv, 9850 + B, magnitude=2.0 ** 12)
    got = four_test.run(dart, x).double().cpu().numpy()
    used = 0
    for s, n in enumerate(x.lens):
        for r in range(x.B + 1):
            at = lambda j: int(n) + (int(x.depths[s][j - 1]) if j else 0)  # noqa: E731
            seen = [0] + ([1 + i for i in root_path(x.parents[s], r - 1)] if r else [])
            for h in range(Hq):
                g = h // (Hq // Hkv)
                keys = np.concatenate([x.ctx[s][0][:, g], np.stack([rope(x.kt[s, j, g], at(j), four_test.THETA) for j in seen])])
                y = rope(x.q[s, r, h], at(r), four_test.THETA)
                z = four_test.SCALE * keys @ y
                e = four_test.SCALE * (np.abs(keys) @ np.abs(y)).max() * (2 ** -7 + 2 ** -10)
                best = int(z.argmax())
                if z[best] - np.partition(z, -2)[-2] < 40 + 2 * e:
                    continue
                used += 1
                want = x.ctx[s][1][best, g] if best < n else x.vt[s, seen[best - int(n)], g]
                assert (np.abs(got[s, r, h] - want) <= np.abs(want) * (2 ** -8 + (3 * 2 ** -11 if best < n else 2 ** -8) + 2 ** -16) + 1e-30).all(), (s, r, h)
    assert used > 2 * Hq * (x.B + 1) // 10
