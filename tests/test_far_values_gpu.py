"""Values of the cache and of the tree that lie far from one another, over pages
of codes: the larger ones are the output, to the tolerances of
test_paged_attn_gpu.py and test_four_bits_gpu.py."""
import pytest
import torch

import four_data as fd
import serve_data as sd
import test_four_bits_gpu as four_test
import test_paged_attn_gpu as paged_test
from test_paged_attn_gpu import dart  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,tree", [(2.0 ** -110, 2.0 ** 30), (2.0 ** -70, 2.0 ** 60), (2.0 ** -30, 2.0 ** 30), (2.0 ** -45, 1.0), (2.0 ** 60, 2.0 ** -40),
                                        (2.0 ** -110, 2.0 ** 110), (2.0 ** -20, 2.0 ** 80), (0.0, 2.0 ** 110)],
                         ids=str)
@pytest.mark.parametrize("shape", [(0, 8, 2), (3, 16, 4), (20, 8, 2), (300, 4, 2)], ids=str)
@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_one_side_far_above(dart, kind, shape, cache, tree):  # noqa: F811
    B, Hq, Hkv = shape
    x = (fd.attn_data4 if kind == "e2m1" else lambda *a: sd.attn_data(*a[:4], True, *a[4:]))(2, B, [300, 128], 32, Hq, Hkv, 9750 + B)
    x.pool[3].mul_(cache)
    x.ctx = [(k, v * cache) for k, v in x.ctx]
    x.dev = (x.dev[0], x.dev[1], (x.dev[2] * tree).contiguous())
    x.vt = x.vt * tree
    t = four_test if kind == "e2m1" else paged_test
    got = t.run(dart, x)
    assert torch.isfinite(got.float()).all()
    t.check(x, got)
