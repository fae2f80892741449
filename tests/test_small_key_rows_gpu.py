"""Keys near the smallest floats in e2m1 pages: their codes are the definition's
too, although a power of two over a block scale may leave the floats there and
remainders of products lie below them."""
import numpy as np
import pytest
import torch

from test_four_bits_exact_gpu import dart, wrong_codes  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [-126, -124, -122, -119, -115, -108, -61, -59])
def test_rows_near_the_smallest_floats(dart, exponent):  # noqa: F811
    g = np.random.default_rng(-exponent)
    kv = torch.from_numpy(g.standard_normal((3, 1800, 16, 128))).mul(2.0 ** exponent).to(torch.bfloat16).float()
    assert wrong_codes(dart, kv, [0, 3000, 131000], 8) == 0


def test_rows_of_all_magnitudes(dart):  # noqa: F811
    """A row of each magnitude from the smallest number on."""
    g = np.random.default_rng(8)
    kv = torch.from_numpy(g.standard_normal((1, 260, 4, 128)))
    kv = (kv * torch.exp2(torch.arange(260) - 133.0)[None, :, None, None]).to(torch.bfloat16).float()
    kv = torch.where(kv.abs() > 2.0 ** 125, 0.0, kv)  # (a rotation may leave the floats)
    assert wrong_codes(dart, kv, [77], 2) == 0
