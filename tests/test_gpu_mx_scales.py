"""The product with scales at the ends of their range."""
import numpy as np
import pytest
import torch

from paper_2109_12497_b200 import binding as B
from test_gpu_mx import random_mx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(3, 130, 500), (200, 140, 300), (2100, 2200, 300)])
def test_product_of_any_two_scales(m, n, k):
    """Scales of two neighbouring bytes each: products are multiples of a quarter of 2^(sum of the lower ones), at most 36 * 4 of
    it, so that sums of 500 are below 2^20 quarters and exact in binary32, whose normal range they stay in: 2^-126 < unit / 4 and
    500 * 144 units < 2^128."""
    assert k * 36 * 4 * 4 < 2 ** 24
    for lo_a, lo_b in ((0, 252), (252, 0), (2, 245), (30, 224), (200, 54), (0, 131), (132, 0), (63, 69), (253, 100), (120, 244)):
        unit = lo_a + lo_b - 254
        assert unit - 2 >= -126 and unit + 17 < 128
        a, va = random_mx(m, k, lo_a, lo_a, min(lo_a + 2, 255))
        b, vb = random_mx(n, k, lo_b + 1, lo_b, min(lo_b + 2, 255))
        out = torch.full((m, n), 7.0, device="cuda")
        B.uq_mx_product(a, b, out, None, None)
        assert np.array_equal(out.double().cpu().numpy(), va @ vb.T)
