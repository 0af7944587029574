"""Layer norm where its tests of every size do not go: values at the ends of a type's range."""
import numpy as np
import pytest
import torch

from paper_2109_12497_b200 import binding as B
from test_gpu_mx import DT, as_matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [1, 3, 255, 300, 1001, 2047, 4001, 8191, 8201])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_beyond_a_row_reaches_its_sums(cols, dtype):
    """Rows of one large value, whose mean times 1 / deviation is beyond binary32 while every (x - mean) rstd is 0: in places that a
    thread has beyond the row's end nothing may become of that product.  Powers of two and whole numbers: all is exact."""
    rows, big, rstd = 5, 2.0 ** 120, 2.0 ** 20
    x = as_matrix(np.full((rows, cols), big), DT[dtype], 1, 1)
    d = np.random.default_rng(cols).integers(-2, 3, (rows, cols)).astype(np.float64)
    t, dx = as_matrix(d, DT[dtype], 1, 1), as_matrix(np.zeros((rows, cols)), DT[dtype], 1, 1)
    dg, db = torch.full((cols,), 9.0, device="cuda"), torch.full((cols,), 9.0, device="cuda")
    ws = torch.empty(B.uq_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.uq_layer_norm_backward(t, x, None, torch.full((rows,), big, device="cuda"), torch.full((rows,), rstd, device="cuda"), dx, dg, db, ws)
    assert not dg.any() and np.array_equal(db.double().cpu().numpy(), d.sum(0))
    got = dx.double().cpu().numpy()
    # sum t is a whole number below 2^24; its product with 1 / cols, the difference and the product with rstd: three roundings, and dx's
    want = rstd * (d - d.mean(1, keepdims=True))
    e = 4 * 2.0 ** -24 * rstd * (np.abs(d) + np.abs(d.mean(1, keepdims=True)))
    assert (np.abs(got - want) <= e + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (np.abs(want) + e)).all()
