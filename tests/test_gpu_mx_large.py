"""Quantization of matrices of more than 300 tiles of 128 x 128, bit for bit: a CTA takes a whole tile there."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2109_12497_b200 import binding as B
from test_gpu_mx import DT, as_matrix, check_mx, empty_mx, spread, status

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,pad,offset", [(2565, 2048, 0, 0), (2565, 1992, 8, 8), (2530, 2043, 3, 1), (2433, 2029, 0, 0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [0, 16])
def test_quantize_is_the_definition_bit_for_bit(rows, cols, pad, offset, dtype, bits):
    assert -(-rows // 128) * -(-cols // 128) > 300
    g = as_matrix(spread(rows, cols, rows + cols), DT[dtype], pad, offset)
    x, seed = g.double().cpu().numpy(), 0x0F1E2D3C4B5A6978
    h = ref.draws(rows, cols, seed) if bits else None
    q, qt, q1, qt1 = empty_mx(rows, cols, 16), empty_mx(cols, rows, 32), empty_mx(rows, cols, 16), empty_mx(cols, rows, 32)
    st = status()
    B.uq_mx_quantize(g, seed, bits, q, qt, st)               # both from one read
    check_mx(q, x, h)
    check_mx(qt, np.ascontiguousarray(x.T), None if h is None else np.ascontiguousarray(h.T))
    B.uq_mx_quantize(g, seed, bits, q1, None, st)            # and either alone: the same
    B.uq_mx_quantize(g, seed, bits, None, qt1, st)
    for one, both, n in ((q1, q, rows), (qt1, qt, cols)):
        assert torch.equal(one.codes, both.codes)
        got, want = (ref.unpack(m.codes.cpu().numpy(), m.scales.cpu().numpy(), m.rows, m.cols)[1:] for m in (one, both))
        assert all(np.array_equal(a, b) for a, b in zip(got, want))
    assert int(st.item()) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_blocks_that_are_not_finite(dtype):
    rows, cols = 2530, 2043
    x = spread(rows, cols, 3)
    for r, c, v in ((0, 0, np.nan), (127, 2042, np.inf), (1300, 1000, -np.inf), (2529, 2042, np.nan)):
        x[r, c] = v
    for bits in (0, 16):
        g = as_matrix(x, DT[dtype], 1, 1)
        xs, h = g.double().cpu().numpy(), ref.draws(rows, cols, 5) if bits else None
        q, qt, st = empty_mx(rows, cols), empty_mx(cols, rows), status()
        B.uq_mx_quantize(g, 5, bits, q, None, st)
        B.uq_mx_quantize(g, 5, bits, None, qt, st)
        assert int(st.item()) == B.UQ_STATUS_NONFINITE
        check_mx(q, xs, h)
        check_mx(qt, np.ascontiguousarray(xs.T), None if h is None else np.ascontiguousarray(h.T))
