"""Layer norm's rows of whole 16-byte accesses, of every kernel: rows that fill its threads and rows that do not, more rows than the
CTAs have at once, and rows that are longer than a CTA's registers, aligned and not."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2109_12497_b200 import binding as B
from test_gpu_layer_norm import EPS, U, backward_bounds, cuda, f64, forward_bounds, inputs
from test_gpu_mx import DT, as_matrix, check_mx, empty_mx, status

pytestmark = pytest.mark.gpu

# by their columns: a warp with one piece and with two, 64 to 512 threads, two CTAs (backward), the kernels of any length
CLASSES = [248, 256, 504, 512, 1016, 1024, 2040, 2048, 4056, 4096, 8152, 8192, 16360, 16384]
TALL = [(8001, 256), (8003, 504), (4003, 1024), (2001, 2040), (1803, 4096), (1001, 8152), (501, 16384), (310, 16376)]
LONG = [(3, 16392), (130, 16400), (67, 40008), (130, 16393), (200, 20001)]
SIZES = [(5, c) for c in CLASSES] + TALL + LONG
WIDE = ((0, 0), (8, 8))                                      # (padding, offset): rows on 16 bytes if the columns are whole
BOTH = {c: ((0, 0), (3, 1)) for _, c in LONG}


def places(cols):
    return BOTH.get(cols, WIDE)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(rows, cols, dtype):
    x, gamma, beta, _ = inputs(rows, cols, rows + cols)
    for pad, offset in places(cols):
        t, y = as_matrix(x, DT[dtype], pad, offset), as_matrix(np.zeros((rows, cols)), DT[dtype], pad, offset)
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        B.uq_layer_norm(t, cuda(gamma), cuda(beta), EPS, y, mean, rstd)
        xs = f64(t)
        want, wm, wr = ref.layer_norm(xs, gamma, beta, EPS)
        em, er, ey = forward_bounds(xs, gamma, beta, wm, wr, cols)
        assert (np.abs(f64(mean) - wm) <= em).all() and (np.abs(f64(rstd) - wr) <= er).all()
        assert (np.abs(f64(y) - want) <= ey + U[dtype] * (np.abs(want) + ey)).all()


@pytest.mark.parametrize("rows,cols", [(5, c) for c in CLASSES] + [(2501, 96), (1001, 1024), (700, 2040), (301, 8192), (160, 16376)] + LONG)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantized_on_the_way_out(rows, cols, dtype):
    x, gamma, beta, _ = inputs(rows, cols, rows * 3 + cols)
    for pad, offset in places(cols):
        t, y = as_matrix(x, DT[dtype], pad, offset), as_matrix(np.zeros((rows, cols)), DT[dtype], pad, offset)
        q, q2, st = empty_mx(rows, cols, 16), empty_mx(rows, cols), status()
        B.uq_layer_norm(t, cuda(gamma), cuda(beta), EPS, y, None, None, q, st)
        xs = f64(t)
        want, wm, wr = ref.layer_norm(xs, gamma, beta, EPS)
        ey = forward_bounds(xs, gamma, beta, wm, wr, cols)[2]
        assert (np.abs(f64(y) - want) <= ey + U[dtype] * (np.abs(want) + ey)).all()
        check_mx(q, f64(y), None)
        B.uq_layer_norm(t, cuda(gamma), cuda(beta), EPS, None, None, None, q2, st)
        need = 16 * -(-cols // 32)
        assert torch.equal(q.codes[:, :need], q2.codes) and torch.equal(q.scales, q2.scales) and int(st.item()) == 0


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(rows, cols, dtype):
    x, gamma, _, dy = inputs(rows, cols, rows * 5 + cols)
    for (pad, offset), grad in zip(places(cols), ("f32", "bf16")):
        t, d = as_matrix(x, DT[dtype], pad, offset), as_matrix(dy, DT[dtype], 2 * pad, offset)
        dx = as_matrix(np.zeros((rows, cols)), DT[dtype], pad, offset)
        xs, ds = f64(t), f64(d)
        mean, rstd = (v.astype(np.float32) for v in ref.layer_norm(xs, None, None, EPS)[1:])
        dg, db = torch.empty(cols, dtype=DT[grad], device="cuda"), torch.empty(cols, dtype=DT[grad], device="cuda")
        ws = torch.full((B.uq_layer_norm_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
        B.uq_layer_norm_backward(d, t, cuda(gamma), cuda(mean), cuda(rstd), dx, dg, db, ws)
        args = ds, xs, gamma, mean.astype(np.float64), rstd.astype(np.float64)
        for got, want, e, kind in zip((dx, dg, db), ref.layer_norm_backward(*args), backward_bounds(*args, cols, rows), (dtype, grad, grad)):
            assert (np.abs(f64(got) - want) <= e + U[kind] * (np.abs(want) + e)).all()
        assert torch.isnan(dx.as_strided((rows, cols + pad), (cols + pad, 1))[:, cols:]).all()
