"""Layer norm's rows in shared memory at the border of what a kernel may have without asking for more: 48 KiB of dynamic and
static memory together."""
import multiprocessing

import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2109_12497_b200 import binding as B
from test_gpu_layer_norm import EPS, U, backward_bounds, cuda, f64, forward_bounds, inputs
from test_gpu_mx import DT, as_matrix, check_mx, empty_mx

pytestmark = pytest.mark.gpu

# (pass, type, columns, padding, offset) whose ring takes at most 48 KiB, and more with the kernel's own arrays.  Each list has a
# kernel once: what a kernel was granted for longer rows, it keeps.
FIRST_CALLS = {
    "shortest": [("forward", "f32", 4089, 0, 0), ("forward", "f32", 4092, 0, 0), ("quantized", "f32", 4089, 0, 0),
                 ("forward", "bf16", 8169, 0, 0), ("forward", "bf16", 8176, 0, 0), ("quantized", "bf16", 8169, 0, 0),
                 ("quantized", "bf16", 8176, 0, 0), ("backward", "f32", 505, 0, 0), ("backward", "f32", 508, 0, 0),
                 ("backward", "f32", 2041, 0, 0), ("backward", "f32", 2044, 0, 0), ("backward", "bf16", 4073, 0, 0),
                 ("backward", "bf16", 4080, 0, 0)],
    "longest": [("forward", "f32", 4092, 3, 1), ("forward", "f32", 4092, 4, 4), ("quantized", "f32", 4092, 4, 0),
                ("forward", "bf16", 8184, 3, 1), ("forward", "bf16", 8184, 8, 8), ("quantized", "bf16", 8184, 3, 1),
                ("quantized", "bf16", 8184, 8, 0), ("backward", "f32", 508, 3, 1), ("backward", "f32", 508, 4, 4),
                ("backward", "f32", 2044, 3, 1), ("backward", "f32", 2044, 4, 4), ("backward", "bf16", 4088, 3, 1),
                ("backward", "bf16", 4088, 8, 8)],
}


def one_call(kind, dtype, cols, pad, offset):
    """The call against its definition; None, or what is wrong."""
    rows = 3
    x, gamma, beta, dy = inputs(rows, cols, cols)
    t = as_matrix(x, DT[dtype], pad, offset)
    xs = f64(t)
    if kind == "backward":
        d, dx = as_matrix(dy, DT[dtype], pad, offset), as_matrix(np.zeros((rows, cols)), DT[dtype], pad, offset)
        mean, rstd = (v.astype(np.float32) for v in ref.layer_norm(xs, None, None, EPS)[1:])
        dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        ws = torch.empty(B.uq_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        B.uq_layer_norm_backward(d, t, cuda(gamma), cuda(mean), cuda(rstd), dx, dg, db, ws)
        args = f64(d), xs, gamma, mean.astype(np.float64), rstd.astype(np.float64)
        for got, want, e, u in zip((dx, dg, db), ref.layer_norm_backward(*args), backward_bounds(*args, cols, rows),
                                   (U[dtype], U["f32"], U["f32"])):
            assert (np.abs(f64(got) - want) <= e + u * (np.abs(want) + e)).all()
        return
    y = as_matrix(np.zeros((rows, cols)), DT[dtype], pad, offset)
    q = empty_mx(rows, cols) if kind == "quantized" else None
    B.uq_layer_norm(t, cuda(gamma), cuda(beta), EPS, y, None, None, q)
    want, mean, rstd = ref.layer_norm(xs, gamma, beta, EPS)
    e = forward_bounds(xs, gamma, beta, mean, rstd, cols)[2]
    assert (np.abs(f64(y) - want) <= e + U[dtype] * (np.abs(want) + e)).all()
    if q is not None:
        check_mx(q, f64(y), None)


def first_calls(which, results):
    for call in FIRST_CALLS[which]:
        try:
            one_call(*call)
        except Exception as e:                               # refused, or not the definition's
            results.put((call, repr(e)))
    results.put(None)


@pytest.mark.parametrize("which", FIRST_CALLS)
def test_the_first_call_of_a_process_is_not_refused(which):
    ctx = multiprocessing.get_context("spawn")
    results = ctx.Queue()
    child = ctx.Process(target=first_calls, args=(which, results))
    child.start()
    wrong = list(iter(lambda: results.get(timeout=300), None))
    child.join()
    assert wrong == []
