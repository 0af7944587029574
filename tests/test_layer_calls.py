"""The layer operators' argument checks, on the host: nothing here reaches a launch, so no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2109_12497_b200 import binding as B
from paper_2109_12497_b200 import build as uq_build

P = 0x10000
BAD, WS, UNSUPPORTED, OK = B.UQ_ERR_BAD_ARG, B.UQ_ERR_WORKSPACE, B.UQ_ERR_UNSUPPORTED, B.UQ_OK


@pytest.fixture(scope="module")
def lib():
    uq_build.build()
    return B.lib()


def mx(rows=64, cols=100, stride=64, codes=P, scales=P):
    return C.byref(B.uq_mx(rows, cols, stride, codes, scales))


def test_sizes(lib):
    for rows, cols, tiles in ((0, 5, 0), (1, 1, 1), (128, 128, 1), (129, 128, 2), (128, 129, 2), (300, 1000, 24)):
        assert lib.uq_mx_scale_bytes(rows, cols) == tiles * 512 == B.mx_scale_bytes(rows, cols)
    assert lib.uq_mx_scale_bytes(-1, 5) == 0 and lib.uq_mx_scale_bytes(1 << 31, 5) == 0
    assert lib.uq_layer_norm_workspace_bytes(-1, 5) == 0 and lib.uq_layer_norm_workspace_bytes(0, 5) == 0
    assert lib.uq_layer_norm_workspace_bytes(1, 5) >= 2 * 5 * 4
    for cols in (100, 1000, 2000, 4000, 8000, 12000, 20000):
        sizes = [lib.uq_layer_norm_workspace_bytes(rows, cols) for rows in range(1, 5000, 7)]
        assert sizes == sorted(sizes)                        # a workspace for many rows does for fewer
    last = 0
    for rows in (1, 10, 100, 1000, 10 ** 6):                 # more rows never need less, and at most some megabytes for 1000 columns
        n = lib.uq_layer_norm_workspace_bytes(rows, 1000)
        assert last <= n <= 16 << 20
        last = n


def test_quantize_refuses(lib):
    def call(x=P, rows=64, cols=100, ld=100, dtype=B.UQ_F32, bits=0, q=mx(), qt=None, status=None):
        return lib.uq_mx_quantize(x, rows, cols, ld, dtype, 0, bits, q, qt, status, None)
    assert call(x=None) == BAD and call(x=P + 2) == BAD and call(ld=99) == BAD and call(dtype=2) == BAD
    assert call(dtype=B.UQ_BF16, x=P + 1) == BAD
    assert call(bits=32) == BAD and call(bits=-1) == BAD and call(q=None) == BAD and call(status=P + 2) == BAD
    assert call(rows=-1, q=mx(-1)) == BAD and call(rows=(1 << 30) + 1, q=mx((1 << 30) + 1)) == BAD
    for bad in (mx(rows=63), mx(cols=101), mx(stride=48), mx(stride=72), mx(codes=None), mx(codes=P + 8), mx(scales=None),
                mx(scales=P + 4)):
        assert call(q=bad) == BAD
    assert call(qt=mx()) == BAD                              # not the transposed shape
    assert call(q=None, qt=mx(100, 64, 16)) == BAD           # its rows hold 32 bytes
    big = 1 << 30
    assert call(rows=big, cols=big, ld=big, q=mx(big, big, big)) == UNSUPPORTED
    assert call(x=None, rows=0, q=mx(0, 100, 0, None, None)) == OK and call(cols=0, q=mx(64, 0, 0, None, None)) == OK


def test_dequantize_refuses(lib):
    def call(q=mx(), out=P, ld=100, dtype=B.UQ_F32):
        return lib.uq_mx_dequantize(q, out, ld, dtype, None)
    assert call(q=None) == BAD and call(out=None) == BAD and call(ld=99) == BAD and call(dtype=7) == BAD and call(out=P + 2) == BAD
    assert call(q=mx(stride=40)) == BAD and call(q=mx(rows=-1)) == BAD
    assert call(q=mx(0, 100, 0, None, None), out=None) == OK


def test_product_refuses(lib):
    def call(a=mx(), b=mx(30), add=None, add_ld=0, out=P, ld=30, dtype=B.UQ_F32, status=None):
        return lib.uq_mx_product(a, b, add, add_ld, out, ld, dtype, status, None)
    assert call(a=None) == BAD and call(b=None) == BAD and call(b=mx(30, 99)) == BAD and call(out=None) == BAD
    assert call(ld=29) == BAD and call(dtype=3) == BAD and call(out=P + 1) == BAD and call(status=P + 1) == BAD
    assert call(add=P, add_ld=29) == BAD and call(add=P + 2, add_ld=30) == BAD
    assert call(a=mx(64, 0, 0), b=mx(30, 0, 0)) == BAD       # a sum over nothing
    assert call(a=mx(scales=None)) == BAD and call(b=mx(30, codes=P + 4)) == BAD
    big = 1 << 30
    assert call(a=mx(big), b=mx(big), ld=big) == UNSUPPORTED
    assert call(a=mx(0, 100, 0, None, None), out=None) == OK


def test_layer_norm_refuses(lib):
    F = C.c_float
    def call(x=P, rows=4, cols=100, ld=100, dtype=B.UQ_F32, gamma=P, beta=P, eps=1e-5, y=P, y_ld=100, mean=P, rstd=P, q=None, status=None):
        return lib.uq_layer_norm(x, rows, cols, ld, dtype, gamma, beta, F(eps), y, y_ld, mean, rstd, q, status, None)
    assert call(x=None) == BAD and call(ld=99) == BAD and call(y_ld=99) == BAD and call(dtype=9) == BAD and call(cols=0) == BAD
    assert call(eps=-1.0) == BAD and call(eps=float("nan")) == BAD
    assert call(gamma=P + 2) == BAD and call(beta=P + 2) == BAD and call(mean=P + 1) == BAD and call(rstd=P + 3) == BAD
    assert call(y=None, mean=None, rstd=None) == BAD         # nothing to write
    assert call(q=mx(5)) == BAD and call(q=mx(4, 100, 48)) == BAD and call(status=P + 1) == BAD
    assert call(x=None, rows=0, y=None) == OK


def test_layer_norm_backward_refuses(lib):
    def call(dy=P, dy_ld=100, x=P, x_ld=100, rows=4, cols=100, dtype=B.UQ_F32, gamma=P, mean=P, rstd=P, dx=P, dx_ld=100, dg=P, db=P,
             grad=B.UQ_F32, ws=P, n=1 << 20):
        return lib.uq_layer_norm_backward(dy, dy_ld, x, x_ld, rows, cols, dtype, gamma, mean, rstd, dx, dx_ld, dg, db, grad, ws, n, None)
    for kw in (dict(dy=None), dict(x=None), dict(dy_ld=99), dict(x_ld=99), dict(dx_ld=99), dict(cols=0), dict(dtype=4), dict(grad=4),
               dict(mean=None), dict(rstd=None), dict(gamma=P + 1), dict(dg=P + 2), dict(db=P + 2), dict(dx=P + 2),
               dict(dx=None, dg=None, db=None), dict(rows=-1)):
        assert call(**kw) == BAD, kw
    assert call(ws=None) == WS and call(n=64) == WS and call(ws=P + 4) == WS


def test_the_binding_refuses_shapes_and_types():
    f = torch.zeros
    with pytest.raises(ValueError, match="codes"):
        B.MxMatrix(4, 100, f(4, 63, dtype=torch.uint8), f(512, dtype=torch.uint8))
    with pytest.raises(ValueError, match="codes"):
        B.MxMatrix(4, 100, f(4, 64, dtype=torch.int8), f(512, dtype=torch.uint8))
    with pytest.raises(ValueError, match="scales"):
        B.MxMatrix(4, 100, f(4, 64, dtype=torch.uint8), f(511, dtype=torch.uint8))
    with pytest.raises(ValueError, match="negative"):
        B.MxMatrix(-1, 100)
    m = B.MxMatrix(4, 100, f(4, 64, dtype=torch.uint8), f(512, dtype=torch.uint8))
    wide = B.MxMatrix(4, 101, f(4, 64, dtype=torch.uint8), f(512, dtype=torch.uint8))
    with pytest.raises(ValueError, match="columns"):
        B.uq_mx_product(m, wide, f(4, 4))
    with pytest.raises(ValueError, match="out must be"):
        B.uq_mx_product(m, m, f(4, 5))
    with pytest.raises(ValueError, match="float32 or bfloat16|out must be"):
        B.uq_mx_dequantize(m, f(4, 100, dtype=torch.float16))
    with pytest.raises(ValueError, match="contiguous"):
        B.uq_mx_quantize(f(100, 4).t(), 0, 0, m, None)
    with pytest.raises(ValueError, match="CUDA"):
        B.uq_mx_quantize(f(4, 100), 0, 0, m, None)
    with pytest.raises(ValueError, match="must not overlap"):
        B.uq_layer_norm(f(1, 100).expand(4, 100), None, None, 1e-5, f(4, 100))
    with pytest.raises(ValueError, match="gamma|CUDA"):
        B.uq_layer_norm(f(4, 100), f(99), None, 1e-5, f(4, 100))


def test_the_layer_refuses():
    from paper_2109_12497_b200.layers import NormLinear
    with pytest.raises(ValueError, match="at least one"):
        NormLinear(0, 10, 10)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        NormLinear(1, 10, 10, torch.float16)
    layer = NormLinear(4, 10, 6, device="cpu")               # (its buffers alone; no call is made)
    assert layer.size == 2 * 10 + 60 and layer.segments() == [0, 10, 20, 80]
    x = torch.zeros(4, 10, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="no parameters"):
        layer.forward(x)
    with pytest.raises(ValueError, match="theta must be float32"):
        layer.load(torch.zeros(80, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match=">= 80"):
        layer.load(torch.zeros(79))
    layer.gamma = torch.ones(10)
    for rows in (0, 5):
        with pytest.raises(ValueError, match="1 to 4 rows"):
            layer.infer(torch.zeros(rows, 10, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="grad must be"):
        layer.backward(x, torch.zeros(4, 6, dtype=torch.bfloat16), torch.zeros(70), 0)
