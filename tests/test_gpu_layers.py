"""layers.NormLinear: the layer operators as they are used together, up to the quantized step that takes their gradients."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2109_12497_b200 import binding as B
from paper_2109_12497_b200.layers import NormLinear
from paper_2109_12497_b200.pipeline import Quantizer
from test_gpu_layer_norm import backward_bounds

pytestmark = pytest.mark.gpu


def make(tokens, d_in, d_out, dtype, seed):
    r = np.random.default_rng(seed)
    layer = NormLinear(tokens, d_in, d_out, dtype)
    theta = np.concatenate([1 + 0.2 * r.standard_normal(d_in), 0.2 * r.standard_normal(d_in),
                            r.standard_normal(d_out * d_in) / np.sqrt(d_in)]).astype(np.float32)
    x = torch.from_numpy(r.standard_normal((tokens, d_in)) + 0.3).to(dtype).cuda()
    dy = torch.from_numpy(r.standard_normal((tokens, d_out)) * 2.0 ** r.integers(-8, 0, (tokens, 1))).to(dtype).cuda()
    return layer, torch.from_numpy(theta).cuda(), x, dy


def fake(v, h=None):
    """v quantized along its rows, as values."""
    return ref.values(*ref.quantize(np.ascontiguousarray(v), None if h is None else np.ascontiguousarray(h)), v.shape[1])


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("tokens,d_in,d_out", [(1, 32, 16), (70, 100, 50), (129, 257, 300), (256, 1024, 512)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
def test_forward_and_backward_stage_by_stage(tokens, d_in, d_out, dtype, grad_dtype):
    """Each stage against its definition on what the stage before left in the layer's buffers (rounded values decide 4-bit
    codes, so an end-to-end comparison would test the luck of a border)."""
    u = 2.0 ** -24 if dtype is torch.float32 else 2.0 ** -8
    ug = 2.0 ** -24 if grad_dtype is torch.float32 else 2.0 ** -8
    layer, theta, x, dy = make(tokens, d_in, d_out, dtype, tokens)
    layer.load(theta)
    out = layer.forward(x)
    W = f64(theta[2 * d_in:]).reshape(d_out, d_in)
    y, w, wt = f64(layer.y), fake(W), fake(W.T)
    def close(got, a, b, unit):
        want, size = a @ b.T, np.abs(a) @ np.abs(b).T
        assert (np.abs(f64(got) - want) <= (a.shape[1] + 1) * 2.0 ** -23 * size + unit * np.abs(want) * 1.01 + 1e-30).all()
    close(out, fake(y), w, u)
    kept = out.clone()
    assert torch.equal(layer.infer(x), kept)                 # the same codes, the same product
    if tokens > 1:
        few = torch.empty(3 if tokens > 3 else 1, d_out, dtype=dtype, device="cuda")
        layer.infer(x[:few.shape[0]], few)
        close(few, fake(y[:few.shape[0]]), w, u)
    layer.forward(x)
    row = torch.full((layer.size + 5,), 7.0, dtype=grad_dtype, device="cuda")
    dx = layer.backward(x, dy, row[3:3 + layer.size], 77)
    h = ref.draws(tokens, d_out, 77)
    d = f64(dy)
    close(layer.dx_in, fake(d, h), wt, u)
    grads = row[3:3 + layer.size]
    close(grads[2 * d_in:].view(d_out, d_in), fake(d.T, h.T), fake(y.T), ug)
    g = f64(theta[:d_in])
    args = f64(layer.dx_in), f64(x), g, f64(layer.mean), f64(layer.rstd)
    want = ref.layer_norm_backward(*args)
    for got, ref_v, e, unit in zip((dx, grads[:d_in], grads[d_in:2 * d_in]), want, backward_bounds(*args, d_in, tokens), (u, ug, ug)):
        assert (np.abs(f64(got) - ref_v) <= e + unit * (np.abs(ref_v) + e)).all()
    assert (row[:3] == 7).all() and (row[-2:] == 7).all()
    assert layer.status_bits() == 0


def test_workers_gradients_through_the_quantized_step_to_the_update():
    """Four workers' rows filled by the layer, aggregated by the quantizer and applied: the average is within the quantizer's
    own bound of the rows' mean, and theta moves by it."""
    M, tokens, d_in, d_out = 4, 64, 96, 40
    layer, theta, _, _ = make(tokens, d_in, d_out, torch.bfloat16, 1)
    q = Quantizer(M, layer.size, torch.float32, seg_off=layer.segments(), s=127)
    g = torch.zeros(M, q.stride, device="cuda")
    before = theta.clone()
    momentum = torch.zeros_like(theta)
    for step in range(3):
        layer.load(theta)
        for m in range(M):
            _, _, x, dy = make(tokens, d_in, d_out, torch.bfloat16, 10 * step + m + 2)
            layer.forward(x)
            layer.backward(x, dy, g[m], seed=1000 * step + m)
        avg = q.step(g, seed=step)
        W = f64(q.W)
        mean = f64(g[:, :layer.size]).mean(0)
        bound = np.repeat(W / 127, np.diff(layer.segments())) * 1.001      # a level is off by less than one step of W / s
        assert (np.abs(f64(avg) - mean) <= bound + 1e-30).all() and np.abs(mean).max() > 0
        q.aggregate_decode_update(theta, momentum, lr=0.1, mu=0.9)
    assert q.status_bits() == 0 and layer.status_bits() == 0
    assert torch.isfinite(theta).all() and not torch.equal(theta, before)


def test_the_average_gradient_is_unbiased_over_seeds():
    """The weight's gradient over 400 seeds of the stochastic rounding against the one of the unrounded dy: each element is a sum
    over the tokens of independent two-point variables, its standard error taken from the sample."""
    tokens, d_in, d_out, n = 64, 32, 24, 400
    layer, theta, x, dy = make(tokens, d_in, d_out, torch.float32, 5)
    layer.load(theta)
    layer.forward(x)
    got = torch.empty(n, layer.size, device="cuda")
    for k in range(n):
        layer.backward(x, dy, got[k], 7919 * k + 1)
    w = f64(got[:, 2 * d_in:]).reshape(n, d_out, d_in)
    want = f64(dy).T @ fake(f64(layer.y).T).T
    err = w.std(0, ddof=1) / np.sqrt(n)
    assert (np.abs(w.mean(0) - want) <= 6 * err + 1e-5 * np.abs(want).max()).all()


def test_captured_and_replayed_beside_eager_calls():
    layer, theta, x, dy = make(100, 128, 64, torch.bfloat16, 9)
    grad = torch.empty(layer.size, device="cuda")
    def step():
        layer.load(theta)
        layer.forward(x)
        layer.backward(x, dy, grad, 3)
    step()
    torch.cuda.synchronize()
    want = [grad.clone(), layer.dx.clone(), layer.out.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        for t in (grad, layer.dx, layer.out):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((grad, layer.dx, layer.out), want))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((grad, layer.dx, layer.out), want))


def test_non_finite_gradients_are_reported():
    layer, theta, x, dy = make(40, 64, 64, torch.bfloat16, 2)
    layer.load(theta)
    layer.forward(x)
    dy[3, 5] = float("nan")
    grad = torch.zeros(layer.size, device="cuda")
    layer.backward(x, dy, grad, 1)
    assert layer.status_bits() == B.UQ_STATUS_NONFINITE
    assert torch.isnan(grad[2 * 64:].view(64, 64)[5]).all()  # the row of the output that it belongs to
    assert torch.isfinite(grad[2 * 64:].view(64, 64)[:5]).all()
