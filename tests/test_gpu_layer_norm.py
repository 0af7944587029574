"""Layer norm, forward and backward, against 64-bit definitions."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2109_12497_b200 import binding as B
from test_gpu_mx import DT, as_matrix, check_mx, empty_mx, status

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}                   # one rounding to the type
EPS = 1e-5
SIZES = [(1, 1), (1, 7), (2, 32), (3, 33), (5, 255), (4, 256), (7, 1000), (3, 1025), (2, 2048), (300, 100), (5, 5001), (2, 8200),
         (3, 16384), (2, 40003), (1000, 24), (9, 8201), (700, 9000), (5, 16383), (330, 12280)]


def inputs(rows, cols, seed):
    r = np.random.default_rng(seed)
    x = r.standard_normal((rows, cols)) * 2.0 ** r.integers(-4, 5, (rows, 1)) + r.standard_normal((rows, 1))
    gamma = (1 + 0.5 * r.standard_normal(cols)).astype(np.float32)
    beta = r.standard_normal(cols).astype(np.float32)
    dy = r.standard_normal((rows, cols)) * 2.0 ** r.integers(-6, 3, (rows, 1))
    return x, gamma, beta, dy


def f64(t):
    return t.double().cpu().numpy()


def cuda(v):
    return None if v is None else torch.from_numpy(v).cuda()


def forward_bounds(x, gamma, beta, mean, rstd, cols):
    """How far binary32 may be off, in units of u = 2^-24.  A value goes through at most L = cols / 256 + 53 additions: a chain
    in its thread (32 values, or cols / 256 where rows are longer than a CTA holds), 5 levels in the warp, 16 warps:
      mean:  L u mean|x|, and 2 u |mean| for 1 / cols and the product with it
      var:   each square's factor is off by u |x - mean| + |error of the mean|; the sum and the product L + 4 more
      rstd:  half the relative error of var, u for adding eps, 3 u for the root (an approximation of 2 units in the last place,
             4 u, whose square, 24 u^2, is left by a Newton step of three roundings)
      y:     |x - mean| rstd (rel. error of rstd + 4 u) + rstd |error of the mean|, times gamma, and u for each result."""
    u, L = 2.0 ** -24, cols / 256 + 53
    e_mean = L * u * np.abs(x).mean(1) + 2 * u * np.abs(mean)
    c = np.abs(x - mean[:, None])
    var = (c ** 2).mean(1)
    e_var = 2 * (c * (u * c + e_mean[:, None])).mean(1) + e_mean ** 2 + (L + 4) * u * var
    rel = 0.5 * e_var * rstd ** 2 * 1.01 + 4 * u
    e_rstd = rstd * rel
    g = 1.0 if gamma is None else np.abs(gamma)
    e_y = (c * rstd[:, None] * (rel[:, None] + 4 * u) + rstd[:, None] * e_mean[:, None]) * g * 1.01
    e_y = e_y + (0.0 if beta is None else u * (np.abs(beta) + c * rstd[:, None] * g))
    return e_mean, e_rstd, e_y


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(rows, cols, dtype):
    x, gamma, beta, _ = inputs(rows, cols, rows + cols)
    for pad, offset, with_g, with_b in ((0, 0, True, True), (3, 1, True, False), (8, 8, False, True), (0, 0, False, False)):
        g, b = gamma if with_g else None, beta if with_b else None
        t = as_matrix(x, DT[dtype], pad, offset)
        xs = t.double().cpu().numpy()
        y = as_matrix(np.zeros((rows, cols)), DT[dtype], pad, offset)
        whole = y.as_strided((rows, cols + pad), (cols + pad, 1))
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        B.uq_layer_norm(t, cuda(g), cuda(b), EPS, y, mean, rstd)
        want, wm, wr = ref.layer_norm(xs, g, b, EPS)
        em, er, ey = forward_bounds(xs, g, b, wm, wr, cols)
        assert (np.abs(mean.double().cpu().numpy() - wm) <= em).all()
        assert (np.abs(rstd.double().cpu().numpy() - wr) <= er).all()
        ey = ey + U[dtype] * (np.abs(want) + ey)
        assert (np.abs(y.double().cpu().numpy() - want) <= ey).all()
        assert torch.isnan(whole[:, cols:]).all()


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantized_on_the_way_out_is_the_result_quantized(rows, cols, dtype):
    x, gamma, beta, _ = inputs(rows, cols, rows * 3 + cols)
    t = as_matrix(x, DT[dtype], 1, 1)
    y, q, q2, st = torch.empty(rows, cols, dtype=DT[dtype], device="cuda"), empty_mx(rows, cols, 16), empty_mx(rows, cols, 16), status()
    B.uq_layer_norm(t, cuda(gamma), cuda(beta), EPS, y, None, None, q, st)
    check_mx(q, y.double().cpu().numpy(), None)
    B.uq_layer_norm(t, cuda(gamma), cuda(beta), EPS, None, None, None, q2, st)       # without the result itself
    check_mx(q2, y.double().cpu().numpy(), None)
    assert int(st.item()) == 0


def test_forward_special_rows():
    """Constant rows (variance 0), rows of one value, a large mean, and NaN or infinity, which stay in their row."""
    cols = 300
    x = np.random.default_rng(0).standard_normal((6, cols))
    x[0], x[1], x[2] = 0.0, 3.0, x[2] + 1000
    x[4, 7], x[5, 299] = np.nan, np.inf
    t = as_matrix(x, torch.float32)
    y, mean, rstd, q, st = torch.empty(6, cols, device="cuda"), torch.empty(6, device="cuda"), torch.empty(6, device="cuda"), empty_mx(6, cols), status()
    B.uq_layer_norm(t, None, None, EPS, y, mean, rstd, q, st)
    y = y.double().cpu().numpy()
    assert (y[0] == 0).all() and (np.abs(y[1]) <= 3 * 2.0 ** -22 / EPS ** 0.5).all()
    assert abs(float(rstd[0]) - EPS ** -0.5) <= 2.0 ** -22 * EPS ** -0.5
    xs = t.double().cpu().numpy()
    want, wm, wr = ref.layer_norm(xs[2:4], None, None, EPS)
    assert (np.abs(y[2:4] - want) <= forward_bounds(xs[2:4], None, None, wm, wr, cols)[2] + 2.0 ** -24 * np.abs(want)).all()
    assert np.isnan(y[4]).all() and np.isnan(y[5]).all() and np.isfinite(y[:4]).all()
    assert int(st.item()) == B.UQ_STATUS_NONFINITE
    _, scales, _ = ref.unpack(q.codes.cpu().numpy(), q.scales.cpu().numpy(), 6, cols)
    assert (scales[4:] == 255).all() and (scales[:4] != 255).all()


def backward_bounds(dy, x, gamma, mean, rstd, cols, rows):
    """Binary32, u = 2^-24, chains as in the forward pass (L additions per sum over a row; a sum over the rows is a chain of
    at most R = rows additions):
      xh: 2 u relative to |x - mean| rstd, and u |x| rstd for the difference;  t: u relative
      the two means: (L + 4) u of the mean of magnitudes, with xh's error in the second
      dx: rstd (u-errors of its three terms);  dgamma: sum |dy| (error of xh + u |xh|) + R u sum |dy xh|;  dbeta: R u sum |dy|."""
    u, L = 2.0 ** -24, cols / 256 + 53
    c = np.abs(x - mean[:, None])
    xh = c * rstd[:, None]
    e_xh = 3 * u * xh
    t = np.abs(dy if gamma is None else dy * gamma)
    m1, m2 = t.mean(1, keepdims=True), (t * xh).mean(1, keepdims=True)
    e1 = (L + 4) * u * m1
    e2 = (L + 6) * u * m2 + (t * e_xh).mean(1, keepdims=True)
    e_dx = rstd[:, None] * (4 * u * (t + m1 + xh * m2) + e1 + xh * e2 + e_xh * m2) * 1.01
    a = np.abs(dy)
    e_g = ((a * (e_xh + u * xh)).sum(0) + (rows + 2) * u * (a * xh).sum(0)) * 1.01
    return e_dx, e_g, (rows + 2) * u * a.sum(0)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(rows, cols, dtype):
    x, gamma, beta, dy = inputs(rows, cols, rows * 5 + cols)
    for pad, offset, with_g, grad in ((0, 0, True, "f32"), (3, 1, True, "bf16"), (8, 8, False, "f32")):
        g = gamma if with_g else None
        t, d = as_matrix(x, DT[dtype], pad, offset), as_matrix(dy, DT[dtype], pad + 1, offset)
        xs, ds = t.double().cpu().numpy(), d.double().cpu().numpy()
        mean, rstd = (v.astype(np.float32) for v in ref.layer_norm(xs, g, None, EPS)[1:])
        dx = as_matrix(np.zeros((rows, cols)), DT[dtype], pad, offset)
        row = torch.full((2 * cols + 2,), 9.0, dtype=DT[grad], device="cuda")        # a piece of a worker's row, oddly placed
        dg, db = row[1:1 + cols], row[1 + cols:1 + 2 * cols]
        ws = torch.full((B.uq_layer_norm_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
        B.uq_layer_norm_backward(d, t, cuda(g), cuda(mean), cuda(rstd), dx, dg, db, ws)
        m64, r64 = mean.astype(np.float64), rstd.astype(np.float64)
        wx, wg, wb = ref.layer_norm_backward(ds, xs, g, m64, r64)
        ex, eg, eb = backward_bounds(ds, xs, g, m64, r64, cols, rows)
        for got, want, e, kind in ((dx, wx, ex, dtype), (dg, wg, eg, grad), (db, wb, eb, grad)):
            assert (np.abs(got.double().cpu().numpy() - want) <= e + U[kind] * (np.abs(want) + e)).all()
        assert float(row[0]) == 9.0 and float(row[-1]) == 9.0
        for parts in ((None, dg, db), (dx, None, None), (dx, dg, None), (None, None, db)):   # any of the three alone: the same values
            before = [None if p is None else p.clone() for p in parts]
            for p in parts:
                if p is not None:
                    p.fill_(3.0)
            B.uq_layer_norm_backward(d, t, cuda(g), cuda(mean), cuda(rstd), *parts, ws)
            for p, w in zip(parts, before):
                assert p is None or torch.equal(p, w)


def test_gradient_against_differences():
    """sum(w * y) differentiated numerically in 64 bits: the gradients that backward gives for dy = w."""
    rows, cols = 3, 40
    x, gamma, beta, w = inputs(rows, cols, 1)
    f = lambda a, g, b: float((w * ref.layer_norm(a, g, b, EPS)[0]).sum())
    t, d = as_matrix(x, torch.float32), as_matrix(w, torch.float32)
    x, w = t.double().cpu().numpy(), d.double().cpu().numpy()
    g64, b64 = gamma.astype(np.float64), beta.astype(np.float64)
    y, mean, rstd = torch.empty(rows, cols, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.uq_layer_norm(t, cuda(gamma), cuda(beta), EPS, y, mean, rstd)
    dx, dg, db = torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(B.uq_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.uq_layer_norm_backward(d, t, cuda(gamma), mean, rstd, dx, dg, db, ws)
    h = 1e-5

    def numeric(at, k):
        v = at.copy()
        v.reshape(-1)[k] += h
        hi = v.copy()
        v.reshape(-1)[k] -= 2 * h
        return hi, v
    # the difference quotient is off by h^2 f''' / 6 and by rounding of sums of size ~100 over 2 h: below 1e-5 with these inputs
    for k in range(0, rows * cols, 7):
        hi, lo = numeric(x, k)
        assert abs((f(hi, g64, b64) - f(lo, g64, b64)) / (2 * h) - float(dx.reshape(-1)[k])) <= 1e-4
    for k in range(0, cols, 3):
        hi, lo = numeric(g64, k)
        assert abs((f(x, hi, b64) - f(x, lo, b64)) / (2 * h) - float(dg[k])) <= 1e-4
        hi, lo = numeric(b64, k)
        assert abs((f(x, g64, hi) - f(x, g64, lo)) / (2 * h) - float(db[k])) <= 1e-4


def test_no_rows():
    x = torch.empty(0, 50, device="cuda")
    e = torch.empty(0, device="cuda")
    dg, db = torch.full((50,), 5.0, device="cuda"), torch.full((50,), 5.0, device="cuda")
    B.uq_layer_norm(x, None, None, EPS, torch.empty(0, 50, device="cuda"), e, e)
    B.uq_layer_norm_backward(x, x, None, e, e, None, dg, db, torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert not dg.any() and not db.any()                     # a sum over no rows


def test_in_graphs_that_share_a_workspace_and_on_streams():
    rows, cols = 200, 1000
    ws = torch.empty(B.uq_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    sets = []
    for k in range(2):
        x, gamma, _, dy = inputs(rows, cols, k)
        t, d, g = as_matrix(x, torch.bfloat16), as_matrix(dy, torch.bfloat16), cuda(gamma)
        mean, rstd, dx = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(d)
        y, dg, db = torch.empty_like(d), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")

        def step(t=t, d=d, g=g, mean=mean, rstd=rstd, dx=dx, y=y, dg=dg, db=db):
            B.uq_layer_norm(t, g, None, EPS, y, mean, rstd)
            B.uq_layer_norm_backward(d, t, g, mean, rstd, dx, dg, db, ws)
        step()
        torch.cuda.synchronize()
        want = [v.clone() for v in (y, dx, dg, db)]
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        sets.append((graph, (y, dx, dg, db), want, step))     # (the step holds the buffers that the graph reads)
    for _ in range(2):
        for graph, got, want, _ in sets:
            for v in got:
                v.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_offsets_beyond_32_bits():
    """More than 2^31 elements: the last rows are those of the same rows by themselves, and the sums over the rows are whole."""
    rows, cols = 262_200, 8_192
    x = torch.full((rows, cols), 0.5, dtype=torch.bfloat16, device="cuda")
    x[:, ::2] = -0.25
    x[-4:] = torch.randn(4, cols, device="cuda").bfloat16()
    gamma, beta = torch.rand(cols, device="cuda") + 0.5, torch.randn(cols, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.uq_layer_norm(x, gamma, beta, EPS, y, mean, rstd)
    small = torch.empty(4, cols, dtype=torch.bfloat16, device="cuda")
    B.uq_layer_norm(x[-4:], gamma, beta, EPS, small)
    assert torch.equal(y[-4:], small)
    dy = torch.ones_like(x)
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(B.uq_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.uq_layer_norm_backward(dy, x, gamma, mean, rstd, y, dg, db, ws)
    assert (db == rows).all()                                # sums of ones below 2^24: exact
    one = torch.empty(4, cols, dtype=torch.bfloat16, device="cuda")
    B.uq_layer_norm_backward(dy[-4:], x[-4:], gamma, mean[-4:], rstd[-4:], one, None, None, ws)
    assert torch.equal(y[-4:], one)


@pytest.mark.parametrize("rows,cols", [(300, 2500), (60, 9001)])
def test_two_backward_passes_at_once(rows, cols):
    """Two streams, a workspace each; rows by a CTA and by a cluster of two."""
    runs = []
    for k in range(2):
        x, gamma, _, dy = inputs(rows, cols, 20 + k)
        t, d, g = as_matrix(x, torch.float32, 1, 1), as_matrix(dy, torch.float32), cuda(gamma)
        mean, rstd = (cuda(v.astype(np.float32)) for v in ref.layer_norm(f64(t), None, None, EPS)[1:])
        outs = [torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")]
        ws = torch.empty(B.uq_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        B.uq_layer_norm_backward(d, t, g, mean, rstd, *outs, ws)
        runs.append((d, t, g, mean, rstd, outs, ws, [o.clone() for o in outs], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for d, t, g, mean, rstd, outs, ws, _, stream in runs:
            with torch.cuda.stream(stream):
                B.uq_layer_norm_backward(d, t, g, mean, rstd, *outs, ws)
    torch.cuda.synchronize()
    for *_, outs, _, want, _ in runs:
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
