"""The layer operators as measurable cases: microscaled 4-bit quantisation and product, layer norm.

A microscaled matrix holds 4-bit E2M1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two per byte, the even
column in the low half, and one power of two (E8M0) for each block of 32 columns of a row.  Rows of codes are
16 * ceil(cols / 32) bytes; the scales lie in tiles of 128 rows x 4 blocks, row r and block b of a tile at byte
(r % 32) * 16 + (r // 32) * 4 + b, the tiles of a strip of 128 rows one after the other.

  quantize        a matrix to 4 bits with blocks along its rows, along its columns, or both, to the nearest value or
                  stochastically; then the values that the codes stand for
  product         D = A B^T (+ add) of two microscaled matrices
  norm            layer norm's forward pass with its statistics
  norm_backward   its backward pass: dx, dgamma, dbeta
  serve           one layer for new tokens: layer norm, quantised on the way out, then the product with kept weights
  train           one layer's backward pass: the gradient quantised stochastically both ways, the products for the
                  input's and the weight's gradient, layer norm's backward pass

Ranges: 1 to 16384 rows, 64 to 16384 columns, odd ones among them; binary32 and bfloat16; padded rows.
"""
import math

import torch

own = False

EPS = 1e-5
TAG = 0x4D584634
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _quantize(rows, cols, dtype, rounding, along, pad=0, name=None):
    c = dict(kind="quantize", rows=rows, cols=cols, dtype=dtype, rounding=rounding, along=along, pad=pad)
    return dict(c, name=name) if name else c


def _product(m, n, k, dtype, add=False, name=None):
    c = dict(kind="product", m=m, n=n, k=k, dtype=dtype, add=add)
    return dict(c, name=name) if name else c


def _norm(kind, rows, cols, dtype, pad=0, name=None):
    c = dict(kind=kind, rows=rows, cols=cols, dtype=dtype, pad=pad)
    return dict(c, name=name) if name else c


def _layer(kind, rows, cols, n, dtype, name=None):
    c = dict(kind=kind, rows=rows, cols=cols, n=n, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a few new tokens' activations in front of a product: latency
        _quantize(4, 4096, "bf16", "nearest", "rows", name="quantize_tokens"),
        # a binary32 gradient of odd sizes in padded rows, for both products of its backward pass
        _quantize(1023, 2037, "f32", "stochastic", "both", 3, name="quantize_odd"),
        # a large batch's gradient for both products of its backward pass
        _quantize(16384, 8192, "bf16", "stochastic", "both", name="quantize_gradient"),
        # one token against a layer's weights: every weight is read for one row
        _product(1, 8192, 4096, "bf16", name="product_token"),
        # a ragged batch of tokens in decoding
        _product(37, 10000, 5010, "bf16", name="product_batch"),
        # a prompt, or a training batch's forward pass
        _product(8192, 8192, 8192, "bf16", name="product_prompt"),
        # a weight's gradient over a batch of tokens, added to that of the batch before
        _product(4000, 4096, 16384, "f32", True, name="product_gradient"),
        # a few tokens' layer norm: latency
        _norm("norm", 3, 4096, "bf16", name="norm_tokens"),
        # layer norm over a training batch
        _norm("norm", 16384, 8192, "bf16", name="norm_batch"),
        # backward of a small layer of odd size
        _norm("norm_backward", 777, 1025, "f32", 2, name="norm_backward_odd"),
        # one layer for sixteen new tokens
        _layer("serve", 16, 4096, 8192, "bf16", name="serve_layer"),
        # one layer's backward pass in training
        _layer("train", 8192, 4096, 8192, "bf16", name="train_layer"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quantize", "quantize", "product", "product", "norm", "norm_backward", "serve", "train"])
    dtype = rng.choice(["f32", "bf16"])
    pad = rng.choice([0, 0, 1, 8])
    if kind == "quantize":
        return _quantize(_log(rng, 1, 8192), _log(rng, 64, 8192), dtype, rng.choice(["nearest", "stochastic"]),
                         rng.choice(["rows", "cols", "both"]), pad)
    if kind == "product":
        return _product(_log(rng, 1, 8192), _log(rng, 64, 8192), _log(rng, 64, 8192), dtype, rng.random() < 0.3)
    if kind in ("norm", "norm_backward"):
        return _norm(kind, _log(rng, 1, 8192), _log(rng, 64, 16384), dtype, pad)
    if kind == "serve":
        return _layer(kind, _log(rng, 1, 64), _log(rng, 64, 8192), _log(rng, 64, 8192), dtype)
    return _layer(kind, _log(rng, 64, 8192), _log(rng, 64, 4096), _log(rng, 64, 8192), dtype)


# ---- elementary forms ---------------------------------------------------------------------------------------------

def _draws(seed, rows, cols, device):
    """The 16-bit random numbers of a matrix's elements: Philox4x32-10 (Salmon et al. 2011) with the seed as its key and
    (column / 8, row, 0, a tag) as its counter; column c takes word (c % 8) / 2, even columns the low half."""
    mask = 0xFFFFFFFF
    c0 = torch.arange(-(-cols // 8), device=device, dtype=torch.int64).expand(rows, -1)
    c1 = torch.arange(rows, device=device, dtype=torch.int64)[:, None].expand_as(c0)
    c2, c3 = torch.zeros_like(c0), torch.full_like(c0, TAG)
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57            # the low 64 bits; the sign is shifted and masked away
        c0, c1, c2, c3 = ((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    w = torch.stack([c0, c1, c2, c3], -1)
    return torch.stack([w & 0xFFFF, w >> 16], -1).reshape(rows, -1)[:, :cols].int()


def _pow2(e):
    """2^e in binary32, -127 <= e <= 127."""
    return torch.where(e < -126, torch.full_like(e, 1 << 22), (e + 127) << 23).int().view(torch.float32)


def _plain_blocks(x, h):
    """Blocks of 32 along the rows of x: codes' magnitudes and signs as values / 2^e [rows, nb, 32], and e [rows, nb]."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    x = torch.nn.functional.pad(x.float(), (0, nb * 32 - cols)).view(rows, nb, 32)
    m, ex = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0, ex - 3 + (m > 0.75).int(), torch.full_like(ex, -127)).clamp(min=-127)
    a = x.abs() * _pow2(-e)[..., None]
    if h is None:
        v = 0.5 * ((a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float())
        v = v + (a > 2.5).float() + (a >= 3.5).float() + 2.0 * (a > 5.0).float()
    else:
        h = torch.nn.functional.pad(h, (0, nb * 32 - cols)).view(rows, nb, 32)
        u = 0.5 + 0.5 * (a >= 2).float() + (a >= 4).float()
        t = a / u
        lo = t.floor()
        v = (lo + (h < ((t - lo) * 65536.0).round()).float()) * u
    return torch.copysign(v, x), e


def _plain_quantize(x, h):
    """The values that the quantised matrix stands for, blocks along the rows."""
    v, e = _plain_blocks(x, h)
    return (v * _pow2(e)[..., None]).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _pack(x, h=None):
    """Codes and scales of x in the layout above."""
    v, e = _plain_blocks(x, h)
    rows, nb = e.shape
    a = v.abs()
    code = (a * 2 - (a > 2).float() * (a - 2) - (a > 4).float() * (a - 4) * 0.5).round().to(torch.uint8)
    code = (code + 8 * torch.signbit(v).to(torch.uint8)).view(rows, nb * 16, 2)
    codes = (code[..., 0] + (code[..., 1] << 4)).contiguous()
    rt, kt = -(-rows // 128), -(-nb // 4)
    s = torch.zeros(rt * 128, kt * 4, dtype=torch.uint8, device=x.device)
    s[:rows, :nb] = (e + 127).to(torch.uint8)
    return codes, s.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _unpack(codes, scales, rows, cols):
    """The binary32 values of codes and scales in the layout above."""
    rt, kt = -(-rows // 128), -(-cols // 128)
    s = scales.view(rt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, kt * 4)[:rows, :-(-cols // 32)]
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    v = grid[torch.stack([codes & 15, codes >> 4], -1).int()].view(rows, -1, 32)
    return (v * _pow2(s.int() - 127)[..., None]).view(rows, -1)[:, :cols]


def _plain_norm(x, gamma, beta):
    x = x.float()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / (c.square().mean(1) + EPS).sqrt()
    return c * rstd[:, None] * gamma + beta, mean, rstd


def _plain_norm_backward(dy, x, gamma, mean, rstd):
    dy, xh = dy.float(), (x.float() - mean[:, None]) * rstd[:, None]
    t = dy * gamma
    dx = rstd[:, None] * (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


# ---- the cases ----------------------------------------------------------------------------------------------------

def _padded(values, pad):
    """values in rows that are `pad` elements longer."""
    rows, cols = values.shape
    buf = torch.zeros(rows, cols + pad, dtype=values.dtype, device=values.device)
    buf[:, :cols] = values
    return buf[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dev, dt = "cuda", DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    def gradient(rows, cols):
        # a gradient's rows differ in size by orders of magnitude
        return normal(rows, cols) * torch.exp2(-8 + 2 * normal(rows, 1))

    def activations(rows, cols):
        # a few columns are much larger than the others
        return normal(rows, cols) * (1 + 9 * (torch.rand(cols, generator=g, device=dev) < 0.01).float()) + 0.1

    def weights(rows, cols):
        return normal(rows, cols) / math.sqrt(cols)

    def affine(cols):
        return 1 + 0.1 * normal(cols), 0.1 * normal(cols)

    def packed(rows, cols):
        codes = torch.empty(rows, 16 * -(-cols // 32), dtype=torch.uint8, device=dev)
        return codes, torch.empty(-(-rows // 128) * -(-cols // 128) * 512, dtype=torch.uint8, device=dev)

    def empty(*shape, dtype=None):
        return torch.empty(*shape, dtype=dtype or dt, device=dev)

    s = dict(case, seed=int(seed) * 1_000_003 + 12345, status=torch.zeros(1, dtype=torch.int32, device=dev), kept={})
    k = case["kind"]
    if k == "quantize":
        r, c = case["rows"], case["cols"]
        make = gradient if case["rounding"] == "stochastic" else activations
        s["x"] = _padded(make(r, c).to(dt), case["pad"])
        if case["along"] != "cols":
            s["q"], s["values"] = packed(r, c), empty(r, c)
        if case["along"] != "rows":
            s["qt"], s["values_t"] = packed(c, r), empty(c, r)
    elif k == "product":
        s["a"], s["b"] = _pack(activations(case["m"], case["k"])), _pack(weights(case["n"], case["k"]))
        s["out"] = empty(case["m"], case["n"])
        s["add"] = normal(case["m"], case["n"]).to(dt) if case["add"] else None
    elif k in ("norm", "norm_backward"):
        r, c = case["rows"], case["cols"]
        s["x"] = _padded(activations(r, c).to(dt), case["pad"])
        s["gamma"], s["beta"] = affine(c)
        if k == "norm":
            s["y"], s["mean"], s["rstd"] = empty(r, c), empty(r, dtype=torch.float32), empty(r, dtype=torch.float32)
        else:
            s["dy"] = _padded(gradient(r, c).to(dt), case["pad"])
            _, s["mean"], s["rstd"] = _plain_norm(s["x"], s["gamma"], s["beta"])
            s["dx"], s["dgamma"], s["dbeta"] = empty(r, c), empty(c, dtype=torch.float32), empty(c, dtype=torch.float32)
    elif k == "serve":
        r, c, n = case["rows"], case["cols"], case["n"]
        s["x"], (s["gamma"], s["beta"]) = activations(r, c).to(dt), affine(c)
        s["w"], s["q"], s["out"] = _pack(weights(n, c)), packed(r, c), empty(r, n)
    else:
        r, c, n = case["rows"], case["cols"], case["n"]
        s["x"], (s["gamma"], s["beta"]) = activations(r, c).to(dt), affine(c)
        y, s["mean"], s["rstd"] = _plain_norm(s["x"], s["gamma"], s["beta"])
        s["yt"], s["wt"] = _pack(y.t().contiguous()), _pack(weights(n, c).t().contiguous())
        s["dy"] = gradient(r, n).to(dt)
        s["q"], s["qt"] = packed(r, n), packed(n, r)
        s["dx_in"], s["dx"], s["dw"] = empty(r, c), empty(r, c), empty(n, c, dtype=torch.float32)
        s["dgamma"], s["dbeta"] = empty(c, dtype=torch.float32), empty(c, dtype=torch.float32)
    return s


def _kept(s, name, rows, cols):
    """The handle of one of the state's microscaled matrices, as a program keeps it beside the buffers."""
    h = s["kept"].get(name)
    if h is None:
        from paper_2109_12497_b200 import binding as B
        h = s["kept"][name] = B.MxMatrix(rows, cols, *s[name])
    return h


def _scratch(s, rows, cols):
    """Layer norm's workspace for its backward pass, which a program keeps too."""
    w = s["kept"].get("workspace")
    if w is None:
        from paper_2109_12497_b200 import binding as B
        w = s["kept"]["workspace"] = torch.empty(B.uq_layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    return w


def run(s):
    k, dt = s["kind"], DTYPES[s["dtype"]]
    if own:
        from paper_2109_12497_b200 import binding as B
    if k == "quantize":
        r, c, bits = s["rows"], s["cols"], 16 if s["rounding"] == "stochastic" else 0
        along_rows, along_cols = s["along"] != "cols", s["along"] != "rows"
        if own:
            q = _kept(s, "q", r, c) if along_rows else None
            qt = _kept(s, "qt", c, r) if along_cols else None
            B.uq_mx_quantize(s["x"], s["seed"], bits, q, qt, s["status"])
            if along_rows:
                B.uq_mx_dequantize(q, s["values"])
            if along_cols:
                B.uq_mx_dequantize(qt, s["values_t"])
            return [s[name] for name in ("values", "values_t") if name in s]
        h = _draws(s["seed"], r, c, s["x"].device) if bits else None
        out = [_plain_quantize(s["x"], h).to(dt)] if along_rows else []
        if along_cols:
            out.append(_plain_quantize(s["x"].t(), None if h is None else h.t()).to(dt))
        return out
    if k == "product":
        m, n, kk = s["m"], s["n"], s["k"]
        if own:
            B.uq_mx_product(_kept(s, "a", m, kk), _kept(s, "b", n, kk), s["out"], s["add"], s["status"])
            return s["out"]
        d = _unpack(*s["a"], m, kk) @ _unpack(*s["b"], n, kk).t()
        return (d if s["add"] is None else d + s["add"].float()).to(dt)
    if k == "norm":
        if own:
            B.uq_layer_norm(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"])
            return s["y"], s["mean"], s["rstd"]
        y, mean, rstd = _plain_norm(s["x"], s["gamma"], s["beta"])
        return y.to(dt), mean, rstd
    if k == "norm_backward":
        if own:
            B.uq_layer_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"],
                                     _scratch(s, s["rows"], s["cols"]))
            return s["dx"], s["dgamma"], s["dbeta"]
        dx, dgamma, dbeta = _plain_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"])
        return dx.to(dt), dgamma, dbeta
    r, c, n = s["rows"], s["cols"], s["n"]
    if k == "serve":
        if own:
            q = _kept(s, "q", r, c)
            B.uq_layer_norm(s["x"], s["gamma"], s["beta"], EPS, None, None, None, q, s["status"])
            B.uq_mx_product(q, _kept(s, "w", n, c), s["out"], None, s["status"])
            return s["out"]
        y = _plain_norm(s["x"], s["gamma"], s["beta"])[0].to(dt)
        return (_plain_quantize(y, None) @ _unpack(*s["w"], n, c).t()).to(dt)
    if own:
        q, qt = _kept(s, "q", r, n), _kept(s, "qt", n, r)
        B.uq_mx_quantize(s["dy"], s["seed"], 16, q, qt, s["status"])
        B.uq_mx_product(q, _kept(s, "wt", c, n), s["dx_in"], None, s["status"])
        B.uq_mx_product(qt, _kept(s, "yt", c, r), s["dw"], None, s["status"])
        B.uq_layer_norm_backward(s["dx_in"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"],
                                 _scratch(s, r, c))
        return s["dx"], s["dw"], s["dgamma"], s["dbeta"]
    h = _draws(s["seed"], r, n, s["dy"].device)
    dy, dyt = _plain_quantize(s["dy"], h), _plain_quantize(s["dy"].t(), h.t())
    dx_in = (dy @ _unpack(*s["wt"], c, n).t()).to(dt)
    dw = dyt @ _unpack(*s["yt"], c, r).t()
    dx, dgamma, dbeta = _plain_norm_backward(dx_in, s["x"], s["gamma"], s["mean"], s["rstd"])
    return dx.to(dt), dw, dgamma, dbeta


def work(case):
    k, e = case["kind"], BYTES[case["dtype"]]
    q = 0.5 + 1 / 32                                          # a microscaled value
    if k == "quantize":
        n = case["rows"] * case["cols"]
        ways = 2 if case["along"] == "both" else 1
        return {"bytes": n * (e + ways * (2 * q + e)), "flops": n * 8 * ways}
    if k == "product":
        m, n, kk = case["m"], case["n"], case["k"]
        return {"bytes": q * kk * (m + n) + e * m * n * (1 + case["add"]), "flops": 2 * m * n * kk}
    r, c = case["rows"], case["cols"]
    if k == "norm":
        return {"bytes": 2 * e * r * c + 8 * (r + c), "flops": 8 * r * c}
    if k == "norm_backward":
        return {"bytes": 3 * e * r * c + 8 * r + 12 * c, "flops": 14 * r * c}
    n = case["n"]
    if k == "serve":
        return {"bytes": e * r * c + 8 * c + 2 * q * r * c + q * n * c + e * r * n, "flops": 2 * r * n * c + 16 * r * c}
    # dy once, its codes written and read; the two other operands; dw, the input's gradient written and read, x, dx
    return {"bytes": e * r * n + 4 * q * r * n + q * c * (n + r) + 4 * n * c + 4 * e * r * c,
            "flops": 4 * r * n * c + 16 * r * n + 14 * r * c}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_quantize(x, h):
    """Neighbours of |x| / 2^e on the grid by a search, and the choice between them, in binary64."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    full = torch.zeros(rows, nb * 32, dtype=torch.float64, device=x.device)
    full[:, :cols] = x
    b = full.view(-1, 32)
    top = b.abs().max(1).values
    e = torch.ceil(torch.log2(top / 6.0)).clamp(min=-127)
    e = e + (6.0 * torch.exp2(e) < top)
    e = torch.where(6.0 * torch.exp2(e - 1) >= top, e - 1, e).clamp(min=-127)
    unit = torch.exp2(e)[:, None]
    a = b.abs() / unit
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    i = (torch.searchsorted(grid, a, right=True) - 1).clamp(max=6)
    below, above = grid[i], grid[i + 1]
    p = (a - below) / (above - below)
    if h is None:
        up = (p > 0.5) | ((p == 0.5) & (i % 2 == 1))
    else:
        k = torch.zeros(rows, nb * 32, dtype=torch.float64, device=x.device)
        k[:, :cols] = h
        up = k.view(-1, 32) < torch.round(p * 65536)
    return (torch.where(up, above, below) * b.sign() * unit).view(rows, -1)[:, :cols]


def _exact_values(codes, scales, rows, cols):
    r = torch.arange(rows, device=codes.device)[:, None]
    c = torch.arange(cols, device=codes.device)[None, :]
    code = (codes.gather(1, (c // 2).expand(rows, -1)) >> (4 * (c % 2)).to(torch.uint8)) & 15
    at = ((r // 128) * -(-cols // 128) + c // 128) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + c // 32 % 4
    m, sign = (code & 7).double(), 1.0 - 2.0 * (code >> 3).double()
    size = torch.where(m < 2, m / 2, (1 + (m % 2) / 2) * torch.exp2((m / 2).floor() - 1))
    return sign * size * torch.exp2(scales[at].double() - 127)


def _exact_norm(x, gamma, beta):
    x = x.double()
    mean = x.sum(1) / x.shape[1]
    var = ((x - mean[:, None]) ** 2).sum(1) / x.shape[1]
    rstd = (var + EPS) ** -0.5
    return (x - mean[:, None]) * rstd[:, None] * gamma.double() + beta.double(), mean, rstd


def _exact_norm_backward(dy, x, gamma, mean, rstd):
    n = x.shape[1]
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    t = dy.double() * gamma.double()
    s1, s2 = t.sum(1, keepdim=True), (t * xh).sum(1, keepdim=True)
    return rstd.double()[:, None] / n * (n * t - s1 - xh * s2), (dy.double() * xh).sum(0), dy.double().sum(0)


def exact(case, seed):
    s = prepare(case, seed)
    k = s["kind"]
    if k == "quantize":
        h = _draws(s["seed"], s["rows"], s["cols"], s["x"].device) if s["rounding"] == "stochastic" else None
        out = [_exact_quantize(s["x"], h)] if s["along"] != "cols" else []
        if s["along"] != "rows":
            out.append(_exact_quantize(s["x"].t(), None if h is None else h.t()))
        return out
    if k == "product":
        d = _exact_values(*s["a"], s["m"], s["k"]) @ _exact_values(*s["b"], s["n"], s["k"]).t()
        return d if s["add"] is None else d + s["add"].double()
    if k == "norm":
        return _exact_norm(s["x"], s["gamma"], s["beta"])
    if k == "norm_backward":
        return _exact_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"])
    r, c, n, dt = s["rows"], s["cols"], s["n"], DTYPES[s["dtype"]]
    if k == "serve":
        # the normalised values are rounded to the activations' type in front of the quantisation, by definition
        y = _exact_norm(s["x"], s["gamma"], s["beta"])[0].to(dt)
        return _exact_quantize(y, None) @ _exact_values(*s["w"], n, c).t()
    h = _draws(s["seed"], r, n, s["dy"].device)
    dx_in = _exact_quantize(s["dy"], h) @ _exact_values(*s["wt"], c, n).t()
    dw = _exact_quantize(s["dy"].t(), h.t()) @ _exact_values(*s["yt"], c, r).t()
    # ... as is the gradient that a product hands to layer norm
    dx, dgamma, dbeta = _exact_norm_backward(dx_in.to(dt), s["x"], s["gamma"], s["mean"], s["rstd"])
    return dx, dw, dgamma, dbeta
