"""Microscaled 4-bit quantization, its values and the product of two such matrices, against 64-bit definitions."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2109_12497_b200 import binding as B

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def as_matrix(x, dtype, pad=0, offset=0):
    """x as a CUDA matrix whose rows are `pad` elements longer and whose first element lies `offset` elements into its buffer."""
    rows, cols = x.shape
    buf = torch.full((offset + rows * (cols + pad) + 8,), float("nan"), dtype=dtype, device="cuda")
    m = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.as_tensor(x, dtype=torch.float64).to(torch.float32).to(dtype))
    return m


def empty_mx(rows, cols, extra=0):
    """A matrix with poisoned buffers; rows of codes `extra` bytes longer."""
    codes = torch.full((rows, 16 * -(-cols // 32) + extra), 0xEE, dtype=torch.uint8, device="cuda")
    scales = torch.full((B.mx_scale_bytes(rows, cols),), 0xDD, dtype=torch.uint8, device="cuda")
    return B.MxMatrix(rows, cols, codes, scales)


def check_mx(m, x, h):
    codes, scales, rest = ref.unpack(m.codes.cpu().numpy(), m.scales.cpu().numpy(), m.rows, m.cols)
    want_codes, want_scales = ref.quantize(x, h)
    assert np.array_equal(scales, want_scales)
    # a zero may have either sign
    assert np.array_equal(np.where(codes == 8, 0, codes), np.where(want_codes == 8, 0, want_codes))
    assert not rest.any()
    need = 16 * -(-m.cols // 32)
    assert (m.codes[:, need:].cpu().numpy() == 0xEE).all()


def spread(rows, cols, seed):
    """Values over many binades, with zeros, whole blocks of zeros, subnormals and exact grid points and ties among them."""
    r = np.random.default_rng(seed)
    x = r.standard_normal((rows, cols)) * 2.0 ** r.integers(-20, 20, (rows, 1))
    x[r.random((rows, cols)) < 0.05] = 0.0
    flat = x.reshape(-1)
    n = flat.size
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.5, 1.0, 3.0])
    at = r.integers(0, n, n // 8 + 1)
    flat[at] = r.choice(ties, at.size) * r.choice([-1.0, 1.0], at.size) * 2.0 ** r.integers(-3, 3, at.size)
    if rows > 2:
        x[1] = 0.0
        x[2] = r.standard_normal(cols) * 2.0 ** -130
    return x.astype(np.float32).astype(np.float64)


SIZES = [(1, 1), (1, 32), (2, 31), (3, 33), (5, 128), (31, 129), (32, 64), (33, 7), (128, 128), (130, 260), (257, 100), (64, 1000)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [0, 16])
def test_quantize_is_the_definition_bit_for_bit(rows, cols, dtype, bits):
    x = spread(rows, cols, rows * 1000 + cols)
    for k, (pad, offset, along) in enumerate([(0, 0, "both"), (3, 1, "both"), (8, 0, "rows"), (0, 0, "rows"), (5, 0, "cols"), (0, 8, "cols")]):
        g = as_matrix(x, DT[dtype], pad, offset)
        xs = g.double().cpu().numpy()
        seed = (0x123456789ABCDEF0 + 77 * k) & 0xFFFFFFFFFFFFFFFF
        q = empty_mx(rows, cols, 16 * (k % 2)) if along != "cols" else None
        qt = empty_mx(cols, rows, 32 * (k % 2)) if along != "rows" else None
        st = status()
        B.uq_mx_quantize(g, seed, bits, q, qt, st)
        h = ref.draws(rows, cols, seed) if bits else None
        if q is not None:
            check_mx(q, xs, h)
        if qt is not None:
            check_mx(qt, xs.T.copy(), None if h is None else h.T.copy())
        assert int(st.item()) == 0


def test_draws_on_both_sides_of_the_threshold():
    """p * 2^16 on integers, on halves of both parities and beside them, in each of the three steps."""
    rows, cols, seed = 64, 512, 99
    h = ref.draws(rows, cols, seed)
    r = np.random.default_rng(5)
    low = r.choice([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0], (rows, cols))
    step = np.where(low < 2, 0.5, np.where(low < 4, 1.0, 2.0))
    t = h + r.choice([0.0, 0.5, 1.0, -0.5, 1.5, 0.5 + 2.0 ** -6, 0.5 - 2.0 ** -6], (rows, cols))
    x = low + step * np.clip(t, 0, 65536) / 65536
    x[:, ::32] = 6.0                                         # the block's exponent is 0
    x = x.astype(np.float32).astype(np.float64) * r.choice([-1.0, 1.0], (rows, cols))
    q, qt = empty_mx(rows, cols), empty_mx(cols, rows)
    B.uq_mx_quantize(as_matrix(x, torch.float32), seed, 16, q, qt, None)
    check_mx(q, x, h)
    check_mx(qt, x.T.copy(), h.T.copy())


def test_extreme_magnitudes():
    big = float(torch.finfo(torch.float32).max)
    x = np.zeros((6, 64))
    x[0, :] = np.linspace(0.1, 1.0, 64) * big
    x[1, 5] = 2.0 ** -149
    x[2, :] = 2.0 ** -126
    x[3, :32] = 1.5 * 2.0 ** -125                            # 6 * 2^-127: the smallest scale still covers it
    x[3, 32:] = np.nextafter(np.float32(1.5 * 2.0 ** -125), np.float32(1.0))
    x[4, 0], x[4, 1:] = big, 1e-30
    x[5, :] = -1.5 * 2.0 ** 127
    x = x.astype(np.float32).astype(np.float64)
    for bits in (0, 16):
        q, qt, st = empty_mx(6, 64), empty_mx(64, 6), status()
        B.uq_mx_quantize(as_matrix(x, torch.float32), 3, bits, q, qt, st)
        h = ref.draws(6, 64, 3) if bits else None
        check_mx(q, x, h)
        check_mx(qt, x.T.copy(), None if h is None else h.T.copy())
        assert int(st.item()) == 0


def test_blocks_that_are_not_finite():
    x = spread(40, 100, 8)
    x[3, 40], x[7, 99], x[39, 0] = np.nan, np.inf, -np.inf
    for dtype in DT.values():
        g = as_matrix(x, dtype)
        xs = g.double().cpu().numpy()
        for bits in (0, 16):
            for q, qt in ((empty_mx(40, 100), None), (None, empty_mx(100, 40)), (empty_mx(40, 100), empty_mx(100, 40))):
                st = status()
                B.uq_mx_quantize(g, 1, bits, q, qt, st)
                assert int(st.item()) == B.UQ_STATUS_NONFINITE
                h = ref.draws(40, 100, 1) if bits else None
                for m, v, d in ((q, xs, h), (qt, xs.T.copy(), None if h is None else h.T.copy())):
                    if m is not None:
                        check_mx(m, v, d)
                        out = torch.zeros(m.rows, m.cols, dtype=dtype, device="cuda")
                        B.uq_mx_dequantize(m, out)
                        want = ref.values(*ref.quantize(v, d), m.cols)
                        assert np.array_equal(out.double().cpu().numpy(), want, equal_nan=True)
    B.uq_mx_quantize(g, 1, 0, empty_mx(40, 100), None, None)         # no status word: nothing to report to


def test_stochastic_rounding_is_unbiased():
    """The mean over 1000 seeds, in units of each value's own standard error: p(1-p) u^2 of a two-point variable."""
    n = 1000
    x = np.random.default_rng(1).standard_normal((4, 64))
    x[:, ::32] = 5.9
    x = x.astype(np.float32).astype(np.float64)
    g, q, qt = as_matrix(x, torch.float32), empty_mx(4, 64), empty_mx(64, 4)
    out, out_t = torch.empty(4, 64, device="cuda"), torch.empty(64, 4, device="cuda")
    total, total_t = torch.zeros(4, 64, dtype=torch.float64, device="cuda"), torch.zeros(64, 4, dtype=torch.float64, device="cuda")
    for seed in range(n):
        B.uq_mx_quantize(g, 1_000_003 * seed, 16, q, qt, None)
        B.uq_mx_dequantize(q, out)
        B.uq_mx_dequantize(qt, out_t)
        total += out
        total_t += out_t
    for t, v in ((total, x), (total_t, x.T)):
        _, scales = ref.quantize(np.ascontiguousarray(v))
        unit = np.repeat(2.0 ** (scales - 127.0), 32, 1)[:, :v.shape[1]]
        a = np.abs(v) / unit
        i = np.clip(np.searchsorted(ref.GRID, a, side="right") - 1, 0, 6)
        u = ref.GRID[i + 1] - ref.GRID[i]
        p = (a - ref.GRID[i]) / u
        sigma = u * np.sqrt(p * (1 - p) / n) * unit
        off = np.abs(t.cpu().numpy() / n - v)
        # 6 sigma of 256 values each, and the 2^-17 of a step that a 16-bit draw may be off
        assert (off <= 6 * sigma + u * unit * 2.0 ** -16).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 40), (129, 257), (64, 1024)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dequantize_every_code_and_scale(rows, cols, dtype):
    r = np.random.default_rng(rows)
    nb = -(-cols // 32)
    codes, scales = r.integers(0, 16, (rows, nb * 32)), r.integers(0, 253, (rows, nb))
    cb, sb = ref.pack(codes, scales)
    m = B.MxMatrix(rows, cols, torch.from_numpy(cb).cuda(), torch.from_numpy(sb).cuda())
    for pad, offset in ((0, 0), (8, 8), (1, 1)):
        out = as_matrix(np.zeros((rows, cols)), DT[dtype], pad, offset)
        B.uq_mx_dequantize(m, out)
        assert np.array_equal(out.double().cpu().numpy(), ref.values(codes, scales, cols))


# ---- product ------------------------------------------------------------------------------------------------------

def random_mx(rows, cols, seed, lo=124, hi=130):
    """A matrix of random codes and scales 2^(lo-127) .. 2^(hi-128), and its values."""
    r = np.random.default_rng(seed)
    nb = -(-cols // 32)
    codes, scales = r.integers(0, 16, (rows, nb * 32)), r.integers(lo, hi, (rows, nb))
    codes[:, cols:] = 0
    cb, sb = ref.pack(codes, scales)
    return B.MxMatrix(rows, cols, torch.from_numpy(cb).cuda(), torch.from_numpy(sb).cuda()), ref.values(codes, scales, cols)


PRODUCTS = [(1, 1, 1), (1, 128, 32), (2, 5, 33), (7, 130, 64), (16, 256, 128), (17, 100, 260), (33, 129, 500), (64, 64, 256),
            (65, 300, 1000), (128, 128, 512), (129, 257, 777), (200, 1000, 96), (256, 512, 384), (300, 3, 2048), (1, 4096, 4096),
            (13, 640, 5010), (513, 260, 4000), (1030, 700, 640),
            (2100, 2200, 700), (2305, 2049, 300), (300, 19001, 256), (19003, 257, 130), (2200, 4500, 64)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product_of_values_whose_sums_are_exact(m, n, k):
    """Scales of one binade: products are multiples of 1/4 up to 36 * 4 and their sums stay below 2^22 in magnitude times 1/4,
    exact in binary32 in any order, so the result is that of the definition bit for bit."""
    a, va = random_mx(m, k, m + k, 127, 129)
    b, vb = random_mx(n, k, n + k + 1, 127, 128)
    assert k * 36 * 2 * 4 < 2 ** 24 or k > 40_000
    want = va @ vb.T
    out = torch.full((m, n), 7.0, device="cuda")
    st = status()
    B.uq_mx_product(a, b, out, None, st)
    assert np.array_equal(out.double().cpu().numpy(), want)
    add = torch.from_numpy(np.random.default_rng(3).integers(-1000, 1000, (m, n)).astype(np.float32)).cuda()
    B.uq_mx_product(a, b, out, add, st)
    assert np.array_equal(out.double().cpu().numpy(), want + add.double().cpu().numpy())
    B.uq_mx_product(a, b, out, out, st)                      # onto itself
    assert np.array_equal(out.double().cpu().numpy(), 2 * want + add.double().cpu().numpy())
    low = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    B.uq_mx_product(a, b, low, None, st)
    assert torch.equal(low, torch.from_numpy(want).float().bfloat16().cuda())
    assert int(st.item()) == 0


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product_of_spread_scales(m, n, k, dtype):
    """Scales over 12 binades, rows of out, add and the codes padded and at odd offsets.  A binary32 sum of k products,
    each addition rounded or truncated, is off by at most k * 2^-23 of the sum of magnitudes."""
    a, va = random_mx(m, k, m * 7 + k, 118, 130)
    b, vb = random_mx(n, k, n * 5 + k, 118, 130)
    wide = torch.full((m, a.codes.shape[1] + 48), 0xFF, dtype=torch.uint8, device="cuda")
    wide[:, :a.codes.shape[1]] = a.codes
    a = B.MxMatrix(m, k, wide, a.scales)
    t = DT[dtype]
    for pad, offset, with_add in ((0, 0, False), (5, 3, True), (8, 0, True)):
        out = as_matrix(np.zeros((m, n)), t, pad, offset)
        whole = out.as_strided((m, n + pad), (n + pad, 1))
        add = as_matrix(np.random.default_rng(9).standard_normal((m, n)) * 50, t, pad + 1, offset) if with_add else None
        B.uq_mx_product(a, b, out, add, None)
        c = add.double().cpu().numpy() if with_add else 0.0
        want, size = va @ vb.T + c, np.abs(va) @ np.abs(vb).T + np.abs(c)
        bound = (k + 1) * 2.0 ** -23 * size
        if dtype == "bf16":
            bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        assert (np.abs(out.double().cpu().numpy() - want) <= bound + 1e-30).all()
        assert torch.isnan(whole[:, n:]).all()               # what lies between the rows is left alone


def test_product_carries_nan_scales_to_their_row_and_column_only():
    m, n, k = 150, 140, 320
    for row_a, row_b in ((17, 139), (149, 0)):
        a, va = random_mx(m, k, 1)
        b, vb = random_mx(n, k, 2)
        at = ((row_a // 128) * 3 + 1) * 512 + (row_a % 32) * 16 + (row_a % 128) // 32 * 4 + 2
        a.scales[at] = 255
        va[row_a] = np.nan
        at = ((row_b // 128) * 3 + 2) * 512 + (row_b % 32) * 16 + (row_b % 128) // 32 * 4 + 1
        b.scales[at] = 255
        vb[row_b] = np.nan
        out = torch.zeros(m, n, device="cuda")
        B.uq_mx_product(a, b, out, None, None)
        assert np.array_equal(np.isnan(out.cpu().numpy()), np.isnan(va @ vb.T))


def test_product_does_not_read_what_is_not_the_matrix():
    """Scales of rows behind the last and bytes between the rows of codes may hold anything, NaN scales among it."""
    for m, n, k in ((5, 9, 100), (130, 200, 300), (2100, 2300, 650)):
        a, va = random_mx(m, k, 3, 127, 128)
        b, vb = random_mx(n, k, 4, 127, 128)
        def poisoned(x, rows):
            codes = torch.full((rows, x.codes.shape[1] + 16), 0x77, dtype=torch.uint8, device="cuda")
            codes[:, :x.codes.shape[1]] = x.codes
            kt = -(-k // 128)
            s = torch.full_like(x.scales, 255).view(-1, kt, 32, 4, 4)
            src = x.scales.view(-1, kt, 32, 4, 4)
            for r in range(rows):
                s[r // 128, :, r % 32, r % 128 // 32] = src[r // 128, :, r % 32, r % 128 // 32]
            return B.MxMatrix(rows, k, codes, s.reshape(-1))
        out = torch.zeros(m, n, device="cuda")
        B.uq_mx_product(poisoned(a, m), poisoned(b, n), out, None, None)
        assert np.array_equal(out.double().cpu().numpy(), va @ vb.T)


def test_on_another_stream_and_in_a_graph():
    m, n, k = 70, 300, 1000
    x = as_matrix(spread(m, k, 2), torch.bfloat16)
    w, vw = random_mx(n, k, 6)
    q, out, st = empty_mx(m, k), torch.empty(m, n, device="cuda"), status()

    def chain():
        B.uq_mx_quantize(x, 5, 16, q, None, st)
        B.uq_mx_product(q, w, out, None, st)
    chain()
    torch.cuda.synchronize()
    want = out.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out.zero_()
        chain()
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(3):
        out.zero_()
        q.codes.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    x.copy_(x * 2)                                           # doubling every value doubles the scales ...
    graph.replay()
    torch.cuda.synchronize()
    scaled = torch.arange(m, device="cuda") != 2             # ... but where e stays at its lower end: row 2 holds values near 2^-130
    assert torch.equal(out[scaled], 2 * want[scaled])


def test_graphs_of_every_form_of_the_product():
    """A tile each, tiles shared by a cluster, pairs of CTAs: captured, then replayed one after the other and on another stream."""
    graphs = []
    for m, n, k in ((512, 4096, 512), (1, 4096, 4096), (182, 836, 7433), (2100, 2200, 700)):
        (a, va), (b, vb) = random_mx(m, k, m, 127, 128), random_mx(n, k, n, 127, 128)
        out, add = torch.zeros(m, n, device="cuda"), torch.ones(m, n, device="cuda")
        B.uq_mx_product(a, b, out, add, None)
        torch.cuda.synchronize()
        want = torch.from_numpy(va @ vb.T + 1).float().cuda()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.uq_mx_product(a, b, out, add, None)
        graphs.append((graph, out, want, a, b, add))
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        for g in graphs:
            g[1].zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for g in graphs + graphs[::-1]:
                g[0].replay()
        torch.cuda.synchronize()
        for g in graphs:
            assert torch.equal(g[1], g[2])


def test_two_streams_at_once():
    """Products of several shapes on two streams at the same time."""
    jobs = [(m, n, k, random_mx(m, k, m, 127, 128), random_mx(n, k, n, 127, 128)) for m, n, k in
            ((1, 4096, 4096), (300, 700, 2048), (16, 1000, 8192), (512, 512, 512))]
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [[torch.zeros(m, n, device="cuda") for m, n, *_ in jobs] for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                for (m, n, k, a, b), t in zip(jobs, o):
                    B.uq_mx_product(a[0], b[0], t, None, None)
    torch.cuda.synchronize()
    for j, (m, n, k, a, b) in enumerate(jobs):
        want = a[1] @ b[1].T
        for o in outs:
            assert np.array_equal(o[j].double().cpu().numpy(), want)


def test_offsets_beyond_32_bits():
    """Matrices of more than 2^31 elements: the last rows are those of the same rows by themselves."""
    rows, cols = 131_080, 16_640
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x.copy_(torch.arange(cols, device="cuda").remainder(997).sub(498).bfloat16().expand(rows, cols))
    x[-8:] = torch.randn(8, cols, device="cuda").bfloat16()
    q, last = B.MxMatrix(rows, cols), B.MxMatrix(8, cols)
    B.uq_mx_quantize(x, 0, 0, q, None, None)
    B.uq_mx_quantize(x[-8:], 0, 0, last, None, None)
    assert torch.equal(q.codes[-8:], last.codes)
    want = torch.empty(8, cols, dtype=torch.bfloat16, device="cuda")
    B.uq_mx_dequantize(last, want)
    B.uq_mx_dequantize(q, x)                                 # over its own input: the calls are in order
    assert torch.equal(x[-8:], want)
    del x, q
    n = 46_400                                               # n * n > 2^31, by pairs of CTAs; and few rows of a long out
    (a, va), (b, vb) = random_mx(64, 96, 1, 127, 128), random_mx(64, 96, 2, 127, 128)
    big = lambda m: B.MxMatrix(n, 96, m.codes.repeat(n // 64, 1), m.scales.repeat(-(-n // 128)))
    a.scales.view(-1, 32, 4, 4)[:, :, 2:] = a.scales.view(-1, 32, 4, 4)[:, :, :2]        # 64 rows twice in a tile of 128
    b.scales.view(-1, 32, 4, 4)[:, :, 2:] = b.scales.view(-1, 32, 4, 4)[:, :, :2]
    out = torch.empty(n, n, dtype=torch.bfloat16, device="cuda")
    B.uq_mx_product(big(a), big(b), out, None, None)
    want = torch.from_numpy(va @ vb.T).float().bfloat16().cuda()
    for i in (0, n // 2 // 64 * 64, n - 64):
        assert torch.equal(out[i:i + 64, -64:], want) and torch.equal(out[i:i + 64, :64], want)
