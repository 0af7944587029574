"""Plain 64-bit definitions of the layer operators (numpy), for the tests: microscaled 4-bit values, their product, layer norm."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TAG = 0x4D584634


def philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 of arrays of counter words."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.asarray(w, dtype=np.uint64) for w in (c0, c1, c2, c3)]
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & m, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, -1)


def draws(rows, cols, seed):
    """The 16-bit draws of a matrix's elements."""
    nb = -(-cols // 8)
    c0 = np.broadcast_to(np.arange(nb), (rows, nb))
    c1 = np.broadcast_to(np.arange(rows)[:, None], (rows, nb))
    w = philox(c0, c1, np.zeros_like(c0), np.full_like(c0, TAG), seed)
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(rows, nb * 8)[:, :cols].astype(np.int64)


def exponent(top):
    """Smallest integer e >= -127 with top <= 6 * 2^e."""
    if top == 0:
        return -127
    e = int(np.floor(np.log2(top))) - 4
    while 6.0 * 2.0 ** e < top:
        e += 1
    return max(e, -127)


def quantize(x, h=None):
    """x [rows, cols] float64 -> (codes [rows, 32 nb] as integers 0..15, scale bytes [rows, nb]); h: the draws, or None."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    full = np.zeros((rows, nb * 32))
    full[:, :cols] = x
    hh = np.zeros((rows, nb * 32), dtype=np.int64)
    if h is not None:
        hh[:, :cols] = h
    codes = np.zeros((rows, nb * 32), dtype=np.int64)
    scales = np.zeros((rows, nb), dtype=np.int64)
    for b in range(nb):
        v = full[:, 32 * b:32 * b + 32]
        finite = np.isfinite(v).all(1)
        e = np.array([exponent(t) if f else 0 for t, f in zip(np.abs(np.where(np.isfinite(v), v, 0)).max(1), finite)])
        a = np.where(finite[:, None], np.abs(np.where(np.isfinite(v), v, 0)), 0) / 2.0 ** e[:, None]
        i = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 6)
        p = (a - GRID[i]) / (GRID[i + 1] - GRID[i])
        if h is None:
            up = (p > 0.5) | ((p == 0.5) & (i % 2 == 1))
        else:
            up = hh[:, 32 * b:32 * b + 32] < np.rint(p * 65536)
        codes[:, 32 * b:32 * b + 32] = np.where(finite[:, None], i + up + 8 * np.signbit(v), 0)
        scales[:, b] = np.where(finite, e + 127, 255)
    return codes, scales


def values(codes, scales, cols):
    """The values of codes [rows, 32 nb] and scale bytes [rows, nb]."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales - 127.0))
    return (v.reshape(*scales.shape, 32) * s[..., None]).reshape(codes.shape)[:, :cols]


def pack(codes, scales):
    """The bytes of codes, and of scales in their tiles."""
    rows, nb = scales.shape
    out = (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)
    kt = -(-nb // 4)
    tiles = np.zeros(-(-rows // 128) * kt * 512, dtype=np.uint8)
    for r in range(rows):
        for b in range(nb):
            tiles[((r // 128) * kt + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4] = scales[r, b]
    return out, tiles


def unpack(code_bytes, tiles, rows, cols):
    """(codes, scales, the scale bytes of the blocks that fill up a row's last tile)."""
    nb, kt = -(-cols // 32), -(-cols // 128)
    b = code_bytes[:, : nb * 16].astype(np.int64)
    codes = np.stack([b & 15, b >> 4], -1).reshape(rows, nb * 32)
    s = tiles.astype(np.int64).reshape(-(-rows // 128), kt, 32, 4, 4).transpose(0, 3, 2, 1, 4).reshape(-1, kt * 4)[:rows]
    return codes, s[:, :nb], s[:, nb:]


def layer_norm(x, gamma, beta, eps):
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    y = xh if gamma is None else xh * gamma
    return y if beta is None else y + beta, mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd):
    xh = (x - mean[:, None]) * rstd[:, None]
    t = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (t - t.mean(1, keepdims=True) - xh * (t * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)
