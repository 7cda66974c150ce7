"""8-bit values with block scales in 64 bits, from the definition: e4m3 (largest value 448) under the least power of two, at least
2^-126, that keeps a block's largest finite magnitude within 448; nearest value, ties to even."""
import numpy as np


def e4m3_table():
    b = np.arange(128)
    e, m = b >> 3, (b & 7).astype(np.float64)
    v = np.where(e > 0, (8 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)
    v[127] = np.nan
    return v


TABLE = e4m3_table()


def decode(q):
    q = np.asarray(q, dtype=np.uint8)
    return np.where(q & 128, -1.0, 1.0) * TABLE[q & 127]


def scale_of(amax):
    """The scale's byte."""
    s = np.ones(np.shape(amax), dtype=np.int64)
    for b in range(1, 255):
        s = np.where(448.0 * 2.0 ** (b - 127.0) < amax, b + 1, s)
    return s


def encode(v):
    """Bytes of values that are within 448 (or not finite)."""
    a = np.abs(v)
    out = np.full(v.shape, 127, dtype=np.int64)
    fin = np.isfinite(v)
    x = a[fin]
    hi = np.clip(np.searchsorted(TABLE[:127], x), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = x - TABLE[lo], TABLE[hi] - x
    out[fin] = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (out | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def _padded(x, block_rows):
    r, c = x.shape
    p = np.zeros((-(-r // block_rows) * block_rows, -(-c // 128) * 128))
    p[:r, :c] = x
    return p


def quantize(x, block_rows=1):
    """(bytes, scale bytes) of a matrix, one scale per block_rows x 128."""
    r, c = x.shape
    p = _padded(np.asarray(x, dtype=np.float64), block_rows)
    b = p.reshape(p.shape[0] // block_rows, block_rows, p.shape[1] // 128, 128)
    s = scale_of(np.where(np.isfinite(b), np.abs(b), 0.0).max((1, 3)))
    q = encode(b / 2.0 ** (s - 127.0)[:, None, :, None])
    return q.reshape(p.shape)[:r, :c], s.astype(np.uint8)


def dequantize(q, s, block_rows=1):
    scale = np.repeat(np.repeat(2.0 ** (s.astype(np.float64) - 127.0), block_rows, 0), 128, 1)
    return decode(q) * scale[: q.shape[0], : q.shape[1]]


def rounded(x):
    return dequantize(*quantize(x))


def expert(xq, g, u, d):
    """E(x) of quantised rows xq and dequantised matrices: (outputs, h)."""
    a = xq @ g.T
    with np.errstate(over="ignore"):
        h = a / (1.0 + np.exp(-a)) * (xq @ u.T)
    return rounded(h) @ d.T, h
