"""MXFP4 in plain numpy, for the tests of the operators that read or write it: no code of the library's."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_bytes(v):
    """[rows, blocks] scale bytes of rows in 64 bits: the exponent of the largest magnitude taken to two significant bits."""
    r, k = v.shape
    blocks = -(-k // 32)
    a = np.zeros((r, blocks * 32))
    a[:, :k] = np.abs(v)
    bad = ~np.isfinite(a).reshape(r, blocks, 32).all(2)
    top = np.where(np.isfinite(a), a, 0.0).reshape(r, blocks, 32).max(2)
    m, e = np.frexp(top)  # top = m 2^e, m in [1/2, 1)
    e = np.where(m >= 0.875, e + 1, e) - 3  # 2^e: m 2^e in [4, 7) or 3.5
    e = np.where(top == 0, -127, np.clip(e, -127, 127)) + 127
    return np.where(bad, 255, e).astype(np.uint8)


def powers(e):
    return np.where(e == 255, np.nan, np.ldexp(1.0, e.astype(np.int64) - 127))


def codes(v, e):
    """[rows, 32 blocks] codes of rows in 64 bits under scale bytes e: nearest of the grid, ties to the even code."""
    r, k = v.shape
    a = np.zeros((r, e.shape[1] * 32))
    with np.errstate(invalid="ignore"):
        a[:, :k] = v / np.repeat(powers(e), 32, axis=1)[:, :k]
    a[np.repeat(e, 32, axis=1) == 255] = 0.0
    m = np.abs(a)
    d = np.abs(m[..., None] - GRID)
    c = d.argmin(-1)  # of two as near the lower one
    odd = (c % 2 == 1) & (c < 7) & (m == (GRID[c] + GRID[np.minimum(c + 1, 7)]) / 2)
    c = np.where(odd, c + 1, c)
    return (c | (np.signbit(a) << 3)).astype(np.uint8)


def values(c, e, k):
    v = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7]
    return (v * np.repeat(powers(e), 32, axis=1))[:, :k]


def packed(c):
    return c[:, 0::2] | (c[:, 1::2] << 4)


def unpacked(b):
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[0], -1)


def place(row, block, blocks):
    return ((row // 128) * -(-blocks // 4) + block // 4) * 512 + (row % 32) * 16 + (row // 32 % 4) * 4 + block % 4


def tiled(e, fill=0):
    """Scale bytes as they lie in memory; `fill`: those of rows behind the last."""
    r, b = e.shape
    t = np.full(-(-r // 128) * -(-b // 4) * 512, fill, np.uint8)
    rows = np.arange(r)[:, None]
    for j in range(-(-b // 4) * 4):
        t[place(rows[:, 0], j, b)] = e[:, j] if j < b else 0
    return t


def from_tiles(t, r, b):
    return t[place(np.arange(r)[:, None], np.arange(b)[None, :], b)]


def quantised(v):
    """(values, packed codes, tiled scales) of rows in 64 bits."""
    e = scale_bytes(v)
    c = codes(v, e)
    return values(c, e, v.shape[1]), packed(c), tiled(e)


def check_quantised(v, e, out, t, fill=0xA5):
    """Rows in 4 bits (packed, with what lies between rows, and scales) hold what the format makes of some values within e of v: the
    scale lies between those of the block's largest magnitude less and more the bound, and each code between those of the
    value less and more the bound, under that scale. Zeros behind the last feature and block, all else as it was."""
    m, n = v.shape
    blocks = -(-n // 32)
    got = from_tiles(t, m, blocks)
    low, high = np.maximum(np.abs(v) - e, 0.0), np.abs(v) + e
    assert (got >= scale_bytes(low)).all() and (got <= scale_bytes(high)).all()
    assert np.array_equal(t, tiled(got, fill))
    assert (out[:, 16 * blocks:] == fill).all()
    c = unpacked(out[:, :16 * blocks])
    assert (c[:, n:] == 0).all()
    q = values(c, got, n)
    least, most = (values(codes(v + s * e, got), got, n) for s in (-1, 1))
    bad = ~((q >= least) & (q <= most))
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:3], q[bad][:3], v[bad][:3])
