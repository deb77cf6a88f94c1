"""The 4-bit cache format in 64 bits, from its definition: every candidate of the grid is tried for every element."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EVEN_FIRST = (0, 2, 4, 6, 1, 3, 5, 7)   # of two equally near values the one with the even code


def encode(x):
    """[..., D] -> (codes uint8 [..., D/2], scales uint8 [..., D/32])."""
    x = np.asarray(x, np.float64)
    b = x.reshape(x.shape[:-1] + (-1, 32))
    finite = np.isfinite(b).all(-1)
    b = np.where(finite[..., None], b, 0.0)
    top = np.abs(b).max(-1)
    m, e = np.frexp(top)                 # top = m * 2^e, m in [0.5, 1)
    e = e - 1 + (m >= 0.875) - 2         # 1.75 and more rounds up to 2 at two significant bits
    e = np.where(top > 0, np.clip(e, -124, 125), -124)
    unit = np.ldexp(1.0, e)[..., None]
    best, off = np.zeros(b.shape, np.int64), np.full(b.shape, np.inf)
    for k in EVEN_FIRST:
        d = np.abs(np.abs(b) - GRID[k] * unit)
        best = np.where(d < off, k, best)
        off = np.minimum(off, d)
    best = (best | np.where(np.signbit(b), 8, 0)).reshape(x.shape)
    best = np.where(np.repeat(finite, 32, -1), best, 0).astype(np.uint8)
    return best[..., 0::2] | best[..., 1::2] << 4, np.where(finite, e + 127, 255).astype(np.uint8)


def decode(codes, scales):
    """The values, fp64 [..., D]."""
    k = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    v = np.where(k & 8, -1.0, 1.0) * GRID[k & 7]
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(unit, 32, -1)
