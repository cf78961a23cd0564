"""Microscaled storage from its definition, in numpy with 64-bit floats: blocks of
32, the scale from the largest magnitude, the nearest value of the format by
distance (ties to the even code).  Shares no code with the library."""
import numpy as np

EMAX = {4: 2, 8: 8}
PAD = {4: 256, 8: 128}


def _grid(bits):
    """Magnitudes of the format, by code."""
    if bits == 4:
        return np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
    g = []
    for code in range(127):  # 127 is NaN
        e, m = code >> 3, code & 7
        g.append(m / 8 * 2.0**-6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(g)


GRID = {b: _grid(b) for b in (4, 8)}


def _nearest(y, bits):
    """Codes of the magnitudes y."""
    g = GRID[bits]
    hi = np.clip(np.searchsorted(g, y), 1, len(g) - 1)
    lo = hi - 1
    down = (y - g[lo] < g[hi] - y) | ((y - g[lo] == g[hi] - y) & (lo % 2 == 0))
    return np.where(down, lo, hi)


def encode(x, bits):
    """(data, scales) of a matrix of 32-bit floats as they are stored."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    pc = -(-cols // PAD[bits]) * PAD[bits]
    p = np.zeros((rows, pc), dtype=np.float32)
    p[:, :cols] = x
    p = p.reshape(rows, pc // 32, 32)
    bad = ~np.isfinite(p).all(-1)
    p = np.where(bad[..., None], np.float32(0), p)
    top = np.abs(p).max(-1)
    field = top.view(np.uint32) >> 23
    s = np.where(bad, 255, np.maximum(field.astype(np.int64) - EMAX[bits], 0))
    y = p.astype(np.float64) * np.exp2(127.0 - np.where(bad, 127, s))[..., None]
    code = _nearest(np.abs(y), bits) | np.signbit(p).astype(np.int64) << (bits - 1)
    code = np.where(bad[..., None], 0, code).reshape(rows, pc).astype(np.uint8)
    if bits == 4:
        code = code[:, 0::2] | code[:, 1::2] << 4
    return np.ascontiguousarray(code), s.astype(np.uint8)


def decode(data, scales, bits, cols):
    """The values that a stored matrix stands for, 64-bit floats."""
    rows = data.shape[0]
    if bits == 4:
        code = np.empty((rows, 2 * data.shape[1]), dtype=np.int64)
        code[:, 0::2], code[:, 1::2] = data & 15, data >> 4
    else:
        code = data.astype(np.int64)
    half = 1 << (bits - 1)
    g = np.concatenate([GRID[bits], np.full(half - len(GRID[bits]), np.nan)])
    v = np.where(code >= half, -g[code % half], g[code % half])
    s = scales.astype(np.float64)
    unit = np.where(scales == 255, np.nan, np.exp2(s - 127))
    return (v * np.repeat(unit, 32, axis=1))[:, :cols]
