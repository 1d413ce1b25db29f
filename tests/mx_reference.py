"""The 4-bit format and its products in 64 bits, written from the format's
definition in numpy (shares no code with the package)."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def store_rows(x, noise=None):
    """(values, scale exponents) of x [rows, cols] float64: exponent 128 marks
    a block with a NaN or an infinity."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    z = np.zeros((rows, nb * 32))
    z[:, :cols] = x
    z = z.reshape(rows, nb, 32)
    r = np.zeros((rows, nb * 32))
    if noise is not None:
        r[:, :cols] = noise
    r = r.reshape(rows, nb, 32)
    top = np.abs(z).max(axis=2)
    bad = ~np.isfinite(top)
    top = np.where(bad, 1.0, top)
    e = np.frexp(top)[1].astype(np.int64) - 3          # floor(log2 top) - 2
    e[top == 0] = -127
    if noise is not None:
        e = np.where(top > 6.0 * np.ldexp(1.0, e), e + 1, e)
    e = np.clip(e, -127, 125)
    y = np.abs(np.where(bad[:, :, None], 0.0, z)) / np.ldexp(1.0, e)[:, :, None]
    if noise is None:
        # the nearest grid value; a tie goes to the even code
        mid = (GRID[1:] + GRID[:-1]) / 2
        c = np.zeros(y.shape, np.int64)
        for i, t in enumerate(mid):
            c += (y > t) | ((y == t) & (i % 2 == 1))
    else:
        c = np.zeros(y.shape, np.int64)
        for i in range(7):
            f = np.clip((y - GRID[i]) / (GRID[i + 1] - GRID[i]), 0.0, None)
            here = (y >= GRID[i]) & (y < GRID[i + 1])
            c = np.where(here, i + (f + (r + 0.5) / 256.0 >= 1.0), c)
        c = np.where(y >= 6.0, 7, c)
    v = GRID[c] * np.ldexp(1.0, e)[:, :, None] * np.where(z < 0, -1.0, 1.0)
    v = np.where(bad[:, :, None], np.nan, v)
    return v.reshape(rows, nb * 32)[:, :cols], np.where(bad, 128, e)


def scale_rows(scales, rows, cols):
    """Scale bytes [rows][padded / 32] of the stored [padded / 256][rows'][8]."""
    kp, rp = -(-cols // 256) * 256, -(-rows // 16) * 16
    return scales.reshape(kp // 256, rp, 8).transpose(1, 0, 2).reshape(rp, kp // 32)[:rows]


def unpack(codes, scales, rows, cols):
    """Values of packed bytes, padding columns included."""
    kp = -(-cols // 256) * 256
    c = codes.reshape(rows, kp // 2)
    n = np.stack([c & 15, c >> 4], axis=2).reshape(rows, kp)
    s = scale_rows(scales, rows, cols)
    v = GRID[n & 7] * np.where(n & 8, -1.0, 1.0) * np.repeat(np.exp2(s.astype(np.float64) - 127.0), 32, axis=1)
    return np.where(np.repeat(s == 255, 32, axis=1), np.nan, v)
