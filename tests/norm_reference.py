"""The layer norm of include/ags_norm.h in 64 bits, with bounds on what fp32
arithmetic may be off.

U is half a step of fp32.  A sum of terms t in any order of at most D additions
each is off by at most D U sum |t|; D below is a row's: 32 terms a lane (or its
share of a long row), 6 steps over a wave, 16 over a block's waves.
"""
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # half a step, relative


def depth(cols):
    return 32 + 22 + 8 * (cols // 8192)


def forward(x, weight, bias, eps, dtype):
    """(y, mean, rstd, and how far each may be off)."""
    x = x.double()
    cols = x.shape[1]
    w = torch.ones(cols, dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros(cols, dtype=torch.float64) if bias is None else bias.double()
    mean = x.mean(dim=1, keepdim=True)
    d = x - mean
    var = d.square().mean(dim=1, keepdim=True)
    rstd = (var + eps).rsqrt()
    z = d * rstd
    y = z * w + b
    D = depth(cols)
    # the sum, and the division by n
    e_mean = (D + 1) * U * x.abs().mean(dim=1, keepdim=True)
    # differences (one rounding, and the mean's error, which adds its square to the
    # variance; their rounding 2 U of a square), squares and sum, division, eps, root,
    # reciprocal.  A half of the variance's relative error.
    e_rstd = rstd * (0.5 * ((D + 5) * U + (e_mean * rstd).square() + 2 * U * e_mean * rstd) + 3 * U)
    e_z = z.abs() * (e_rstd / rstd + 2 * U) + rstd * e_mean
    # the product with the weight and the sum with the bias are one operation
    e_y = w.abs() * e_z * 1.001 + y.abs() * (U + HALF[dtype]) + 1e-38
    return (y, mean[:, 0], rstd[:, 0]), (e_y, e_mean[:, 0] + 1e-45, e_rstd[:, 0])


def backward(dy, x, saved, weight, dtype, dw_dtype):
    """(dx, dweight, dbias, and how far each may be off) for the fp32 statistics
    `saved`, which are taken as they are."""
    dy, x = dy.double(), x.double()
    rows, cols = x.shape
    mean, rstd = saved.double()[0][:, None], saved.double()[1][:, None]
    w = torch.ones(cols, dtype=torch.float64) if weight is None else weight.double()
    z, g = (x - mean) * rstd, dy * w
    m0, m1 = g.mean(dim=1, keepdim=True), (g * z).mean(dim=1, keepdim=True)
    dx = rstd * (g - m0 - z * m1)
    D = depth(cols)
    # z: two roundings; g: one; the means: their sums and a division
    e_m0 = (D + 2) * U * g.abs().mean(dim=1, keepdim=True)
    e_m1 = (D + 5) * U * (g * z).abs().mean(dim=1, keepdim=True)
    e_dx = rstd * (U * (4 * g.abs() + 4 * m0.abs() + 6 * (z * m1).abs()) + e_m0 + z.abs() * e_m1)
    e_dx = 1.001 * e_dx + dx.abs() * HALF[dtype] + 1e-38
    dw, db = (dy * z).sum(dim=0), dy.sum(dim=0)
    e_dw = (rows + 4) * U * (dy * z).abs().sum(dim=0) * 1.001 + dw.abs() * HALF[dw_dtype] + 1e-38
    e_db = (rows + 1) * U * dy.abs().sum(dim=0) * 1.001 + db.abs() * HALF[dw_dtype] + 1e-38
    return (dx, dw, db), (e_dx, e_dw, e_db)
