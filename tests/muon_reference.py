"""Orthogonalised updates (include/ags_muon.h) in 64 bits: from the definition,
and with the roundings that the header names (operands in fp16, X and sums in
fp32), whose distance from the definition is what those roundings cost."""
import torch

DEFAULT = (3.4445, -4.7750, 2.0315)


def _f32(x):
    return x.float().double()


def _half(x, scale):
    return (x * scale).float().half().double() / scale


def orthogonalize(u, steps=5, coefficients=DEFAULT, eps=1e-7, rounded=False):
    abc = [coefficients] * steps if not hasattr(coefficients[0], "__len__") else coefficients
    u = u.double()
    norm = u.square().sum().sqrt() + eps
    x = torch.where(u == 0, u, u / norm)
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    if rounded:
        x = _f32(x)
    for a, b, c in abc:
        xo = _half(x, 2.0 ** 15) if rounded else x
        gram = xo @ xo.t()
        if rounded:
            gram = _half(_f32(gram), 2.0 ** 15)
        p = b * gram + c * (gram @ gram)
        if rounded:
            p = _half(_f32(p), 2.0 ** 14)
        x = a * x + p @ xo
        if rounded:
            x = _f32(x)
    return x.t() if tall else x


def bound(u, **kw):
    """(the result, how far a kernel's may be off in the 2-norm of the
    difference): the rounded form's own distance, twice.  The kernel rounds at
    the same places; sums in another order send some of the roundings to the
    other neighbour, so that its error is another of the same size."""
    want = orthogonalize(u, **kw)
    off = float((orthogonalize(u, rounded=True, **kw) - want).norm())
    # and sums in fp32, of at most 2^15 terms each, three a step and amplified by up to 4 each
    return want, 2 * off + 1e-4 * float(want.norm())


def step(w, m, grads, matrices, lr, momentum, weight_decay, nesterov, **kw):
    """(w, m, bound on the 2-norm of w's error for each matrix) after a step."""
    w, m, g = w.double().clone(), m.double().clone(), grads.double().mean(dim=0)
    tols = []
    for o, rows, cols, scale in matrices:
        at = slice(o, o + rows * cols)
        m[at] = momentum * m[at] + g[at]
        u = g[at] + momentum * m[at] if nesterov else m[at]
        x, off = bound(u.view(rows, cols), **kw)
        w[at] = w[at] * (1 - lr * weight_decay) - lr * scale * x.reshape(-1)
        tols.append(lr * scale * off + 4 * 2.0 ** -24 * (float(w[at].norm()) + lr * scale * float(x.norm())))
    return w, m, tols
