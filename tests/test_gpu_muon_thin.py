"""Long schedules: thin matrices (a side of up to 16) against the singular values in
64 bits, for matrices of every rank, and larger ones.

The usual steps multiply a singular value near zero by 3.4445 each, by 1e17 in 32 of
them: one that is zero must stay zero.
"""
import pytest
import torch

import muon_reference as ref

pytestmark = pytest.mark.gpu

from paper_2603_18112_amd import muon  # noqa: E402

F, B = torch.float32, torch.bfloat16
U = 2.0 ** -24                       # half a step of fp32, relative
STEPS = (5, 6, 8, 10, 11, 12, 16, 32)


def _wide(kind, side, length):
    gen = torch.Generator().manual_seed(side * 10007 + length)
    whole = lambda *shape: torch.randint(-3, 4, shape, generator=gen).float()
    if kind == "ones":
        return torch.ones(side, length)
    if kind == "repeated":           # rows twice (the odd one once)
        return torch.randn((side + 1) // 2, length, generator=gen).repeat(2, 1)[:side].contiguous()
    if kind == "outer":
        return whole(side, 1) @ (whole(1, length) + 4.0)
    if kind == "sums":               # the last row the sum of the others, whole numbers
        u = whole(side, length)
        u[-1] = u[:-1].sum(dim=0)
        return u
    if kind == "rows":               # all but one are zero
        u = torch.zeros(side, length)
        u[side // 2] = torch.randn(length, generator=gen)
        return u
    return torch.randn(side, length, generator=gen)


def _exact(u, steps, coefficients=ref.DEFAULT, eps=1e-7):
    """The result by singular values (those below 2^-40 of the largest are zeros of
    the matrix), and how far a kernel's may be off in the 2-norm: each number's rounding,
    and eigenvalues of U U' / |U|^2 within 2^-49, whose relative error the steps multiply
    by |s f'(s) / f(s)| each."""
    abc = [coefficients] * steps if not hasattr(coefficients[0], "__len__") else coefficients
    left, s, right = torch.linalg.svd(u.double(), full_matrices=False)
    s = torch.where(s < 2.0 ** -40 * s.max(), 0.0, s) / (u.double().norm() + eps)
    off = torch.where(s > 0, 2.0 ** -49 / (s * s), 0.0)
    for a, b, c in abc:
        f, df = s * (a + b * s ** 2 + c * s ** 4), a + 3 * b * s ** 2 + 5 * c * s ** 4
        off = torch.where(s > 0, off * (s * df / f).abs() + 2.0 ** -50, 0.0)
        s = f
    want = left @ torch.diag(s) @ right
    return want, float((2 * U * want.norm() + (off * s).norm()))


def _check(got, want, off, what):
    d = float((got.double().cpu() - want).norm())
    assert torch.isfinite(got).all() and d <= off, f"{what}: {d:.3g} off, {off:.3g} allowed"


@pytest.mark.parametrize("kind", ["ones", "repeated", "outer", "sums", "rows", "full"])
@pytest.mark.parametrize("side,length", [(16, 100), (16, 16), (15, 1000), (7, 3000), (3, 140000), (2, 2), (1, 40)])
@pytest.mark.parametrize("tall", [False, True])
def test_thin_matrices_of_every_rank(kind, side, length, tall):
    u = _wide(kind, side, length)
    x = u.t().contiguous() if tall else u
    for steps in STEPS:
        want, off = _exact(u, steps)
        got = muon.orthogonalize(x.cuda(), steps=steps, dtype="f32")
        _check(got.t() if tall else got, want, off, f"{steps} steps")


@pytest.mark.parametrize("rows,cols", [(100, 150), (150, 17), (300, 300)])
def test_larger_matrices(rows, cols):
    """Of full rank within what the named roundings cost; of rank 1 bounded: singular values
    start below 1, the usual steps keep them below 1.21, and the roundings' 1 % comes on top."""
    for steps in (12, 32):
        u = torch.randn(rows, cols, generator=torch.Generator().manual_seed(rows))
        want, off = ref.bound(u, steps=steps)
        _check(muon.orthogonalize(u.cuda(), steps=steps, dtype="f32"), want, off, f"{steps} steps")
        for kind in ("ones", "outer"):
            got = muon.orthogonalize(_wide(kind, rows, cols).cuda(), steps=steps, dtype="f32").double().cpu()
            assert float(torch.linalg.matrix_norm(got, 2)) <= 1.23


@pytest.mark.parametrize("steps,coefficients", [(32, (1.5, -0.5, 0.0)), (20, (2.0, -1.5, 0.5)), (32, (1.0, 0.0, 0.0)),
                                                (9, [(3.4445, -4.775, 2.0315)] * 7 + [(2.0, -1.5, 0.5)] * 2)])
def test_other_long_schedules(steps, coefficients):
    for kind in ("outer", "full"):
        u = _wide(kind, 12, 700)
        want, off = _exact(u, steps, coefficients)
        _check(muon.orthogonalize(u.cuda(), steps=steps, coefficients=coefficients, dtype="f32"), want, off, kind)


def test_steps_of_a_handle_and_batches():
    kinds = ("ones", "full", "outer")
    us = [_wide(k, 11, 320) for k in kinds]
    got = muon.orthogonalize(torch.stack(us).cuda(), steps=16, dtype="f32")
    n = 11 * 320
    w, m = (torch.zeros(3 * n + 6304).cuda() for _ in range(2))
    grads = torch.zeros(1, 3 * n + 6304)
    other = torch.randn(70, 90, generator=torch.Generator().manual_seed(3))
    for i, u in enumerate(us):
        grads[0, i * n:(i + 1) * n] = u.reshape(-1)
    grads[0, 3 * n:3 * n + 6300] = other.reshape(-1)
    opt = muon.Muon([(i * n, 11, 320, 1.0) for i in range(3)] + [(3 * n, 70, 90, 1.0)], w, m, 1, lr=1.0, momentum=0.0,
                    nesterov=False, steps=16)
    opt.step(grads.cuda())
    for i, u in enumerate(us):
        want, off = _exact(u, 16)
        _check(got[i], want, off, kinds[i])
        assert torch.equal(-w[i * n:(i + 1) * n].view(11, 320), got[i])
        assert torch.equal(muon.orthogonalize(u.cuda(), steps=16, dtype="f32"), got[i])
        assert torch.equal(muon.orthogonalize(u.to(B).cuda(), steps=16), muon.orthogonalize(u.to(B).cuda(), steps=16))
    assert torch.equal(-w[3 * n:3 * n + 6300].view(70, 90), muon.orthogonalize(other.cuda(), steps=16, dtype="f32"))


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 300), (300, 3), (16, 20), (5, 5)])
def test_scales_zeros_and_nonfinite_values(rows, cols):
    u = torch.randn(rows, cols, generator=torch.Generator().manual_seed(rows))
    kw = {"steps": 12, "dtype": "f32"}
    base = muon.orthogonalize(u.cuda(), eps=0.0, **kw)
    for p in (-100, 90):             # powers of two
        assert torch.equal(muon.orthogonalize((u.double() * 2.0 ** p).float().cuda(), eps=0.0, **kw), base)
    x = torch.stack([u, torch.zeros_like(u), u, u]).cuda()
    x[2, 0, 0], x[3, -1, -1] = float("nan"), float("inf")
    for eps in (0.0, 1e-7):
        got = muon.orthogonalize(x, eps=eps, **kw)
        assert torch.isfinite(got[0]).all() and (got[1] == 0).all() and torch.isnan(got[2:]).all()


def test_replayed_from_a_graph():
    x = _wide("outer", 9, 500).cuda()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    muon.orthogonalize(x, steps=10)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = muon.orthogonalize(x, steps=10, dtype="f32")
    for kind in ("ones", "full", "sums"):
        x.copy_(_wide(kind, 9, 500))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, muon.orthogonalize(x, steps=10, dtype="f32"))


@pytest.mark.parametrize("K,dtype", [(1, F), (3, B)])
def test_handles_of_odd_thin_matrices(K, dtype):
    """Elements that fill no piece of eight, one after the other in the workspace: the momentum
    exactly, the weights as the calls by themselves, the buffers between them untouched."""
    shapes = [(1, 1), (13, 7), (3, 1001), (20011, 1), (5, 5), (40, 50), (16, 129), (1, 40000), (300, 11)]
    matrices, at = [], 0
    for r, c in shapes:
        matrices.append((at, r, c, 1.0))
        at += -(-r * c // 8) * 8 + 8
    gen = torch.Generator().manual_seed(K)
    w, m = torch.randn(at, generator=gen), torch.randn(at, generator=gen)
    # whole numbers: their means and the momentum are exact
    m = torch.randint(-8, 9, (at,), generator=gen).float()
    grads = (torch.randint(-8, 9, (K, at), generator=gen) * K).to(dtype)
    wc, mc = w.cuda(), m.cuda()
    opt = muon.Muon(matrices, wc, mc, K, grad_dtype="f32" if dtype is F else "bf16", lr=0.5, momentum=0.5, nesterov=False)
    opt.step(grads.cuda())
    want = 0.5 * m + grads.float().mean(dim=0)
    inside = torch.zeros(at, dtype=torch.bool)
    for o, r, c, _ in matrices:
        inside[o:o + r * c] = True
        x = muon.orthogonalize(want[o:o + r * c].view(r, c).cuda(), dtype="f32").cpu().double().reshape(-1)
        assert ((wc.cpu()[o:o + r * c].double() - (w[o:o + r * c].double() - 0.5 * x)).abs() <=
                U * (w[o:o + r * c].double() - 0.5 * x).abs() * 1.01).all()
    assert torch.equal(mc.cpu()[inside], want[inside])
    assert torch.equal(mc.cpu()[~inside], m[~inside]) and torch.equal(wc.cpu()[~inside], w[~inside])
