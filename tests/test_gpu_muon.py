"""Orthogonalised updates on the GPU: partial permutations, for which one step is
exact, and random matrices within what the named roundings cost
(muon_reference.py)."""
import pytest
import torch

import muon_reference as ref

pytestmark = pytest.mark.gpu

from paper_2603_18112_amd import ags, muon  # noqa: E402

F, B = torch.float32, torch.bfloat16
H = 2.0 ** -8                        # half a step of bf16, relative
DYADIC = (2.0, -1.5, 0.5)

# one element, vectors, sizes around each tile's edge, tall, wide and square
SHAPES = [(1, 1), (1, 9), (9, 1), (4, 4), (16, 70), (65, 16), (64, 64), (63, 200), (130, 129), (129, 1000),
          (600, 64), (257, 300), (512, 512), (700, 1300), (2100, 300)]


def _permutation(rows, cols, seed=0):
    """1 and -1 in 4^j places, no two in a row or column: divided by the norm 2^j
    and after a step with dyadic coefficients every number is exact, as operands
    (at most 11 bits) and as fp32."""
    gen = torch.Generator().manual_seed(seed * 131 + rows * 7 + cols)
    n = 1
    while 4 * n <= min(rows, cols, 256):
        n *= 4
    u = torch.zeros(rows, cols)
    i, j = torch.randperm(rows, generator=gen)[:n], torch.randperm(cols, generator=gen)[:n]
    u[i, j] = torch.randint(0, 2, (n,), generator=gen).float() * 2 - 1
    y = 1.0 / n
    x = n ** -0.5
    return u, u * (x * (2.0 - 1.5 * y + 0.5 * y * y))


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_partial_permutations_are_exact(rows, cols):
    u, want = _permutation(rows, cols)
    for dtype in (F, B):
        got = muon.orthogonalize(u.to(dtype).cuda(), steps=1, coefficients=DYADIC, eps=0.0, dtype="f32")
        assert torch.equal(got.cpu(), want)
    got = muon.orthogonalize(u.cuda(), steps=1, coefficients=DYADIC, eps=0.0)
    assert got.dtype == B and torch.equal(got.cpu(), want.to(B))


def _random(rows, cols, kind, seed=0):
    gen = torch.Generator().manual_seed(seed * 17 + rows * 3 + cols)
    u = torch.randn(rows, cols, generator=gen)
    if kind == "low":                # a few strong directions over weak noise
        r = max(1, min(rows, cols) // 16)
        u = u * 0.01 + torch.randn(rows, r, generator=gen) @ torch.randn(r, cols, generator=gen)
    return u * 1e-3


def _near(got, want, off, what=""):
    d = float((got.double().cpu() - want).norm())
    off = off + (H * float(want.norm()) if got.dtype == B else 0.0)
    assert torch.isfinite(got).all() and d <= off, f"{what}: {d:.3g} off, {off:.3g} allowed"


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind", ["full", "low"])
def test_random_matrices(rows, cols, kind):
    u = _random(rows, cols, kind)
    want, off = ref.bound(u)
    _near(muon.orthogonalize(u.cuda(), dtype="f32"), want, off)
    ub = u.to(B)
    want, off = ref.bound(ub)
    _near(muon.orthogonalize(ub.cuda()), want, off)


@pytest.mark.parametrize("side", [1, 2, 3, 7, 16])
@pytest.mark.parametrize("length", [1, 16, 100, 513, 3000, 140000])
@pytest.mark.parametrize("tall", [False, True])
def test_thin_matrices(side, length, tall):
    """One side of up to 16: X = Q U / |U| with Q rounded to fp32 and sums of `side`
    products, (side + 2) 2^-24 of the sum of magnitudes."""
    u = _random(min(side, length), max(side, length), "full", 4)
    if side == 3:                    # one singular value
        u = u[:, :1] @ u[:1]
    x = u.t().contiguous() if tall else u
    norm = u.double().norm() + 1e-7
    a, q = u.double() @ u.double().t() / norm ** 2, torch.eye(u.shape[0], dtype=torch.float64)
    for _ in range(5):
        p = ref.DEFAULT[0] * torch.eye(u.shape[0], dtype=torch.float64) + ref.DEFAULT[1] * a + ref.DEFAULT[2] * a @ a
        a, q = p @ a @ p, p @ q
    want, tol = q @ u.double() / norm, (u.shape[0] + 2) * 2.0 ** -24 * 1.001 * (q.abs() @ u.double().abs() / norm)
    got = muon.orthogonalize(x.cuda(), dtype="f32").cpu()
    assert (((got.t() if tall else got).double() - want).abs() <= tol + 1e-12 * want.abs()).all()
    # and as the step of a matrix among others
    o = -(-x.numel() // 8) * 8
    other = _random(70, 90, "full", 5)
    w, m = (torch.zeros(o + 6304).cuda() for _ in range(2))
    grads = torch.zeros(1, o + 6304)
    grads[0, :x.numel()], grads[0, o:o + 6300] = x.reshape(-1), other.reshape(-1)
    opt = muon.Muon([(0, *x.shape, 1.0), (o, 70, 90, 1.0)], w, m, 1, lr=1.0, momentum=0.0, nesterov=False)
    opt.step(grads.cuda())
    assert torch.equal(-w[:x.numel()].cpu().view(x.shape), got)
    assert torch.equal(-w[o:o + 6300].view(70, 90), muon.orthogonalize(other.cuda(), dtype="f32"))


@pytest.mark.parametrize("steps,coefficients", [(1, ref.DEFAULT), (2, DYADIC), (12, (1.5, -0.5, 0.0)),
                                                (3, ((3.4445, -4.775, 2.0315), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0)))])
def test_other_schedules(steps, coefficients):
    u = _random(100, 150, "full", 1)
    kw = {"steps": steps, "coefficients": coefficients, "eps": 1e-3}
    want, off = ref.bound(u, **kw)
    _near(muon.orthogonalize(u.cuda(), dtype="f32", **kw), want, off)


@pytest.mark.parametrize("rows,cols", [(5, 7), (64, 130), (200, 33), (300, 300)])
def test_batches_strides_and_neighbours(rows, cols):
    us = [_permutation(rows, cols, seed) for seed in range(5)]
    x, want = torch.stack([a for a, _ in us]).cuda(), torch.stack([b for _, b in us])
    kw = {"steps": 1, "coefficients": DYADIC, "eps": 0.0}
    assert torch.equal(muon.orthogonalize(x, dtype="f32", **kw).cpu(), want)
    wide = torch.full((5, rows + 2, cols + 3), 7.0, dtype=B).cuda()
    xs = wide[:, 1:1 + rows, 2:2 + cols]
    xs.copy_(x)
    out = torch.full((5, rows + 1, cols + 5), 7.0).cuda()
    got = muon.orthogonalize(xs, out=out[:, :rows, 3:3 + cols], **kw)
    assert torch.equal(got.cpu(), want)
    out[:, :rows, 3:3 + cols] = 7.0
    assert (out == 7).all()
    # transposed and repeated inputs are copied
    xt = x.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(muon.orthogonalize(xt, dtype="f32", **kw).cpu(), want)
    same = muon.orthogonalize(x[:1].expand(5, rows, cols), dtype="f32", **kw)
    assert torch.equal(same.cpu(), want[:1].expand(5, rows, cols))
    # each matrix by itself, bit for bit, with the usual steps
    u = torch.stack([_random(rows, cols, "full", s) for s in range(5)]).cuda()
    got = muon.orthogonalize(u, dtype="f32")
    for i in range(5):
        want, off = ref.bound(u[i].cpu())
        _near(got[i], want, off)
    assert torch.equal(muon.orthogonalize(u, dtype="f32"), got)


def test_scales_zeros_and_nonfinite_values():
    u = _random(40, 60, "full", 2)
    base = muon.orthogonalize(u.cuda(), eps=0.0, dtype="f32")
    for p in (-100, 90):             # powers of two: norms whose squares leave fp32
        assert torch.equal(muon.orthogonalize((u.double() * 2.0 ** p).float().cuda(), eps=0.0, dtype="f32"), base)
    x = torch.stack([u, torch.zeros_like(u), u, u]).cuda()
    x[2, 3, 4], x[3, 39, 59] = float("nan"), float("inf")
    for eps in (0.0, 1e-7):
        got = muon.orthogonalize(x, eps=eps, dtype="f32")
        assert torch.isfinite(got[0]).all() and (got[1] == 0).all() and torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    assert torch.equal(muon.orthogonalize(x, eps=0.0, dtype="f32")[0], base)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 300), (300, 3), (16, 20)])
def test_scales_zeros_and_nonfinite_values_of_thin_matrices(rows, cols):
    u = _random(rows, cols, "full", 6)
    base = muon.orthogonalize(u.cuda(), eps=0.0, dtype="f32")
    for p in (-100, 90):
        assert torch.equal(muon.orthogonalize((u.double() * 2.0 ** p).float().cuda(), eps=0.0, dtype="f32"), base)
    x = torch.stack([u, torch.zeros_like(u), u, u]).cuda()
    x[2, 0, 0], x[3, -1, -1] = float("nan"), float("inf")
    for eps in (0.0, 1e-7):
        got = muon.orthogonalize(x, eps=eps, dtype="f32")
        assert torch.isfinite(got[0]).all() and (got[1] == 0).all() and torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    assert torch.equal(muon.orthogonalize(x, eps=0.0, dtype="f32")[0], base)


def test_empty():
    for shape in ((0, 4), (4, 0), (0, 3, 3), (2, 0, 3)):
        assert muon.orthogonalize(torch.empty(shape).cuda()).shape == shape


MATRICES = [(0, 40, 70), (2800, 64, 64), (6896, 130, 20), (9496 + 8, 1, 50), (9560, 90, 1), (9656, 300, 200)]
N_FLAT = 9656 + 60000 + 8


def _state(K, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    w, m = torch.randn(N_FLAT, generator=gen), torch.randn(N_FLAT, generator=gen) * 1e-3
    grads = (torch.randn(1, N_FLAT, generator=gen) + torch.randn(K, N_FLAT, generator=gen)) * 1e-3
    return w, m, grads.to(dtype)


def _scaled(matrices):
    return [(o, r, c, muon.spectral_scale(r, c)) for o, r, c in matrices]


def _check_step(w, m, old_w, old_m, grads, matrices, **kw):
    want_w, want_m, tols = ref.step(old_w, old_m, grads, matrices, **kw)
    gm = grads.double().abs().mean(dim=0) + old_m.double().abs()
    # K sums, the division, one operation with the momentum
    assert ((m.double().cpu() - want_m).abs() <= (grads.shape[0] + 3) * 2.0 ** -24 * gm).all()
    inside = torch.zeros(N_FLAT, dtype=torch.bool)
    for (o, r, c, _), tol in zip(matrices, tols):
        at = slice(o, o + r * c)
        inside[at] = True
        d = float((w.double().cpu()[at] - want_w[at]).norm())
        assert d <= tol, f"{r} x {c}: {d:.3g} off, {tol:.3g} allowed"
    assert torch.equal(w.cpu()[~inside], old_w[~inside]) and torch.equal(m.cpu()[~inside], old_m[~inside])


@pytest.mark.parametrize("K,dtype", [(1, F), (3, B), (8, B), (5, F)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_steps(K, dtype, nesterov):
    """Two steps, the second at another rate; the rest of the buffers untouched."""
    w, m, grads = _state(K, dtype, K)
    wc, mc = w.cuda(), m.cuda()
    kw = {"momentum": 0.9, "weight_decay": 0.1, "nesterov": nesterov}
    opt = muon.Muon(MATRICES, wc, mc, K, grad_dtype="f32" if dtype is F else "bf16", lr=0.05, **kw)
    opt.step(grads.cuda())
    _check_step(wc, mc, w, m, grads, _scaled(MATRICES), lr=0.05, **kw)
    w, m = wc.cpu(), mc.cpu()
    _, _, grads = _state(K, dtype, K + 100)
    opt.set_lr(0.002)
    stack = torch.zeros(K, N_FLAT + 64, dtype=dtype)         # rows that lie apart
    stack[:, :N_FLAT] = grads
    opt.step(stack.cuda())
    _check_step(wc, mc, w, m, grads, _scaled(MATRICES), lr=0.002, **kw)
    opt.close()


def test_step_options():
    w, m, grads = _state(2, F, 9)
    matrices = [(0, 40, 70, 0.0), (2800, 64, 64, 3.0)]
    wc, mc = w.cuda(), m.cuda()
    kw = {"momentum": 0.0, "weight_decay": 0.0, "nesterov": True, "steps": 3, "eps": 1e-5,
          "coefficients": (2.0, -1.5, 0.5)}
    opt = muon.Muon(matrices, wc, mc, 2, lr=0.1, **kw)
    opt.step(grads.cuda())
    _check_step(wc, mc, w, m, grads, matrices, lr=0.1, **kw)
    assert torch.equal(wc[:2800].cpu(), w[:2800])            # scale 0
    none = muon.Muon([], wc, mc, 2)
    before = wc.clone()
    none.step(grads.cuda())
    assert torch.equal(wc, before)


def test_many_matrices_of_every_tile():
    """Enough work for the largest tiles, beside matrices that fill none."""
    shapes = [(2300, 2100), (2048, 2500), (2600, 1030), (3, 5), (70, 2000)]
    matrices, o = [], 0
    for r, c in shapes:
        matrices.append((o, r, c))
        o += -(-r * c // 8) * 8
    w, m = torch.zeros(o).cuda(), torch.zeros(o).cuda()
    grads = torch.zeros(1, o)
    want = torch.zeros(o)
    for (at, r, c) in matrices:
        u, x = _permutation(r, c, 5)
        grads[0, at:at + r * c], want[at:at + r * c] = u.reshape(-1), x.reshape(-1)
    opt = muon.Muon([(at, r, c, 1.0) for at, r, c in matrices], w, m, 1, lr=1.0, momentum=0.5, nesterov=False,
                    steps=1, coefficients=DYADIC, eps=0.0)
    opt.step(grads.cuda())
    assert torch.equal(w.cpu(), -want) and torch.equal(m.cpu(), grads[0])


def test_streams_and_graphs():
    w, m, grads = _state(2, B, 20)
    wc, mc, gc = w.cuda(), m.cuda(), grads.cuda()
    opt = muon.Muon(MATRICES, wc, mc, 2, grad_dtype="bf16", lr=0.03)
    opt.step(gc)
    opt.step(gc)
    want = wc.clone(), mc.clone()
    side = torch.cuda.Stream()
    wc.copy_(w)
    mc.copy_(m)
    opt.step(gc)
    side.wait_stream(torch.cuda.current_stream())
    opt.step(gc, stream=side)                                # waits for the step before
    torch.cuda.synchronize()
    assert torch.equal(wc, want[0]) and torch.equal(mc, want[1])
    x = _random(90, 110, "full", 3).cuda()
    graph, gs = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    opt.step(gc, stream=gs)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=gs):
        opt.step(gc)
        o = muon.orthogonalize(x)
    w2, m2 = w.cuda(), m.cuda()
    eager = muon.Muon(MATRICES, w2, m2, 2, grad_dtype="bf16", lr=0.03)
    wc.copy_(w)
    mc.copy_(m)
    for seed in (21, 22, 23):
        gc.copy_(_state(2, B, seed)[2])
        x.copy_(_random(90, 110, "full", seed))
        if seed == 23:
            opt.set_lr(0.001)
            eager.set_lr(0.001)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager.step(gc)
        assert torch.equal(wc, w2) and torch.equal(mc, m2) and torch.equal(o, muon.orthogonalize(x))


def test_binding_refuses():
    x = torch.zeros(4, 8).cuda()
    for args, kw in (((x.half(),), {}), ((x[0],), {}), ((x,), {"out": x[:3]}), ((x,), {"dtype": "fp8"}),
                     ((x,), {"out": torch.zeros(8, 4).cuda().t()}), ((x,), {"coefficients": [(1.0, 0.0, 0.0)] * 2})):
        with pytest.raises(ValueError):
            muon.orthogonalize(*args, **kw)
    with pytest.raises(ags.AGSError):
        muon.orthogonalize(x, out=x)                         # in place
    with pytest.raises(ags.AGSError):
        muon.orthogonalize(x, steps=0)
    w, m = torch.zeros(64).cuda(), torch.zeros(64).cuda()
    for args, kw in ((([(0, 4, 8)], w, m[:32], 1), {}), (([(0, 4, 8)], w.bfloat16(), m, 1), {}),
                     (([(0, 4, 8)], w, m, 1), {"grad_dtype": "f16"})):
        with pytest.raises(ValueError):
            muon.Muon(*args, **kw)
    opt = muon.Muon([(0, 4, 8)], w, m, 2)
    for g in (torch.zeros(1, 64).cuda(), torch.zeros(2, 64, dtype=B).cuda(), torch.zeros(2, 64)):
        with pytest.raises(ValueError):
            opt.step(g)
    for g in (torch.zeros(2, 56).cuda(), torch.zeros(2, 68).cuda()):
        with pytest.raises(ags.AGSError):
            opt.step(g)
    with pytest.raises(ags.AGSError):
        opt.set_lr(-1.0)
