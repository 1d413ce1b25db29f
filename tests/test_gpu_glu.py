"""Gated products on the GPU: whole numbers, for which every result is exact, and
random ones against 64-bit forms within bounds that follow from the arithmetic.

U is half a step of fp32, H of bf16 (relative).  A sum of n products of bf16
values is off by at most n 2 U times the sum of their magnitudes.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2603_18112_amd import ags, glu  # noqa: E402

F, B = torch.float32, torch.bfloat16
U, H = 2.0 ** -24, 2.0 ** -8
HALF = {F: U, B: H}

# (rows, n, k): single tokens, the ends of the kernel for few rows, one element, sizes
# around each tile's edge, contracted axes cut in parts, whole tiles
SIZES = [(1, 1, 1), (1, 64, 128), (2, 17, 65), (16, 33, 100), (17, 100, 640), (32, 16, 64), (33, 16, 64), (40, 1, 7),
         (64, 32, 64), (65, 33, 129), (100, 500, 70), (129, 65, 1000), (256, 128, 512), (300, 257, 311),
         (70, 48, 8200), (1000, 40, 130), (513, 520, 257), (2048, 1024, 192), (2100, 1100, 520), (3000, 2100, 321)]


def _exact_act(act, g):
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    c = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def _whole(rows, n, k, seed=0):
    """x, gate, up, dh of whole numbers such that |g| is about 128, where both
    activations are g or 0 and their derivatives 1 or 0 exactly, and every product
    and sum is a whole number that its type holds."""
    gen = torch.Generator().manual_seed(seed * 1009 + rows * 31 + n * 17 + k)

    def sparse(r, c, terms):
        v = torch.randint(-1, 2, (r, c), generator=gen).float()
        return v * (torch.rand(r, c, generator=gen) < terms / c)

    x = torch.randint(-1, 2, (rows, k), generator=gen).float()
    x[:, 0] = 1.0
    gate, up = sparse(n, k, 12), sparse(n, k, 40)
    gate[:, 0] = 128.0 * (torch.randint(0, 4, (n,), generator=gen) > 0) * 2 - 128.0
    dh = torch.randint(-1, 2, (rows, n), generator=gen).float()
    g, u = x @ gate.t(), x @ up.t()
    assert (g.abs() >= 105).all() and (g.abs() <= 256).all() and (u.abs() <= 256).all()
    return x, gate, up, dh


def _whole_results(x, gate, up, dh):
    x, gate, up, dh = (t.double() for t in (x, gate, up, dh))
    g, u = x @ gate.t(), x @ up.t()
    a, on = g.clamp(min=0.0), (g > 0).double()
    dg, du = dh * u * on, dh * a
    for s in (dg.abs().t() @ x.abs(), du.abs().t() @ x.abs(), dg.abs() @ gate.abs() + du.abs() @ up.abs()):
        assert s.numel() == 0 or s.max() < 2 ** 24
    return g, u, a * u, dg @ gate + du @ up, dg.t() @ x, du.t() @ x


def _rounded(t, dtype):
    return t.float().to(dtype)          # whole numbers below 2^24: one rounding


@pytest.mark.parametrize("rows,n,k", SIZES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_whole_numbers_are_exact(rows, n, k, act):
    x, gate, up, dh = _whole(rows, n, k)
    g, u, h, dx, dgate, dup = _whole_results(x, gate, up, dh)
    w = glu.Weight(gate.cuda(), up.bfloat16().float().cuda())
    xc, dc = x.bfloat16().cuda(), dh.bfloat16().cuda()
    got, saved = glu.gated_linear(xc, w, act=act, save=True)
    assert torch.equal(got.cpu(), _rounded(h, B))
    assert torch.equal(glu.gated_linear(xc, w, act=act, dtype="f32").cpu(), h.float())
    lines = w.lines
    assert (saved[:, 2 * lines:] == 0).all()         # whole numbers up to 256 need 16 of the 24 bits
    z = saved.cpu()[:, :2 * lines].contiguous().view(B).view(rows, -1, 2, 16)
    assert torch.equal(z[:, :, 0].reshape(rows, -1)[:, :n].double(), g)
    assert torch.equal(z[:, :, 1].reshape(rows, -1)[:, :n].double(), u)
    assert (z[:, :, 0].reshape(rows, -1)[:, n:] == 0).all() and (z[:, :, 1].reshape(rows, -1)[:, n:] == 0).all()
    for s in (saved, None):
        for dt in ("bf16", "f32"):
            got = glu.gated_linear_backward(dc, xc, w, saved=s, act=act, dw_dtype=dt)
            want = _rounded(dx, B), _rounded(dgate, B if dt == "bf16" else F), _rounded(dup, B if dt == "bf16" else F)
            for a, b, what in zip(got, want, ("dx", "dgate", "dup")):
                assert a.dtype == b.dtype and torch.equal(a.cpu(), b), (what, s is None, dt)
    only = glu.gated_linear_backward(dc, xc, w, saved=saved, act=act, need_dw=False)
    assert torch.equal(only[0].cpu(), _rounded(dx, B)) and only[1] is None and only[2] is None
    only = glu.gated_linear_backward(dc, xc, w, saved=saved, act=act, need_dx=False)
    assert only[0] is None and torch.equal(only[1].cpu(), _rounded(dgate, B))


def _random(rows, n, k, seed=0):
    gen = torch.Generator().manual_seed(seed * 1013 + rows * 7 + n * 3 + k)
    x = torch.randn(rows, k, generator=gen).bfloat16()
    gate, up = (torch.randn(n, k, generator=gen).mul(1.5 / math.sqrt(k)).bfloat16() for _ in range(2))
    return x, gate, up, torch.randn(rows, n, generator=gen).bfloat16()


def _results(x, gate, up, dh, act, saved):
    """(h, dx, dgate, dup) in 64 bits and how far each may be off; saved: g and u
    went through 24 bits, 17 of them significant, on the way to the gradients."""
    x, gate, up, dh = (t.double() for t in (x, gate, up, dh))
    k, n, rows = x.shape[1], gate.shape[0], x.shape[0]
    g, u = x @ gate.t(), x @ up.t()
    eg, eu = (2 * U * k * (x.abs() @ w.abs().t()) for w in (gate, up))
    a, da = _exact_act(act, g)
    # |act'| <= 1.13, |act''| <= 0.8; the functions in fp32: within 8 U of |g| (a), of 1 + |g| (da)
    ea = 1.13 * eg + 8 * U * g.abs()
    h = a * u
    e_h = ea * u.abs() + a.abs() * eu + ea * eu + 2 * U * h.abs()
    if saved:
        eg, eu = eg + 2.0 ** -17 * g.abs() * 1.01, eu + 2.0 ** -17 * u.abs() * 1.01
        ea = 1.13 * eg + 8 * U * g.abs()
    eda = 0.8 * eg + 8 * U * (1 + g.abs())
    dg, du = dh * u * da, dh * a
    e_dg = dh.abs() * (eu * da.abs() + u.abs() * eda + eu * eda) + H * dg.abs() * 1.01
    e_du = dh.abs() * ea + H * du.abs() * 1.01
    dx = dg @ gate + du @ up
    e_dx = e_dg @ gate.abs() + e_du @ up.abs() + 2 * U * 2 * n * 1.01 * (dg.abs() @ gate.abs() + du.abs() @ up.abs())
    out = [(h, e_h), (dx, e_dx)]
    for d, e in ((dg, e_dg), (du, e_du)):
        out.append((d.t() @ x, e.t() @ x.abs() + 2 * U * rows * 1.01 * (d.abs().t() @ x.abs())))
    return out


def _within(got, want, tol, what):
    off = (got.double().cpu() - want).abs() - tol - HALF[got.dtype] * want.abs() - HALF[got.dtype] * tol - 1e-38
    assert torch.isfinite(got).all() and (off <= 0).all(), f"{what}: {float(off.max()):.3g} beyond its bound"


@pytest.mark.parametrize("rows,n,k", [(1, 100, 64), (20, 40, 333), (130, 70, 200), (600, 300, 500)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_random_numbers(rows, n, k, act):
    x, gate, up, dh = _random(rows, n, k)
    w = glu.Weight(gate.cuda(), up.cuda())
    h, saved = glu.gated_linear(x.cuda(), w, act=act, save=True)
    for s in (saved, None):
        want = _results(x, gate, up, dh, act, s is not None)
        _within(h, *want[0], "h")
        got = glu.gated_linear_backward(dh.cuda(), x.cuda(), w, saved=s, act=act, dw_dtype="f32")
        for a, b, what in zip(got, want[1:], ("dx", "dgate", "dup")):
            _within(a, *b, what)
    h32 = glu.gated_linear(x.cuda(), w, act=act, dtype="f32")
    _within(h32, *want[0], "h in fp32")
    # in the norm the results are as near as their roundings: bf16's half step is at most
    # 2^-8 of a value, uniform roundings 2^-8 / sqrt 3, two of them one after the other
    for a, b in zip((h32, *got), want):
        assert float((a.double().cpu() - b[0]).norm() / b[0].norm()) < H


def test_gradient_against_differences():
    rows, n, k = 3, 20, 40
    x, gate, up, dh = _random(rows, n, k, 1)
    for act in ("silu", "gelu"):
        def loss(x, gate, up):
            return float((_exact_act(act, x @ gate.t())[0] * (x @ up.t()) * dh.double()).sum())

        w = glu.Weight(gate.cuda(), up.cuda())
        grads = glu.gated_linear_backward(dh.cuda(), x.cuda(), w, act=act, dw_dtype="f32")
        tols = [t[1] for t in _results(x, gate, up, dh, act, False)[1:]]
        for i, at in ((0, (0, 5)), (0, (2, 39)), (1, (19, 3)), (2, (7, 0))):
            step, sides = 1e-4, []
            for sign in (1, -1):
                args = [t.double().clone() for t in (x, gate, up)]
                args[i][at] += sign * step
                sides.append(loss(*args))
            diff = (sides[0] - sides[1]) / (2 * step)
            tol = float(tols[i][at]) + HALF[grads[i].dtype] * abs(diff) + 1e-5 * (1 + abs(diff))
            assert abs(diff - float(grads[i][at])) <= tol


@pytest.mark.parametrize("rows,n,k", [(5, 30, 64), (200, 30, 64), (200, 40, 100)])
def test_strides_shapes_and_neighbours(rows, n, k):
    """Inputs that are slices of wider rows (aligned or not), transposed or of more
    axes; gradients into a replica's row, whose other elements stay."""
    x, gate, up, dh = _whole(rows, n, k, 2)
    g, u, h, dx, dgate, dup = _whole_results(x, gate, up, dh)
    w = glu.Weight(gate.t().contiguous().cuda().t().contiguous(), up.cuda())
    for lead, wide in ((8, 80), (3, 11)):
        buf = torch.full((rows, k + wide), 9.0).bfloat16().cuda()
        xs = buf[:, lead:lead + k]
        xs.copy_(x)
        assert torch.equal(glu.gated_linear(xs, w).cpu(), _rounded(h, B))
        hb = torch.full((rows, n + wide), 9.0).bfloat16().cuda()
        hs = hb[:, lead:lead + n]
        hs.copy_(dh)
        row = torch.full((2 * n * k + 24,), 4.0).cuda()
        dg, du = row[8:8 + n * k].view(n, k), row[8 + n * k + 3:8 + 2 * n * k + 3].view(n, k)
        got = glu.gated_linear_backward(hs, xs, w, dgate=dg, dup=du)
        assert torch.equal(got[0].cpu(), _rounded(dx, B))
        assert torch.equal(dg.cpu(), dgate.float()) and torch.equal(du.cpu(), dup.float())
        assert (row[:8] == 4).all() and (row[8 + n * k:8 + n * k + 3] == 4).all() and (row[8 + 2 * n * k + 3:] == 4).all()
        got = glu.gated_linear_backward(hs, xs, w, dgate=dg, dup=du, accumulate=True, need_dx=False)
        assert torch.equal(dg.cpu(), 2 * dgate.float()) and torch.equal(du.cpu(), 2 * dup.float())
    xt = x.bfloat16().t().contiguous().cuda().t()
    assert torch.equal(glu.gated_linear(xt, w).cpu(), _rounded(h, B))
    x3 = x.bfloat16().view(rows // 5, 5, k).cuda()
    assert torch.equal(glu.gated_linear(x3, w).cpu(), _rounded(h, B).view(rows // 5, 5, n))
    d3 = glu.gated_linear_backward(dh.bfloat16().view(rows // 5, 5, n).cuda(), x3, w, need_dw=False)[0]
    assert torch.equal(d3.cpu(), _rounded(dx, B).view(rows // 5, 5, k))
    one = dh[:1].expand(rows, n)
    want = _whole_results(x, gate, up, one)
    got = glu.gated_linear_backward(one.bfloat16().cuda()[:1].expand(rows, n), x3.view(rows, k), w, dw_dtype=F)
    assert torch.equal(got[0].cpu(), _rounded(want[3], B)) and torch.equal(got[1].cpu(), want[4].float())
    # through the C-ABI: rows of h and dx that lie apart
    s = torch.cuda.current_stream().cuda_stream
    out = torch.full((rows, n + 5), 3.0).cuda()
    xc = x.bfloat16().cuda()
    ws = torch.empty(glu.ags_glu_backward_workspace(rows, n, k) + 16, dtype=torch.uint8, device="cuda")
    glu.ags_glu_forward(xc.data_ptr(), rows, k, w.c, 0, out.data_ptr(), ags.AGS_F32, n + 5, None, ws.data_ptr(),
                        ws.numel(), s)
    assert torch.equal(out[:, :n].cpu(), h.float()) and (out[:, n:] == 3).all()
    dxo, dc = torch.full((rows, k + 3), 3.0).bfloat16().cuda(), dh.bfloat16().cuda()
    glu.ags_glu_backward(dc.data_ptr(), n, xc.data_ptr(), rows, k, None, w.c, 0, dxo.data_ptr(), k + 3, None, None,
                         ags.AGS_BF16, 1, 0, ws.data_ptr(), ws.numel(), s)
    assert torch.equal(dxo[:, :k].cpu(), _rounded(dx, B)) and (dxo[:, k:] == 3).all()


def test_weight_updates_in_place():
    x, gate, up, dh = _whole(40, 30, 50, 3)
    w = glu.Weight(torch.randn(30, 50).cuda(), torch.randn(30, 50).cuda())
    p = w.data.data_ptr()
    flat = torch.cat([gate.flatten(), torch.zeros(3), up.flatten()]).cuda()
    w.update(flat[:1500].view(30, 50), flat[1503:].view(30, 50))
    assert w.data.data_ptr() == p
    assert torch.equal(glu.gated_linear(x.bfloat16().cuda(), w).cpu(), _rounded(_whole_results(x, gate, up, dh)[2], B))
    m = torch.randn(30, 50).cuda()
    w.update(m, m)
    z = w.data.view(-1, 2, 16, 64)              # one panel to 32 lines: k is below 64
    assert torch.equal(z[:, 0].reshape(-1, 64)[:30, :50], m.bfloat16()) and torch.equal(z[:, 0], z[:, 1])
    assert (z[:, 0].reshape(-1, 64)[30:] == 0).all() and (z[:, 0].reshape(-1, 64)[:, 50:] == 0).all()


def test_empty():
    e = torch.empty
    w = glu.Weight(torch.ones(5, 8).cuda(), torch.ones(5, 8).cuda())
    x, dh = e(0, 8, dtype=B).cuda(), e(0, 5, dtype=B).cuda()
    h, saved = glu.gated_linear(x, w, save=True)
    assert h.shape == (0, 5)
    dx, dg, du = glu.gated_linear_backward(dh, x, w, saved=saved)
    assert dx.shape == (0, 8) and (dg == 0).all() and (du == 0).all()
    dg.fill_(2.0)
    glu.gated_linear_backward(dh, x, w, dgate=dg, dup=du, accumulate=True)
    assert (dg == 2).all()
    w = glu.Weight(e(0, 8).cuda(), e(0, 8).cuda())
    x = torch.ones(4, 8, dtype=B).cuda()
    assert glu.gated_linear(x, w).shape == (4, 0)
    dx, dg, du = glu.gated_linear_backward(e(4, 0, dtype=B).cuda(), x, w)
    assert (dx == 0).all() and dg.shape == (0, 8)
    w = glu.Weight(e(5, 0).cuda(), e(5, 0).cuda())
    assert (glu.gated_linear(e(4, 0, dtype=B).cuda(), w) == 0).all()
    assert (glu.gated_linear(e(400, 0, dtype=B).cuda(), w) == 0).all()
    dx, dg, du = glu.gated_linear_backward(torch.ones(4, 5, dtype=B).cuda(), e(4, 0, dtype=B).cuda(), w)
    assert dx.shape == (4, 0) and dg.shape == (5, 0)


@pytest.mark.parametrize("rows,k", [(9, 64), (300, 100)])
def test_nonfinite_values_stay_in_their_rows(rows, k):
    """Padding beside a row that holds them included: what pads k or n must not
    spread them."""
    n = 20
    x, gate, up, dh = _random(rows, n, k, 4)
    w = glu.Weight(gate.cuda(), up.cuda())
    good = glu.gated_linear(x.cuda(), w)
    gx = glu.gated_linear_backward(dh.cuda(), x.cuda(), w, need_dw=False)[0]
    x[3] = float("nan")
    x[rows - 1, k - 1] = float("inf")
    h = glu.gated_linear(x.cuda(), w)
    keep = [i for i in range(rows) if i not in (3, rows - 1)]
    assert torch.isnan(h[3]).all() and not torch.isfinite(h[rows - 1]).all()
    assert torch.equal(h[keep], good[keep])
    dx = glu.gated_linear_backward(dh.cuda(), x.cuda(), w, need_dw=False)[0]
    assert torch.isnan(dx[3]).all() and torch.equal(dx[keep], gx[keep])


def test_streams_and_graphs():
    x, gate, up, dh = (t.cuda() for t in _random(150, 80, 200, 5))
    w = glu.Weight(gate, up)
    want = glu.gated_linear(x, w, save=True)
    grads = glu.gated_linear_backward(dh, x, w, saved=want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = glu.gated_linear(x, w, save=True)
        back = glu.gated_linear_backward(dh, x, w, saved=got[1])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and all(torch.equal(p, q) for p, q in zip(back, grads))
    graph, few = torch.cuda.CUDAGraph(), x[:3].clone()
    with torch.cuda.graph(graph):
        w.update(gate, up)
        h, saved = glu.gated_linear(x, w, save=True)
        back = glu.gated_linear_backward(dh, x, w, saved=saved)
        token = glu.gated_linear(few, w, act="gelu")
    for seed in (6, 7, 8):
        for t, v in zip((x, gate, up, dh), _random(150, 80, 200, seed)):
            t.copy_(v)
        few.copy_(x[:3])
        graph.replay()
        torch.cuda.synchronize()
        e = glu.Weight(gate, up)
        eh, es = glu.gated_linear(x, e, save=True)
        eb = glu.gated_linear_backward(dh, x, e, saved=es)
        assert torch.equal(h, eh) and all(torch.equal(p, q) for p, q in zip(back, eb))
        assert torch.equal(token, glu.gated_linear(few, e, act="gelu"))


def test_binding_refuses():
    x, m = torch.zeros(4, 8, dtype=B).cuda(), torch.zeros(5, 8).cuda()
    w = glu.Weight(m, m)
    for args in ((m, m[:3]), (m, m.bfloat16()), (m.half(), m.half()), (m, m.cpu()), (m.t(), m.t())):
        with pytest.raises(ValueError):
            glu.Weight(*args)
    with pytest.raises(ValueError):
        w.update(m[:, :7], m[:, :7])
    for args, kw in (((x.float(), w), {}), ((x[:, :7], w), {}), ((x, w), {"act": "relu"}), ((x, w), {"dtype": "fp8"}),
                     ((x.float().requires_grad_().bfloat16(), w), {})):
        with pytest.raises(ValueError):
            glu.gated_linear(*args, **kw)
    dh, big = torch.zeros(4, 5, dtype=B).cuda(), torch.zeros(5, 8).cuda()
    for args, kw in (((dh[:3], x, w), {}), ((dh, x, w), {"saved": dh}), ((dh, x, w), {"dgate": big}),
                     ((dh, x, w), {"dgate": big, "dup": big.bfloat16()}), ((dh, x, w), {"accumulate": True}),
                     ((dh, x, w), {"dgate": big, "dup": big, "need_dw": False}), ((dh.float(), x, w), {}),
                     ((dh, x, w), {"dgate": big, "dup": torch.zeros(5, 9).cuda()[:, :8]})):
        with pytest.raises(ValueError):
            glu.gated_linear_backward(*args, **kw)
    with pytest.raises(ags.AGSError):
        glu.gated_linear_backward(dh, x, w, dgate=big, dup=big)          # the same memory twice
