"""Gated products and orthogonalised updates of elements that lie beyond 2^32 of
their buffers: by row strides, by many rows, by a matrix's place."""
import pytest
import torch

import test_gpu_glu as gated

pytestmark = pytest.mark.gpu

from paper_2603_18112_amd import glu, muon  # noqa: E402

F, B = torch.float32, torch.bfloat16


def _spread(t, stride):
    """t's rows `stride` elements apart."""
    rows, cols = t.shape
    out = torch.as_strided(torch.empty((rows - 1) * stride + cols, dtype=t.dtype, device="cuda"), (rows, cols), (stride, 1))
    out.copy_(t)
    return out


@pytest.mark.parametrize("rows,stride", [(5, (1 << 30) + 64),        # few rows, copied first
                                         (1060, 1 << 22)])           # read where they lie
def test_gated_rows_far_apart(rows, stride):
    x, gate, up, dh = gated._random(rows, 40, 128)
    w = glu.Weight(gate.cuda(), up.cuda())
    near = glu.gated_linear(x.cuda(), w, save=True)
    grads = glu.gated_linear_backward(dh.cuda(), x.cuda(), w, saved=near[1])
    again = glu.gated_linear_backward(dh.cuda(), x.cuda(), w)
    xs = _spread(x, stride)
    far = glu.gated_linear(xs, w, save=True)
    assert all(torch.equal(a, b) for a, b in zip(far, near))
    ds = _spread(dh, stride)
    got = glu.gated_linear_backward(ds, xs, w, saved=far[1])
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
    got = glu.gated_linear_backward(ds, xs, w)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_gated_weight_gradients_far_apart():
    x, gate, up, dh = gated._random(70, 1060, 64)
    w = glu.Weight(gate.cuda(), up.cuda())
    want = glu.gated_linear_backward(dh.cuda(), x.cuda(), w)
    zero = torch.zeros(1060, 64, dtype=B)
    a, b = _spread(zero, 1 << 22), _spread(zero, 1 << 22)
    glu.gated_linear_backward(dh.cuda(), x.cuda(), w, dgate=a, dup=b, need_dx=False)
    assert torch.equal(a, want[1]) and torch.equal(b, want[2])


def test_gated_many_rows():
    """saved and the gradients between the passes beyond 2^32 bytes; the last rows
    against the same rows by themselves (tiles of another size add in the same order
    over 64 columns or differ within the bounds)."""
    rows, n, k, last = 80000, 10000, 64, 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, k, generator=gen, device="cuda").to(B)
    dh = torch.randn(rows, n, generator=gen, device="cuda").to(B)
    gate, up = (torch.randn(n, k, generator=gen, device="cuda").mul(0.19).to(B) for _ in range(2))
    w = glu.Weight(gate, up)
    h, saved = glu.gated_linear(x, w, save=True)
    assert saved.numel() > 1 << 32
    dx, dgate, dup = glu.gated_linear_backward(dh, x, w, saved=saved, dw_dtype="f32")
    want = gated._results(x[-last:].cpu(), gate.cpu(), up.cpu(), dh[-last:].cpu(), "silu", True)
    gated._within(h[-last:], *want[0], "h")
    gated._within(dx[-last:], *want[1], "dx")
    # a weight's gradients over all rows: those of pieces, added in 64 bits
    parts = [torch.zeros(n, k, dtype=torch.float64, device="cuda") for _ in range(2)]
    for r in range(0, rows, 8000):
        piece = slice(r, r + 8000)
        got = glu.gated_linear_backward(dh[piece], x[piece], w, saved=saved[piece], dw_dtype="f32", need_dx=False)
        for p, g in zip(parts, got[1:]):
            p += g
    for p, g in zip(parts, (dgate, dup)):
        # Partial sums of r random terms are about sqrt(r) of one; were each of `rows`
        # additions to lose a step (2 U) of its sum the same way, 4/3 U rows sqrt(rows) were lost
        # of a result of sqrt(rows).
        assert float((g.double() - p).norm() / p.norm()) <= 2 * 2.0 ** -24 * rows


def test_matrices_far_apart():
    us = torch.stack(_cases(3, 50, 70))
    near = muon.orthogonalize(us.to(B).cuda(), dtype="f32")
    each = (1 << 31) + 64
    x = torch.as_strided(torch.empty(2 * each + 50 * 70, dtype=B, device="cuda"), (3, 50, 70), (each, 70, 1))
    x.copy_(us)
    out = torch.as_strided(torch.empty(2 * each + 50 * 70, dtype=F, device="cuda"), (3, 50, 70), (each, 70, 1))
    assert torch.equal(muon.orthogonalize(x, out=out), near)
    assert torch.equal(muon.orthogonalize(_spread(us[1].to(B), 1 << 27), dtype="f32"), near[1])


def _cases(count, rows, cols):
    gen = torch.Generator().manual_seed(7)
    return [torch.randn(rows, cols, generator=gen) for _ in range(count)]


def test_a_matrix_behind_2_32_elements():
    u, v = _cases(2, 60, 90)
    at, size = (1 << 32) + 64, 60 * 90
    w, m = (torch.empty(at + size + 8, device="cuda") for _ in range(2))
    grads = torch.empty(2, at + size + 8, dtype=B, device="cuda")
    small_w, small_m = torch.zeros(2 * size, device="cuda"), torch.zeros(2 * size, device="cuda")
    small_g = torch.empty(2, 2 * size, dtype=B, device="cuda")
    for i, (place, t) in enumerate(((0, u), (at, v))):
        for b in (w, m):
            b[place:place + size] = 0.0
        grads[:, place:place + size] = t.reshape(-1).to(B).cuda()
        small_g[:, i * size:(i + 1) * size] = t.reshape(-1).to(B).cuda()
    one = muon.Muon([(0, 60, 90), (at, 60, 90)], w, m, 2, grad_dtype="bf16", lr=0.1)
    two = muon.Muon([(0, 60, 90), (size, 60, 90)], small_w, small_m, 2, grad_dtype="bf16", lr=0.1)
    one.step(grads)
    two.step(small_g)
    for i, place in enumerate((0, at)):
        assert torch.equal(w[place:place + size], small_w[i * size:(i + 1) * size])
        assert torch.equal(m[place:place + size], small_m[i * size:(i + 1) * size])
