"""Layer norm of rows whose mean is far above their spread, constant rows among
them: the differences from the mean must not hold the mean's rounding.

U is half a step of fp32.  The kernels take the mean in 64 bits (D additions, 2^-53 each) as
two fp32 numbers, whose sum is within 2^-48 of it; the first difference's rounding is U of
itself and 2^-48 of the mean, the second's U of itself.
"""
import pytest
import torch

import norm_reference as ref

pytestmark = pytest.mark.gpu

from paper_2603_18112_amd import norm  # noqa: E402

F, B = torch.float32, torch.bfloat16
U = 2.0 ** -24
VALUES = (10000.1, 123456.7, 1000000.3, -0.1, 3.3e-30, -2.7e37, 1e-40)
COLS = (1, 3, 100, 513, 1000, 1025, 2049, 4096, 4097, 8193, 16385, 20000, 32769, 40000)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", [F, B])
def test_constant_rows(cols, dtype):
    x = torch.tensor(VALUES)[:, None].expand(len(VALUES), cols).contiguous().to(dtype)
    gen = torch.Generator().manual_seed(cols)
    w, b = torch.randn(cols, generator=gen), torch.randn(cols, generator=gen)
    y, saved = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), eps=1e-5, dtype="f32", save=True)
    assert torch.equal(y.cpu(), b.expand(len(VALUES), cols))
    assert torch.equal(saved[0].cpu(), x[:, 0].float())
    # eps to fp32, root, reciprocal
    assert ((saved[1].double().cpu() * 1e-5 ** 0.5 - 1).abs() <= 3 * U).all()
    dx, dw, _ = norm.layer_norm_backward(x.cuda(), x.cuda(), saved, w.cuda())
    assert (dw == 0).all()


@pytest.mark.parametrize("cols", COLS[2:])
@pytest.mark.parametrize("mean,spread", [(1000.1, 1.0), (1.0e6, 1.0), (-3.0e5, 0.3), (2.0e12, 3.0e6)])
def test_means_above_the_spread(cols, mean, spread):
    gen = torch.Generator().manual_seed(cols)
    x = (mean + spread * torch.randn(5, cols, generator=gen, dtype=torch.float64)).float()
    w, b = torch.randn(cols, generator=gen), torch.randn(cols, generator=gen)
    y, saved = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), save=True)
    xd, D = x.double(), ref.depth(cols)
    mu = xd.mean(dim=1, keepdim=True)
    d = xd - mu
    rstd = (d.square().mean(dim=1, keepdim=True) + 1e-5).rsqrt()
    z = d * rstd
    e_d = (D * 2.0 ** -53 + 3 * 2.0 ** -48) * mu.abs()
    e_rstd = 0.5 * ((D + 5) * U + 4 * U + (e_d * rstd).square() + 2 * e_d * rstd) + 3 * U
    e_y = w.double().abs() * (z.abs() * (e_rstd + 3 * U) + e_d * rstd) * 1.001 + (z * w + b).abs() * 2 * U
    assert ((y.double().cpu() - (z * w + b)).abs() <= e_y).all()
    assert ((saved[0].double().cpu() - mu[:, 0]).abs() <= 1.001 * U * mu[:, 0].abs()).all()
    assert ((saved[1].double().cpu() / rstd[:, 0] - 1).abs() <= e_rstd.max() + U).all()


@pytest.mark.parametrize("cols", COLS[2:])
@pytest.mark.parametrize("one", [1.0, 200.0, -3.0e33])
def test_bf16_rows_of_one_value_but_for_few(cols, one):
    """The least spread that bf16 has: neighbours of 8 bits.  hi and lo hold the mean to
    2^-48 (sums of up to 24 bits are exact); the variance is the squares' less lo's."""
    x = torch.full((3, cols), one, dtype=torch.float64)
    for row, count in enumerate((1, 3, cols // 3)):
        x[row, 5:5 + 2 * count:2] = one * (1 + 2.0 ** -7)
    x = x.to(B)
    y, saved = norm.layer_norm(x.cuda(), eps=0.0, dtype="f32", save=True)
    xd, D = x.double(), ref.depth(cols)
    mu = xd.mean(dim=1, keepdim=True)
    d = xd - mu
    rstd = d.square().mean(dim=1, keepdim=True).rsqrt()
    z = d * rstd
    e_d = 2.0 ** -46 * mu.abs()
    e_rstd = 0.5 * ((D + 9) * U + 2.0 ** -48 * (mu * rstd).square() + 2 * e_d * rstd) + 3 * U
    assert ((y.double().cpu() - z).abs() <= (z.abs() * (e_rstd + 4 * U) + e_d * rstd) * 1.001).all()
    assert ((saved[1].double().cpu() / rstd[:, 0] - 1).abs() <= e_rstd[:, 0] + U).all()


@pytest.mark.parametrize("cols", [70, 1000, 3000, 8000, 20000, 40000])
@pytest.mark.parametrize("size,eps", [(1.0e18, 1e-5), (3.0e25, 1e-5), (2.0e37, 0.0), (1.0e-25, 0.0), (1.0e-30, 1e-34)])
@pytest.mark.parametrize("dtype", [F, B])
def test_squares_outside_fp32(cols, size, eps, dtype):
    """Beside a row inside.  The scale is a power of two: the same roundings (a square below
    2^-126 loses bits, 2^-150 of a sum above 2^-118)."""
    gen = torch.Generator().manual_seed(cols)
    x = torch.randn(5, cols, generator=gen)
    x[:4] *= size
    x[1] += 3 * size
    x = x.to(dtype)
    w, b = torch.randn(cols, generator=gen), torch.randn(cols, generator=gen)
    y, saved = norm.layer_norm(x.cuda(), w.cuda(), b.cuda(), eps=eps, dtype="f32", save=True)
    for got, want, tol in zip((y, *saved), *ref.forward(x, w, b, eps, F)):
        assert torch.isfinite(got).all() and ((got.double().cpu() - want).abs() <= tol + want.abs() * U).all()


@pytest.mark.parametrize("cols", [200, 5000, 40000])
@pytest.mark.parametrize("dtype", [F, B])
def test_nonfinite_rows(cols, dtype):
    gen = torch.Generator().manual_seed(cols)
    x, dy = (torch.randn(4, cols, generator=gen).to(dtype) for _ in range(2))
    good = norm.layer_norm(x.cuda(), save=True)
    x[0, 3], x[1, cols - 1], x[3, 0] = float("inf"), float("nan"), -float("inf")
    y, saved = norm.layer_norm(x.cuda(), save=True)
    assert torch.isnan(y[[0, 1, 3]]).all() and torch.equal(y[2], good[0][2])
    dx, dw, db = norm.layer_norm_backward(dy.cuda(), x.cuda(), saved)
    assert torch.isnan(dx[[0, 1, 3]]).all() and torch.isfinite(dx[2]).all()
    assert torch.isnan(dw).all() and torch.isfinite(db).all()


def test_a_single_element_beside_large_ones():
    """A first element, a last one and one in the middle far above the others."""
    gen = torch.Generator().manual_seed(1)
    for at in (0, 777, 2047):
        for dtype in (F, B):
            x = torch.randn(3, 2048, generator=gen)
            x[:, at] = torch.tensor([1.0e6, -3.0e4, 500.0])
            x = x.to(dtype)
            y, saved = norm.layer_norm(x.cuda(), dtype="f32", save=True)
            (ry, rm, rr), (ey, em, er) = ref.forward(x, None, None, 1e-5, F)
            for got, want, tol in ((y, ry, ey), (saved[0], rm, em), (saved[1], rr, er)):
                assert ((got.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("cols", [100, 5000, 40000])
def test_eps_below_the_smallest_fp32_number(cols):
    """Constant rows have z = 0 with any eps above zero."""
    x = torch.full((3, cols), 7.0).cuda()
    for eps in (1e-38, 1e-46, 1e-300):
        y, saved = norm.layer_norm(x, eps=eps, save=True)
        assert (y == 0).all() and torch.isfinite(saved).all()
        dx, dw, db = norm.layer_norm_backward(torch.zeros_like(x), x, saved)
        assert (dx == 0).all() and (dw == 0).all()
