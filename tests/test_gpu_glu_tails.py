"""GELU of hidden units far below zero, in fp32: g (1 + erf(g / sqrt 2)) / 2 is a
small number there, and rounded like any other."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2603_18112_amd import glu  # noqa: E402

U = 2.0 ** -24


@pytest.mark.parametrize("rows", [1, 20, 40, 300])       # few rows, tiles
def test_small_results_keep_their_bits(rows):
    """g is exact (one product).  The function in fp32, relative: the fit 1.5 U, 1 / x and 2^x an
    ulp (2 U) each, seven operations of the polynomial at a condition of 1.8 and four
    products, 20 U in all; the exponent -g g / 2, of two roundings and a constant's (2.6 U), costs
    1.3 g g U."""
    g = torch.linspace(-12.5, 6.0, 700).bfloat16()
    one = torch.ones_like(g)
    w = glu.Weight(g[:, None].cuda(), one[:, None].cuda())
    x = torch.ones(rows, 1, dtype=torch.bfloat16).cuda()
    h = glu.gated_linear(x, w, act="gelu", dtype="f32").double().cpu()
    gd = g.double()
    want = 0.5 * gd * torch.erfc(-gd / math.sqrt(2.0))
    assert ((h - want).abs() <= (20 + 1.4 * gd * gd) * U * want.abs() + 2.0 ** -126).all()
    # rounded once more to bf16
    h = glu.gated_linear(x, w, act="gelu").double().cpu()
    assert ((h - want).abs() <= (2.0 ** -8 + (22 + 1.4 * gd * gd) * U) * want.abs() + 2.0 ** -126).all()
    # du = dh act(g) in bf16, dgate's column is dg: act' within 24 U of its two terms, whose second is
    # |g| times the density
    dh = torch.ones(rows, 700, dtype=torch.bfloat16).cuda()
    _, dgate, dup = glu.gated_linear_backward(dh[:1], x[:1], w, act="gelu", dw_dtype="f32")
    assert ((dup[:, 0].double().cpu() - want).abs() <= (2.0 ** -8 + (22 + 1.4 * gd * gd) * U) * want.abs() + 2.0 ** -126).all()
    c, e = 0.5 * torch.erfc(-gd / math.sqrt(2.0)), torch.exp(-0.5 * gd * gd) / math.sqrt(2.0 * math.pi)
    d = c + gd * e
    tol = 2.0 ** -8 * d.abs() + (24 + 1.4 * gd * gd) * U * 1.01 * (c + (gd * e).abs()) + 2.0 ** -126
    assert ((dgate[:, 0].double().cpu() - d).abs() <= tol).all()
