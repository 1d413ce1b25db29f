"""libags layer norm on the host: the binding's names, workspace sizes and
argument checks (no GPU; only calls that fail before any HIP call), and the
reference the GPU tests use."""
import ctypes
import os
import re

import pytest
import torch

import norm_reference as ref
from paper_2603_18112_amd import _build, ags, norm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, Y, Z, V, W, S, P, Q = (0x1000000000 * (i + 1) for i in range(8))       # never dereferenced
F, B = ags.AGS_F32, ags.AGS_BF16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB):
        _build.build()
    return norm._lib()


def test_header_declares_the_binding_names():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ags_norm.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ags_[a-z_]+)\s*\(", text))) == sorted(norm.EXPORTS)


def _raises(status, f, *args, **kw):
    with pytest.raises(ags.AGSError) as e:
        f(*args, **kw)
    assert e.value.status == status and ags.ags_last_error(None), e.value


def test_workspace(lib):
    assert norm.ags_layer_norm_backward_workspace(0, 10) == 0
    assert norm.ags_layer_norm_backward_workspace(10, 0) == 0
    for rows, cols in ((1, 1), (1000, 512), (1 << 20, 4096), (7, 1 << 24), (1 << 30, 16385)):
        n = norm.ags_layer_norm_backward_workspace(rows, cols)
        assert n % (8 * cols) == 0 and 8 * cols <= n <= 8 * cols * 2048
    with pytest.raises(ags.AGSError):
        norm.ags_layer_norm_backward_workspace(-1, 4)
    assert lib.ags_layer_norm_backward_workspace(4, 4, ctypes.POINTER(ctypes.c_size_t)()) == ags.AGS_E_ARG


def test_forward_refuses(lib):
    f = norm.ags_layer_norm
    good = [X, B, 4, 64, 64, W, V, F, 1e-5, Y, B, 64, S]

    def bad(status, **change):
        args = list(good)
        for i, v in change.items():
            args[int(i[1:])] = v
        _raises(status, f, *args)

    for i in (1, 7, 10):
        bad(ags.AGS_E_ARG, **{f"a{i}": 2})                       # types
    bad(ags.AGS_E_ARG, a8=-1.0)
    bad(ags.AGS_E_ARG, a8=float("nan"))
    bad(ags.AGS_E_ARG, a8=float("inf"))
    bad(ags.AGS_E_ARG, a2=-1)
    bad(ags.AGS_E_LAYOUT, a3=(1 << 24) + 1, a4=1 << 25, a11=1 << 25)
    bad(ags.AGS_E_LAYOUT, a2=(1 << 40) + 1)
    bad(ags.AGS_E_ARG, a0=None)
    bad(ags.AGS_E_ARG, a9=None)
    bad(ags.AGS_E_ARG, a4=63)
    bad(ags.AGS_E_ARG, a11=63)
    bad(ags.AGS_E_ARG, a4=1 << 62)                               # a range that would wrap
    bad(ags.AGS_E_ALIGN, a0=X + 1)
    bad(ags.AGS_E_ALIGN, a5=W + 2)
    bad(ags.AGS_E_ALIGN, a12=S + 2)
    bad(ags.AGS_E_ARG, a9=X + 128)                               # y over x
    bad(ags.AGS_E_ARG, a12=Y + 4)                                # saved over y
    bad(ags.AGS_E_ARG, a9=W)                                     # y over the weight
    f(None, B, 0, 64, 64, W, V, F, 1e-5, None, B, 64, None)      # nothing to do
    f(None, B, 4, 0, 1, None, None, F, 1e-5, None, B, 1, None)


def test_backward_refuses(lib):
    f, ws = norm.ags_layer_norm_backward, norm.ags_layer_norm_backward_workspace(4, 64)
    good = [X, 64, Y, B, 4, 64, 64, S, W, F, Z, 64, V, P, F, 0, Q, ws]

    def bad(status, **change):
        args = list(good)
        for i, v in change.items():
            args[int(i[1:])] = v
        _raises(status, f, *args)

    for i in (3, 9, 14):
        bad(ags.AGS_E_ARG, **{f"a{i}": 7})
    bad(ags.AGS_E_ARG, a15=2)                                    # accumulate
    bad(ags.AGS_E_ARG, a10=None, a12=None, a13=None)             # nothing wanted
    bad(ags.AGS_E_ARG, a0=None)
    bad(ags.AGS_E_ARG, a2=None)
    bad(ags.AGS_E_ARG, a7=None)
    bad(ags.AGS_E_ARG, a1=63)
    bad(ags.AGS_E_ARG, a11=63)
    bad(ags.AGS_E_ALIGN, a12=V + 2)
    bad(ags.AGS_E_ARG, a16=None)                                 # workspace
    bad(ags.AGS_E_ARG, a17=ws - 1)
    bad(ags.AGS_E_ALIGN, a16=Q + 8)
    bad(ags.AGS_E_ARG, a10=X)                                    # dx over dy
    bad(ags.AGS_E_ARG, a13=V + 4)                                # dbias over dweight
    bad(ags.AGS_E_ARG, a16=Z)                                    # workspace over dx
    bad(ags.AGS_E_LAYOUT, a5=1 << 25, a1=1 << 25, a6=1 << 25, a11=1 << 25)
    f(X, 64, Y, B, 0, 64, 64, S, W, F, Z, 64, V, P, F, 1)        # no rows, added: nothing to do
    f(X, 64, Y, B, 4, 0, 64, S, W, F, Z, 64, V, P, F, 0)         # no columns


def test_binding_refuses_without_a_gpu():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA"):
        norm.layer_norm(x)
    with pytest.raises(ValueError, match="gradient"):
        norm.layer_norm(x.requires_grad_())
    with pytest.raises(ValueError, match="differ"):
        norm.layer_norm_backward(x, x[:1], torch.zeros(2, 2))


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 16), (5, 100), (2, 9000)])
def test_reference_against_torch_and_its_bounds(rows, cols):
    gen = torch.Generator().manual_seed(rows * 1000 + cols)
    x = torch.randn(rows, cols, generator=gen) + 3.0
    w, b, dy = (torch.randn(*s, generator=gen) for s in ((cols,), (cols,), (rows, cols)))
    xd, wd, bd = (t.double().requires_grad_() for t in (x, w, b))
    y = torch.nn.functional.layer_norm(xd, (cols,), wd, bd, 1e-5)
    y.backward(dy.double())
    (ry, rm, rr), (ey, em, er) = ref.forward(x, w, b, 1e-5, torch.float32)
    assert torch.allclose(ry, y.detach(), rtol=1e-12, atol=1e-12)
    saved = torch.stack([rm, rr])
    (dx, dw, db), _ = ref.backward(dy, x, saved, w, torch.float32, torch.float32)
    assert torch.allclose(dx, xd.grad, rtol=1e-9, atol=1e-11)
    assert torch.allclose(dw, wd.grad, rtol=1e-9, atol=1e-11) and torch.allclose(db, bd.grad, rtol=1e-9, atol=1e-11)
    # plain fp32 arithmetic stays inside the bounds, and they are no wider than a few hundred steps
    y32 = torch.nn.functional.layer_norm(x, (cols,), w, b, 1e-5)
    assert ((y32.double() - ry).abs() <= ey).all()
    if cols > 1:
        assert (ey <= 2.0 ** -14 * (ry.abs() + w.abs() * 10)).all()
