"""libags orthogonalised updates on the host: the binding's names, sizes and
argument checks (no GPU; only calls that fail before any HIP call), and the
reference the GPU tests use."""
import ctypes
import os
import re

import pytest
import torch

import muon_reference as ref
from paper_2603_18112_amd import _build, ags, muon

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, Y, Z, W = (0x1000000000 * (i + 1) for i in range(4))       # never dereferenced
F, B = ags.AGS_F32, ags.AGS_BF16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB):
        _build.build()
    return muon._lib()


def test_header_declares_the_binding_names():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ags_muon.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ags_[a-z_]+)\s*\(", text))) == sorted(muon.EXPORTS)
    assert ctypes.sizeof(muon.ags_muon_schedule) == 24 and ctypes.sizeof(muon.ags_muon_matrix) == 32
    assert ctypes.sizeof(muon.ags_muon_config) == 80


def _raises(status, f, *args, **kw):
    with pytest.raises(ags.AGSError) as e:
        f(*args, **kw)
    assert e.value.status == status and ags.ags_last_error(None), e.value


def test_workspace(lib):
    f = muon.ags_muon_orthogonalize_workspace
    assert f(0, 5, 5) == 0 and f(3, 0, 5) == 0 and f(3, 5, 0) == 0
    for rows, cols in ((1, 1), (5, 70), (70, 5), (1000, 512)):
        s, pitch = min(rows, cols), -(-cols // 64) * 64
        assert f(1, rows, cols) >= rows * pitch * 8 + s * s * 4
        assert f(7, rows, cols) == 7 * f(1, rows, cols)
    _raises(ags.AGS_E_ARG, f, -1, 5, 5)
    _raises(ags.AGS_E_ARG, f, 1, -5, 5)
    _raises(ags.AGS_E_LAYOUT, f, 1, (1 << 20) + 1, 1)
    _raises(ags.AGS_E_LAYOUT, f, 1, 1 << 16, (1 << 15) + 1)
    _raises(ags.AGS_E_LAYOUT, f, 1, 1 << 20, 2049)
    _raises(ags.AGS_E_LAYOUT, f, (1 << 20) + 1, 1, 1)
    assert lib.ags_muon_orthogonalize_workspace(1, 4, 4, ctypes.POINTER(ctypes.c_size_t)()) == ags.AGS_E_ARG


def test_orthogonalize_refuses(lib):
    ws = muon.ags_muon_orthogonalize_workspace(2, 8, 40)
    good = [X, B, 2, 8, 40, 320, 40, muon.make_schedule(), Y, F, 320, 40, Z, ws]

    def bad(status, **change):
        args = list(good)
        for i, v in change.items():
            args[int(i[1:])] = v
        _raises(status, muon.ags_muon_orthogonalize, *args)

    bad(ags.AGS_E_ARG, a1=2)
    bad(ags.AGS_E_ARG, a9=2)
    bad(ags.AGS_E_ARG, a0=None)
    bad(ags.AGS_E_ARG, a8=None)
    bad(ags.AGS_E_ARG, a6=39)
    bad(ags.AGS_E_ARG, a11=39)
    bad(ags.AGS_E_ARG, a5=319)                                   # matrices that overlap
    bad(ags.AGS_E_ARG, a10=319)
    bad(ags.AGS_E_ARG, a6=1 << 50)
    bad(ags.AGS_E_ARG, a10=1 << 50)
    bad(ags.AGS_E_ALIGN, a0=X + 1)
    bad(ags.AGS_E_ALIGN, a8=Y + 2)
    bad(ags.AGS_E_ALIGN, a12=Z + 8)
    bad(ags.AGS_E_ARG, a12=None)
    bad(ags.AGS_E_ARG, a13=ws - 1)
    bad(ags.AGS_E_ARG, a8=X + 64)                                # out over x
    bad(ags.AGS_E_ARG, a12=Y)                                    # workspace over out
    bad(ags.AGS_E_ARG, a3=-1)
    # 2^20 matrices of 20 tiles each: more threads than a launch holds
    ws = muon.ags_muon_orthogonalize_workspace(1 << 20, 64, 1280)
    far = 1 << 46
    _raises(ags.AGS_E_LAYOUT, muon.ags_muon_orthogonalize, far, B, 1 << 20, 64, 1280, 81920, 1280,
            muon.make_schedule(), 2 * far, B, 81920, 1280, 4 * far, ws)
    muon.ags_muon_orthogonalize(None, F, 0, 8, 40, 320, 40, muon.make_schedule(), None, F, 320, 40)   # nothing to do


@pytest.mark.parametrize("kw", [
    {"steps": 0}, {"steps": 33}, {"eps": -1.0}, {"eps": float("nan")}, {"coefficients": (float("inf"), 0.0, 0.0)},
    {"coefficients": (4.0, 0.0, 0.0)},                           # 4^2 is too large for the second step
    {"coefficients": (1.0, 5.0, 0.0), "steps": 1},               # b A alone too large
    {"coefficients": (1.0, -3.0, -3.0), "steps": 1}])
def test_schedules_that_are_refused(lib, kw):
    ws = muon.ags_muon_orthogonalize_workspace(1, 8, 40)
    _raises(ags.AGS_E_ARG, muon.ags_muon_orthogonalize, X, B, 1, 8, 40, 320, 40, muon.make_schedule(**kw), Y, F, 320,
            40, Z, ws)


def test_schedules_that_pass(lib):
    """They get as far as the device checks, which need a GPU."""
    for kw in ({}, {"coefficients": (1.5, -0.5, 0.0), "steps": 32}, {"coefficients": (2.0, -1.5, 0.5)},
               {"coefficients": (4.0, 0.0, 0.0), "steps": 1}, {"coefficients": [(3.4445, -4.775, 2.0315)] * 4 + [(1.5, -0.5, 0.0)]}):
        muon.ags_muon_orthogonalize(None, F, 1, 0, 40, 0, 40, muon.make_schedule(**kw), None, F, 0, 40)
    with pytest.raises(ValueError):
        muon.make_schedule(coefficients=[(1.0, 0.0, 0.0)] * 4)


def _cfg(matrices=((0, 4, 8, 1.0), (64, 8, 4, 1.0)), n_flat=96, K=2, **kw):
    return muon.make_config(matrices, n_flat, K, **kw)


def test_config_refuses(lib):
    f = muon.ags_muon_workspace_bytes
    assert f(_cfg()) > 0 and f(_cfg(())) > 0
    for status, change in (
            (ags.AGS_E_ARG, {"K": 0}), (ags.AGS_E_LAYOUT, {"n_flat": 95}), (ags.AGS_E_LAYOUT, {"n_flat": -1}),
            (ags.AGS_E_ALIGN, {"matrices": [(4, 4, 4, 1.0)]}), (ags.AGS_E_LAYOUT, {"matrices": [(-8, 4, 4, 1.0)]}),
            (ags.AGS_E_LAYOUT, {"matrices": [(0, 4, 8, 1.0), (24, 2, 4, 1.0)]}),
            (ags.AGS_E_ARG, {"matrices": [(0, 0, 8, 1.0)]}), (ags.AGS_E_ARG, {"matrices": [(0, 4, 8, -1.0)]}),
            (ags.AGS_E_ARG, {"matrices": [(0, 4, 8, float("nan"))]}), (ags.AGS_E_ARG, {"lr": -0.1}),
            (ags.AGS_E_ARG, {"lr": float("inf")}), (ags.AGS_E_ARG, {"momentum": 1.0}),
            (ags.AGS_E_ARG, {"momentum": float("nan")}), (ags.AGS_E_ARG, {"weight_decay": -1.0}),
            (ags.AGS_E_ARG, {"steps": 0}), (ags.AGS_E_ARG, {"coefficients": (9.0, 0.0, 0.0)})):
        _raises(status, f, _cfg(**change))
    cfg = _cfg()
    for field, value in (("grad_dtype", 2), ("nesterov", 2), ("n_matrices", -1)):
        old = getattr(cfg, field)
        setattr(cfg, field, value)
        _raises(ags.AGS_E_ARG, f, cfg)
        setattr(cfg, field, old)
    assert lib.ags_muon_workspace_bytes(None, ctypes.byref(ctypes.c_size_t())) == ags.AGS_E_ARG
    _raises(ags.AGS_E_ARG, muon.ags_muon_init, cfg, None, Y)
    _raises(ags.AGS_E_ALIGN, muon.ags_muon_init, cfg, X + 4, Y)
    _raises(ags.AGS_E_ARG, muon.ags_muon_init, cfg, X, X + 64)   # m over w
    assert lib.ags_muon_step(None, X, 96, None) == ags.AGS_E_ARG and lib.ags_muon_set_lr(None, 0.1) == ags.AGS_E_ARG
    lib.ags_muon_destroy(None)


def test_binding_refuses_without_a_gpu():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA"):
        muon.orthogonalize(x)
    with pytest.raises(ValueError, match="gradient"):
        muon.orthogonalize(x.requires_grad_())
    with pytest.raises(ValueError, match="CUDA"):
        muon.Muon([(0, 2, 8)], torch.zeros(16), torch.zeros(16), 1)


@pytest.mark.parametrize("rows,cols", [(6, 20), (20, 6), (12, 12), (1, 7)])
def test_reference_against_singular_values(rows, cols):
    u = torch.randn(rows, cols, dtype=torch.float64, generator=torch.Generator().manual_seed(rows))
    left, s, right = torch.linalg.svd(u, full_matrices=False)
    s = s / (u.norm() + 1e-7)
    for _ in range(5):
        s = s * (3.4445 - 4.775 * s ** 2 + 2.0315 * s ** 4)
    want = left @ torch.diag(s) @ right
    got = ref.orthogonalize(u)
    assert torch.allclose(got, want, atol=1e-10)
    assert float((ref.orthogonalize(u, rounded=True) - got).norm()) < 0.01 * float(got.norm())
    assert (ref.orthogonalize(torch.zeros(rows, cols), eps=0.0, rounded=True) == 0).all()
