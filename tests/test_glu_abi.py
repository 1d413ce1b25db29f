"""libags gated products on the host: the binding's names, sizes and argument
checks (no GPU; only calls that fail before any HIP call)."""
import ctypes
import os
import re

import pytest
import torch

from paper_2603_18112_amd import _build, ags, glu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, Y, Z, V, W, S, P, Q = (0x1000000000 * (i + 1) for i in range(8))       # never dereferenced
F, B = ags.AGS_F32, ags.AGS_BF16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB):
        _build.build()
    return glu._lib()


def test_header_declares_the_binding_names():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ags_glu.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ags_[a-z_]+)\s*\(", text))) == sorted(glu.EXPORTS)
    assert ctypes.sizeof(glu.ags_glu_weight) == 24


def _raises(status, f, *args, **kw):
    with pytest.raises(ags.AGSError) as e:
        f(*args, **kw)
    assert e.value.status == status and ags.ags_last_error(None), e.value


@pytest.mark.parametrize("n,k,size", [(0, 0, 0), (0, 5, 0), (5, 0, 0), (1, 1, 32 * 64 * 2), (16, 64, 32 * 64 * 2),
                                      (17, 65, 64 * 128 * 2), (4096, 1000, 8192 * 1024 * 2)])
def test_bytes(lib, n, k, size):
    assert glu.ags_glu_bytes(n, k) == size


def test_sizes_and_workspaces(lib):
    for f in (glu.ags_glu_bytes, lambda n, k: glu.ags_glu_forward_workspace(1, n, k),
              lambda n, k: glu.ags_glu_backward_workspace(1, n, k)):
        _raises(ags.AGS_E_ARG, f, -1, 4)
        _raises(ags.AGS_E_LAYOUT, f, 4, (1 << 20) + 1)
        _raises(ags.AGS_E_LAYOUT, f, (1 << 20) + 1, 4)
    for f in (glu.ags_glu_forward_workspace, glu.ags_glu_backward_workspace):
        _raises(ags.AGS_E_ARG, f, -1, 4, 4)
        _raises(ags.AGS_E_LAYOUT, f, (1 << 30) + 1, 4, 4)
        _raises(ags.AGS_E_LAYOUT, f, 1 << 30, 1 << 20, 4)
        for rows, n, k in ((0, 5, 5), (1, 1, 1), (33, 17, 65), (1 << 20, 100, 100), (100, 0, 7), (100, 7, 0)):
            assert f(rows, n, k) >= rows * (-(-k // 64) * 64) * 2
    assert lib.ags_glu_bytes(4, 4, ctypes.POINTER(ctypes.c_size_t)()) == ags.AGS_E_ARG


def _w(n=16, k=64, data=W):
    return glu.ags_glu_weight(data, n, k)


def _changer(f, good):
    def bad(status, **change):
        args = list(good)
        for i, v in change.items():
            args[int(i[1:])] = v
        _raises(status, f, *args)
    return bad


def test_store_refuses(lib):
    bad = _changer(glu.ags_glu_store, [X, 64, Y, 64, F, _w()])
    bad(ags.AGS_E_ARG, a4=2)
    bad(ags.AGS_E_ARG, a0=None)
    bad(ags.AGS_E_ARG, a2=None)
    bad(ags.AGS_E_ARG, a1=63)
    bad(ags.AGS_E_ARG, a3=63)
    bad(ags.AGS_E_ALIGN, a0=X + 2)
    bad(ags.AGS_E_ALIGN, a5=_w(data=W + 8))
    bad(ags.AGS_E_ARG, a5=_w(data=None))
    bad(ags.AGS_E_ARG, a5=_w(data=X + 64))                       # over gate
    bad(ags.AGS_E_ARG, a5=_w(n=-1))
    bad(ags.AGS_E_LAYOUT, a5=_w(k=1 << 21), a1=1 << 21, a3=1 << 21)
    glu.ags_glu_store(None, 1, None, 1, F, _w(0, 4, None))       # nothing to do


def test_forward_refuses(lib):
    ws = glu.ags_glu_forward_workspace(40, 16, 64)
    bad = _changer(glu.ags_glu_forward, [X, 40, 64, _w(), 0, Y, B, 16, S, Q, ws])
    bad(ags.AGS_E_ARG, a4=2)                                     # activation
    bad(ags.AGS_E_ARG, a6=5)
    bad(ags.AGS_E_ARG, a1=-1)
    bad(ags.AGS_E_LAYOUT, a1=(1 << 30) + 1)
    bad(ags.AGS_E_ARG, a0=None)
    bad(ags.AGS_E_ARG, a5=None)
    bad(ags.AGS_E_ARG, a2=63)
    bad(ags.AGS_E_ARG, a7=15)
    bad(ags.AGS_E_ALIGN, a0=X + 1)
    bad(ags.AGS_E_ALIGN, a8=S + 8)
    bad(ags.AGS_E_ARG, a9=None)
    bad(ags.AGS_E_ARG, a10=ws - 1)
    bad(ags.AGS_E_ALIGN, a9=Q + 4)
    bad(ags.AGS_E_ARG, a5=X + 16)                                # h over x
    bad(ags.AGS_E_ARG, a8=Y)                                     # saved over h
    bad(ags.AGS_E_ARG, a9=W)                                     # workspace over the weight
    bad(ags.AGS_E_ARG, a3=_w(n=-3))
    glu.ags_glu_forward(None, 0, 64, _w(), 0, None, B, 16)       # nothing to do
    glu.ags_glu_forward(X, 40, 64, _w(0, 64, None), 0, None, B, 1, None, Q, ws)


def test_backward_refuses(lib):
    ws = glu.ags_glu_backward_workspace(40, 16, 64)
    good = [X, 16, Y, 40, 64, S, _w(), 1, Z, 64, V, P, B, 64, 0, Q, ws]
    bad = _changer(glu.ags_glu_backward, good)
    bad(ags.AGS_E_ARG, a7=2)
    bad(ags.AGS_E_ARG, a12=2)
    bad(ags.AGS_E_ARG, a14=2)
    bad(ags.AGS_E_ARG, a8=None, a10=None, a11=None)              # nothing wanted
    bad(ags.AGS_E_ARG, a10=None)                                 # one of the two
    bad(ags.AGS_E_ARG, a11=None)
    bad(ags.AGS_E_ARG, a0=None)
    bad(ags.AGS_E_ARG, a2=None)
    bad(ags.AGS_E_ARG, a1=15)
    bad(ags.AGS_E_ARG, a9=63)
    bad(ags.AGS_E_ARG, a13=63)
    bad(ags.AGS_E_ALIGN, a5=S + 2)
    bad(ags.AGS_E_ALIGN, a15=Q + 8)
    bad(ags.AGS_E_ARG, a16=ws - 1)
    bad(ags.AGS_E_ARG, a8=X)                                     # dx over dh
    bad(ags.AGS_E_ARG, a11=V + 128)                              # dup over dgate
    bad(ags.AGS_E_ARG, a15=S)                                    # workspace over saved
    glu.ags_glu_backward(None, 16, None, 0, 64, None, _w(), 0, Z, 64, V, P, B, 64, 1)    # no rows, added


def test_binding_refuses_without_a_gpu():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA"):
        glu.Weight(x, x)
    with pytest.raises(ValueError, match="gradient"):
        glu.gated_linear(x.requires_grad_(), None)
