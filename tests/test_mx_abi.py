"""libags 4-bit operators on the host: the binding's names, sizes and argument
checks (no GPU; only calls that fail before any HIP call), and the reference
the GPU tests use."""
import ctypes
import os
import re

import numpy as np
import pytest

import mx_reference as ref
from paper_2603_18112_amd import _build, ags, mx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, Y, Z, V, W = (0x1000000000 * (i + 1) for i in range(5))       # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB):
        _build.build()
    return mx._lib()


def test_header_declares_the_binding_names():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ags_mx.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ags_[a-z_]+)\s*\(", text))) == sorted(mx.EXPORTS)
    assert ctypes.sizeof(mx.ags_mx_tensor) == 32


@pytest.mark.parametrize("rows,cols,codes,scales", [
    (0, 0, 0, 0), (3, 0, 0, 0), (0, 5, 0, 0), (1, 1, 128, 128), (1, 256, 128, 128), (17, 257, 17 * 256, 32 * 16),
    (4096, 25088, 4096 * 12544, 4096 * 784)])
def test_bytes(lib, rows, cols, codes, scales):
    assert mx.ags_mx_bytes(rows, cols) == (codes, scales)


@pytest.mark.parametrize("rows,cols,status", [
    (-1, 5, ags.AGS_E_ARG), (5, -1, ags.AGS_E_ARG), (1, (1 << 24) + 1, ags.AGS_E_LAYOUT),
    ((1 << 26) + 1, 256, ags.AGS_E_LAYOUT), (1 << 62, 0, ags.AGS_E_LAYOUT), (1 << 62, 1, ags.AGS_E_LAYOUT)])
def test_size_limits(lib, rows, cols, status):
    with pytest.raises(ags.AGSError) as e:
        mx.ags_mx_bytes(rows, cols)
    assert e.value.status == status and ags.ags_last_error(None)


def _raises(status, f, *args, **kw):
    with pytest.raises(ags.AGSError) as e:
        f(*args, **kw)
    assert e.value.status == status, e.value


def _t(rows, cols, codes=Y, scales=Z):
    return mx.ags_mx_tensor(codes, scales, rows, cols)


def test_quantize_refuses(lib):
    q, bf = mx.ags_mx_quantize, ags.AGS_BF16
    _raises(ags.AGS_E_ARG, q, X, 2, 4, 64, 64, None, 0, _t(4, 64), None)           # type
    _raises(ags.AGS_E_ARG, q, X, bf, 4, 64, 64, None, 0, None, None)               # no output
    _raises(ags.AGS_E_ARG, q, None, bf, 4, 64, 64, None, 0, _t(4, 64), None)
    _raises(ags.AGS_E_ALIGN, q, X + 1, bf, 4, 64, 64, None, 0, _t(4, 64), None)
    _raises(ags.AGS_E_ARG, q, X, bf, 4, 64, 63, None, 0, _t(4, 64), None)          # stride
    _raises(ags.AGS_E_ARG, q, X, bf, 4, 64, 64, V, 63, _t(4, 64), None)            # noise stride
    _raises(ags.AGS_E_ARG, q, X, bf, 4, 64, 64, None, 0, _t(4, 65), None)          # sizes differ
    _raises(ags.AGS_E_ARG, q, X, bf, 4, 64, 64, None, 0, None, _t(4, 64))
    _raises(ags.AGS_E_ALIGN, q, X, bf, 4, 64, 64, None, 0, _t(4, 64, Y + 8), None)
    _raises(ags.AGS_E_ARG, q, X, bf, 4, 64, 64, None, 0, _t(4, 64, None), None)
    _raises(ags.AGS_E_ARG, q, X, bf, 4, 64, 64, None, 0, _t(4, 64, X + 64), None)  # out over x
    _raises(ags.AGS_E_ARG, q, X, bf, 4, 64, 64, None, 0, _t(4, 64, Y, Y), None)    # scales over codes
    _raises(ags.AGS_E_ARG, q, X, bf, -1, 64, 64, None, 0, _t(-1, 64), None)
    _raises(ags.AGS_E_LAYOUT, q, X, bf, 4, 1 << 25, 1 << 25, None, 0, _t(4, 1 << 25), None)
    # the rows of a transposed form are padded too
    _raises(ags.AGS_E_LAYOUT, q, X, bf, (1 << 24) + 1, 4, 4, None, 0, None, _t(4, (1 << 24) + 1))
    q(X, bf, 0, 64, 64, None, 0, _t(0, 64), None)                                   # nothing to do


def test_dequantize_refuses(lib):
    d = mx.ags_mx_dequantize
    _raises(ags.AGS_E_ARG, d, _t(4, 64), None, ags.AGS_F32, 64)
    _raises(ags.AGS_E_ARG, d, _t(4, 64), X, 7, 64)
    _raises(ags.AGS_E_ARG, d, _t(4, 64), X, ags.AGS_F32, 63)
    _raises(ags.AGS_E_ALIGN, d, _t(4, 64), X + 2, ags.AGS_F32, 64)
    _raises(ags.AGS_E_ARG, d, _t(4, 64), Y, ags.AGS_F32, 64)
    assert lib.ags_mx_dequantize(None, X, 0, 64, None) == ags.AGS_E_ARG


def test_product_and_linear_refuse(lib):
    p, bf = mx.ags_mx_product, ags.AGS_BF16
    a, b = _t(4, 64, Y, Z), _t(8, 64, V, W)
    _raises(ags.AGS_E_ARG, p, a, _t(8, 65, V, W), X, bf, 8)
    _raises(ags.AGS_E_ARG, p, a, b, X, 3, 8)
    _raises(ags.AGS_E_ARG, p, a, b, X, bf, 7)
    _raises(ags.AGS_E_ARG, p, a, b, None, bf, 8)
    _raises(ags.AGS_E_ARG, p, a, b, X, bf, 8, accumulate=2)
    _raises(ags.AGS_E_ARG, p, a, b, Y, bf, 8)                                       # out over a
    _raises(ags.AGS_E_ALIGN, p, a, b, X + 1, bf, 8)
    _raises(ags.AGS_E_LAYOUT, p, _t(1 << 20, 64, Y, Z), _t(1 << 20, 64, V, W), X, bf, 1 << 20)
    lin = mx.ags_mx_linear
    assert mx.ags_mx_linear_workspace(4, 8, 64) == 0                               # few rows: one kernel
    need = mx.ags_mx_linear_workspace(40, 8, 64)
    assert need > 0
    _raises(ags.AGS_E_ARG, lin, X, bf, 40, 64, b, Y, bf, 8, None, 0)                # no workspace
    _raises(ags.AGS_E_ARG, lin, X, bf, 40, 64, b, Y, bf, 8, Z, need - 1)
    _raises(ags.AGS_E_ALIGN, lin, X, bf, 40, 64, b, Y, bf, 8, Z + 8, need)
    _raises(ags.AGS_E_ARG, lin, X, bf, 4, 63, b, Y, bf, 8, Z, need)
    _raises(ags.AGS_E_ARG, lin, X, bf, 4, 64, b, X, bf, 8, Z, need)
    _raises(ags.AGS_E_ARG, lin, X, bf, 4, 64, b, Y, 5, 8, Z, need)
    _raises(ags.AGS_E_ARG, mx.ags_mx_product_workspace, -1, 2, 3)
    _raises(ags.AGS_E_LAYOUT, mx.ags_mx_linear_workspace, 1 << 20, 1 << 20, 64)
    lin(X, bf, 0, 64, b, Y, bf, 8)                                                  # nothing to do


def test_reference_nearest_by_hand():
    x = np.zeros((1, 64))
    x[0, :8] = [4.0, 0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5.0]       # every tie, scale 1
    x[0, 32:38] = [7.99, -6.5, 0.2501, 0.2499, 5.0001, 0.7499]
    v, e = ref.store_rows(x)
    assert e.tolist() == [[0, 0]]
    assert v[0, :8].tolist() == [4.0, 0.0, -1.0, 1.0, 2.0, -2.0, 4.0, 4.0]
    assert v[0, 32:38].tolist() == [6.0, -6.0, 0.5, 0.0, 6.0, 0.5]


def test_reference_stochastic_by_hand():
    x = np.zeros((1, 32))
    x[0, :5] = [6.5, 3.5, 1.0, 0.125, 0.25]                          # scale 2: 3.25 1.75 0.5 0.0625 0.125
    r = np.zeros((1, 32))
    r[0, :5] = [191, 128, 0, 223, 191]
    v, e = ref.store_rows(x, r)
    assert e[0, 0] == 1
    # fractions .25, .5, 0, .125, .25 with (r + 1/2) / 256 = .748, .502, .002, .873, .748
    assert v[0, :5].tolist() == [6.0, 4.0, 1.0, 0.0, 0.0]
    r[0, :5] = [192, 127, 255, 224, 192]
    v, _ = ref.store_rows(x, r)
    assert v[0, :5].tolist() == [8.0, 3.0, 1.0, 1.0, 1.0]


def test_reference_stochastic_is_unbiased():
    """The mean over all 256 bytes is within half a byte's step."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((1, 32))
    mean = np.zeros((1, 32))
    for r in range(256):
        v, e = ref.store_rows(x, np.full((1, 32), r))
        mean += v / 256
    step = np.where(np.abs(x) < 2 * 2.0 ** e[0, 0], 0.5, np.where(np.abs(x) < 4 * 2.0 ** e[0, 0], 1.0, 2.0))
    assert np.all(np.abs(mean - x) <= step * 2.0 ** e[0, 0] / 512 + 1e-12)


@pytest.mark.parametrize("rows,stride", [((1 << 26), 1 << 40), (1 << 24, (1 << 62) // (1 << 24)), (3, 1 << 62)])
def test_strides_past_any_address_space(rows, stride):
    # (rows - 1) * stride elements of 4 bytes pass 2^64, or come near it: the
    # size of the buffer must not wrap to a small one.
    for row_stride, noise in ((stride, None), (64, V)):
        with pytest.raises(ags.AGSError) as e:
            mx.ags_mx_quantize(X, ags.AGS_F32, rows, 64, row_stride, noise, stride, _t(rows, 64), None)
        assert e.value.status == ags.AGS_E_ARG and "stride" in str(e.value)


def test_training_calls_refuse(lib):
    bf, U = ags.AGS_BF16, 0x9000000000
    save, back = mx.ags_mx_linear_save, mx.ags_mx_linear_backward
    w, saved = _t(8, 64, V, W), _t(64, 40, U, U + (1 << 24))
    need = mx.ags_mx_linear_save_workspace(40, 8, 64)
    assert need >= sum(mx.ags_mx_bytes(40, 64))
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 64, w, Y, bf, 8, saved, None, 0)                  # no workspace
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 64, w, Y, bf, 8, saved, Z, need - 1)
    _raises(ags.AGS_E_ALIGN, save, X, bf, 40, 64, w, Y, bf, 8, saved, Z + 8, need)
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 64, w, Y, bf, 8, _t(40, 64, U, U + (1 << 24)), Z, need)
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 64, w, Y, bf, 8, _t(64, 40, X, U), Z, need)       # saved over x
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 64, w, Y, bf, 8, _t(64, 40, None, U), Z, need)
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 63, w, Y, bf, 8, saved, Z, need)                  # strides
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 64, w, Y, bf, 7, saved, Z, need)
    _raises(ags.AGS_E_ARG, save, X, 2, 40, 64, w, Y, bf, 8, saved, Z, need)
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 64, w, Y, 2, 8, saved, Z, need)
    _raises(ags.AGS_E_ALIGN, save, X + 1, bf, 40, 64, w, Y, bf, 8, saved, Z, need)
    _raises(ags.AGS_E_ARG, save, X, bf, 40, 64, w, Z, bf, 8, saved, Z, need)                  # y over the workspace
    save(X, bf, 0, 64, w, Y, bf, 8, _t(64, 0))                                                 # nothing to do
    wt = _t(64, 8, V, W)
    need = mx.ags_mx_linear_backward_workspace(40, 8, 64, 1)
    assert need > mx.ags_mx_linear_backward_workspace(40, 8, 64, 0) > 0
    good = dict(d_dy=X, dtype=bf, rows=40, n=8, row_stride=8, d_noise=None, noise_stride=0, saved=saved, wt=wt,
                d_dx=Y, dx_stride=64, d_dw=Z, dw_dtype=ags.AGS_F32, dw_stride=64, accumulate=0,
                d_workspace=0x20000000000, workspace_bytes=need)
    for status, change in (
            (ags.AGS_E_ARG, dict(d_workspace=None)), (ags.AGS_E_ARG, dict(workspace_bytes=need - 1)),
            (ags.AGS_E_ALIGN, dict(d_workspace=0x20000000004)), (ags.AGS_E_ARG, dict(dtype=2)),
            (ags.AGS_E_ARG, dict(dw_dtype=2)), (ags.AGS_E_ARG, dict(accumulate=2)), (ags.AGS_E_ARG, dict(d_dy=None)),
            (ags.AGS_E_ARG, dict(row_stride=7)), (ags.AGS_E_ARG, dict(d_noise=X + (1 << 24), noise_stride=7)),
            (ags.AGS_E_ARG, dict(rows=41)), (ags.AGS_E_ARG, dict(wt=_t(8, 64, V, W))), (ags.AGS_E_ARG, dict(d_dx=None)),
            (ags.AGS_E_ARG, dict(dx_stride=63)), (ags.AGS_E_ARG, dict(d_dw=None)), (ags.AGS_E_ARG, dict(dw_stride=63)),
            (ags.AGS_E_ALIGN, dict(d_dw=Z + 2)), (ags.AGS_E_ARG, dict(d_dw=Y)), (ags.AGS_E_ARG, dict(d_dx=X)),
            (ags.AGS_E_ARG, dict(rows=-1)), (ags.AGS_E_LAYOUT, dict(n=1 << 25, row_stride=1 << 25)),
            (ags.AGS_E_ARG, dict(d_dw=U))):
        _raises(status, back, **{**good, **change})
    assert lib.ags_mx_linear_save_workspace(40, 8, 64, None) == ags.AGS_E_ARG
    assert lib.ags_mx_linear_backward_workspace(40, 8, 64, 1, None) == ags.AGS_E_ARG
    _raises(ags.AGS_E_LAYOUT, mx.ags_mx_linear_save_workspace, 1 << 20, 1 << 20, 64)
    _raises(ags.AGS_E_ARG, mx.ags_mx_linear_backward_workspace, 4, -1, 64, 0)


@pytest.mark.parametrize("m,n", [(1 << 34, 1), (1, 1 << 34), (1 << 31, 2), ((1 << 26) + 1, 1)])
def test_products_over_an_empty_axis_stay_within_a_launch(lib, m, n):
    # operands without columns have no elements to limit their rows: the
    # product of 2^34 by 1 would need 2^36 work-items
    for query in (mx.ags_mx_product_workspace, mx.ags_mx_linear_workspace, mx.ags_mx_linear_save_workspace):
        _raises(ags.AGS_E_LAYOUT, query, m, n, 0)
    _raises(ags.AGS_E_LAYOUT, mx.ags_mx_linear_backward_workspace, 0, m, n, 1)
    _raises(ags.AGS_E_LAYOUT, mx.ags_mx_product, _t(m, 0, None, None), _t(n, 0, None, None), X, ags.AGS_BF16, n)
    assert mx.ags_mx_product_workspace(1 << 26, 256, 0) == 0
    assert mx.ags_mx_product_workspace(m, 0, 0) == 0                                # nothing to do
