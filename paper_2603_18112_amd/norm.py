"""Python binding of the libags layer norm (include/ags_norm.h): argument
marshalling only; both passes run in the HIP kernels of the library.
"""
from __future__ import annotations

import ctypes

from . import ags
from .mx import _check, _dtype, _matrix, _stream, _t, _workspace

EXPORTS = ("ags_layer_norm", "ags_layer_norm_backward_workspace", "ags_layer_norm_backward")

_sig_done = False


def _lib():
    global _sig_done
    lib = ags.load_library()
    if not _sig_done:
        vp, c_int, i32, i64, sz, dbl = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int32, ctypes.c_int64,
                                        ctypes.c_size_t, ctypes.c_double)
        sig = {
            "ags_layer_norm": [vp, c_int, i64, i64, i64, vp, vp, c_int, dbl, vp, c_int, i64, vp, vp],
            "ags_layer_norm_backward_workspace": [i64, i64, ctypes.POINTER(sz)],
            "ags_layer_norm_backward": [vp, i64, vp, c_int, i64, i64, i64, vp, vp, c_int, vp, i64, vp, vp, c_int,
                                        i32, vp, sz, vp],
        }
        for name, args in sig.items():
            f = getattr(lib, name)
            f.restype = c_int
            f.argtypes = args
        _sig_done = True
    return lib


# ------------------------------------------------------------ thin calls --
# Same names and arguments as the C functions; pointers are ints.


def ags_layer_norm(d_x, dtype, rows, cols, x_stride, d_weight, d_bias, w_dtype, eps, d_y, y_dtype, y_stride,
                   d_saved=None, stream=0):
    _check(_lib().ags_layer_norm(d_x, dtype, rows, cols, x_stride, d_weight, d_bias, w_dtype, eps, d_y, y_dtype,
                                 y_stride, d_saved, stream))


def ags_layer_norm_backward_workspace(rows: int, cols: int) -> int:
    b = ctypes.c_size_t(0)
    _check(_lib().ags_layer_norm_backward_workspace(rows, cols, ctypes.byref(b)))
    return b.value


def ags_layer_norm_backward(d_dy, dy_stride, d_x, dtype, rows, cols, x_stride, d_saved, d_weight, w_dtype, d_dx,
                            dx_stride, d_dweight, d_dbias, dw_dtype, accumulate=0, d_workspace=None,
                            workspace_bytes=0, stream=0):
    _check(_lib().ags_layer_norm_backward(d_dy, dy_stride, d_x, dtype, rows, cols, x_stride, d_saved, d_weight,
                                          w_dtype, d_dx, dx_stride, d_dweight, d_dbias, dw_dtype, accumulate,
                                          d_workspace, workspace_bytes, stream))


# ------------------------------------------------------- torch convenience --
# Device memory and streams come from torch; work goes on the current stream
# (choose another with torch.cuda.stream).


def _recorded(*tensors):
    t = _t()
    if t.is_grad_enabled():
        for x in tensors:
            if x is not None and x.requires_grad:
                raise ValueError("an input requires a gradient, which this call does not record: detach it, or call "
                                 "under torch.no_grad() and the backward function for the gradients")


def _vector(v, cols, what, device):
    """(contiguous [cols] or None, its type's code, address)."""
    if v is None:
        return None, ags.AGS_F32, None
    if v.dim() != 1 or v.shape[0] != cols or v.device != device:
        raise ValueError(f"{what} must be [{cols}], on x's device")
    code = _dtype(v.dtype)[0]
    if not v.is_contiguous():
        v = v.contiguous()
    return v, code, v.data_ptr() or None


def _grad_vector(out, wanted, cols, dtype, accumulate, what, device):
    """(gradient [cols] to write, or None; its type's code)."""
    if out is None:
        if not wanted:
            return None, None
        if accumulate:
            raise ValueError(f"accumulate needs {what}")
        code, dt = _dtype(dtype)
        return _t().empty(cols, dtype=dt, device=device), code
    if not wanted:
        raise ValueError(f"{what} is given but not wanted")
    if tuple(out.shape) != (cols,) or out.device != device or (cols > 1 and out.stride(0) != 1):
        raise ValueError(f"{what} must be a contiguous [{cols}], on x's device")
    return out, _dtype(out.dtype)[0]


def layer_norm(x, weight=None, bias=None, eps=1e-5, dtype=None, save=False):
    """y = z weight + bias, z the rows of x [..., cols] at mean 0 and variance 1:
    [..., cols] of `dtype` (x's unless given).  weight, bias: [cols], of one
    type, or None.  save=True returns (y, saved): fp32 [2, rows], the means
    and the reciprocal standard deviations, for the backward pass.  An x whose
    rows are not contiguous is copied first.  Autograd does not see the call,
    so inputs that require a gradient are refused where gradients are
    recorded."""
    t = _t()
    _recorded(x, weight, bias)
    x2, rows, cols, stride = _matrix(x, "x", copy=True)
    code, dev = _dtype(x.dtype)[0], x.device
    out_code, out_dt = _dtype(x.dtype if dtype is None else dtype)
    weight, w_code, w_ptr = _vector(weight, cols, "weight", dev)
    bias, b_code, b_ptr = _vector(bias, cols, "bias", dev)
    if weight is not None and bias is not None and w_code != b_code:
        raise ValueError("weight and bias differ in type")
    y = x.new_empty(x.shape, dtype=out_dt)
    saved = x.new_empty((2, rows), dtype=t.float32) if save else None
    ags_layer_norm(x2.data_ptr() or None, code, rows, cols, max(stride, 1), w_ptr, b_ptr,
                   w_code if weight is not None else b_code, eps, y.data_ptr() or None, out_code, max(cols, 1),
                   (saved.data_ptr() or None) if save else None, _stream(dev))
    return (y, saved) if save else y


def layer_norm_backward(dy, x, saved, weight=None, dweight=None, dbias=None, dw_dtype="f32", accumulate=False,
                        need_dx=True, need_dw=True, need_db=True):
    """The gradients of layer_norm given dy [..., cols] of x's type: (dx [...,
    cols] of x's type, dweight [cols], dbias [cols]), None in place of those
    not wanted.  saved: what layer_norm(save=True) returned.  dweight, dbias:
    written there (views of a replica's row, say), added with `accumulate`;
    else new tensors of `dw_dtype`."""
    t = _t()
    if dy.shape != x.shape or dy.dtype != x.dtype or dy.device != x.device:
        raise ValueError("dy and x differ in shape, type or device")
    x2, rows, cols, x_stride = _matrix(x, "x", copy=True)
    dy2, _, _, dy_stride = _matrix(dy, "dy", copy=True)
    code, dev = _dtype(x.dtype)[0], x.device
    if tuple(saved.shape) != (2, rows) or saved.dtype is not t.float32 or saved.device != dev or \
            not saved.is_contiguous():
        raise ValueError(f"saved must be a contiguous float32 [2, {rows}], on x's device")
    weight, w_code, w_ptr = _vector(weight, cols, "weight", dev)
    dweight, dw_code = _grad_vector(dweight, need_dw, cols, dw_dtype, accumulate, "dweight", dev)
    dbias, db_code = _grad_vector(dbias, need_db, cols, dw_dtype, accumulate, "dbias", dev)
    if None not in (dw_code, db_code) and dw_code != db_code:
        raise ValueError("dweight and dbias differ in type")
    dx = x.new_empty(x.shape) if need_dx else None
    if not (need_dx or need_dw or need_db):
        return None, None, None
    nbytes = ags_layer_norm_backward_workspace(rows, cols) if need_dw or need_db else 0
    ws = _workspace(nbytes, dev)
    if cols and (rows or need_dw or need_db):
        ags_layer_norm_backward(dy2.data_ptr() or None, max(dy_stride, 1), x2.data_ptr() or None, code, rows, cols,
                                max(x_stride, 1), saved.data_ptr() or None, w_ptr, w_code,
                                (dx.data_ptr() or None) if need_dx else None, max(cols, 1),
                                None if dweight is None else dweight.data_ptr(),
                                None if dbias is None else dbias.data_ptr(),
                                ags.AGS_F32 if dw_code is None and db_code is None else dw_code if db_code is None
                                else db_code, int(accumulate), None if ws is None else ws.data_ptr(), nbytes,
                                _stream(dev))
    return dx, dweight, dbias
