"""Python binding of the libags 4-bit operators (include/ags_mx.h): argument
marshalling only; storing, reading back and multiplying run in the HIP
kernels of the library.
"""
from __future__ import annotations

import ctypes
import math

from . import ags

AGS_MX_BLOCK, AGS_MX_PAD, AGS_MX_ROWS = 32, 256, 16
EXPORTS = ("ags_mx_bytes", "ags_mx_quantize", "ags_mx_dequantize", "ags_mx_product_workspace",
           "ags_mx_product", "ags_mx_linear_workspace", "ags_mx_linear", "ags_mx_linear_save_workspace",
           "ags_mx_linear_save", "ags_mx_linear_backward_workspace", "ags_mx_linear_backward")


class ags_mx_tensor(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64)]


_sig_done = False


def _lib():
    global _sig_done
    lib = ags.load_library()
    if not _sig_done:
        P, vp, c_int, i32, i64, sz = (ctypes.POINTER, ctypes.c_void_p, ctypes.c_int, ctypes.c_int32,
                                      ctypes.c_int64, ctypes.c_size_t)
        T = P(ags_mx_tensor)
        sig = {
            "ags_mx_bytes": [i64, i64, P(sz), P(sz)],
            "ags_mx_quantize": [vp, c_int, i64, i64, i64, vp, i64, T, T, vp],
            "ags_mx_dequantize": [T, vp, c_int, i64, vp],
            "ags_mx_product_workspace": [i64, i64, i64, P(sz)],
            "ags_mx_product": [T, T, vp, c_int, i64, i32, vp, sz, vp],
            "ags_mx_linear_workspace": [i64, i64, i64, P(sz)],
            "ags_mx_linear": [vp, c_int, i64, i64, T, vp, c_int, i64, vp, sz, vp],
            "ags_mx_linear_save_workspace": [i64, i64, i64, P(sz)],
            "ags_mx_linear_save": [vp, c_int, i64, i64, T, vp, c_int, i64, T, vp, sz, vp],
            "ags_mx_linear_backward_workspace": [i64, i64, i64, i32, P(sz)],
            "ags_mx_linear_backward": [vp, c_int, i64, i64, i64, vp, i64, T, T, vp, i64, vp, c_int, i64, i32,
                                       vp, sz, vp],
        }
        for name, args in sig.items():
            f = getattr(lib, name)
            f.restype = c_int
            f.argtypes = args
        _sig_done = True
    return lib


def _check(status):
    if status != ags.AGS_OK:
        raise ags.AGSError(status, ags.ags_last_error(None))


# ------------------------------------------------------------ thin calls --
# Same names and arguments as the C functions; pointers are ints.


def ags_mx_bytes(rows: int, cols: int):
    """(bytes of the codes, bytes of the scales)"""
    c, s = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(_lib().ags_mx_bytes(int(rows), int(cols), ctypes.byref(c), ctypes.byref(s)))
    return int(c.value), int(s.value)


def ags_mx_quantize(d_x, dtype, rows, cols, row_stride, d_noise, noise_stride, q, qt, stream=0):
    _check(_lib().ags_mx_quantize(d_x, dtype, rows, cols, row_stride, d_noise, noise_stride,
                                  None if q is None else ctypes.byref(q),
                                  None if qt is None else ctypes.byref(qt), stream))


def ags_mx_dequantize(q, d_out, dtype, row_stride, stream=0):
    _check(_lib().ags_mx_dequantize(ctypes.byref(q), d_out, dtype, row_stride, stream))


def ags_mx_product_workspace(m: int, n: int, k: int) -> int:
    b = ctypes.c_size_t(0)
    _check(_lib().ags_mx_product_workspace(m, n, k, ctypes.byref(b)))
    return b.value


def ags_mx_product(a, b, d_out, dtype, row_stride, accumulate=0, d_workspace=None, workspace_bytes=0,
                   stream=0):
    _check(_lib().ags_mx_product(ctypes.byref(a), ctypes.byref(b), d_out, dtype, row_stride, accumulate,
                                 d_workspace, workspace_bytes, stream))


def ags_mx_linear_workspace(rows: int, n: int, k: int) -> int:
    b = ctypes.c_size_t(0)
    _check(_lib().ags_mx_linear_workspace(rows, n, k, ctypes.byref(b)))
    return b.value


def ags_mx_linear(d_x, dtype, rows, row_stride, w, d_y, y_dtype, y_stride, d_workspace=None,
                  workspace_bytes=0, stream=0):
    _check(_lib().ags_mx_linear(d_x, dtype, rows, row_stride, ctypes.byref(w), d_y, y_dtype, y_stride,
                                d_workspace, workspace_bytes, stream))


def ags_mx_linear_save_workspace(rows: int, n: int, k: int) -> int:
    b = ctypes.c_size_t(0)
    _check(_lib().ags_mx_linear_save_workspace(rows, n, k, ctypes.byref(b)))
    return b.value


def ags_mx_linear_save(d_x, dtype, rows, row_stride, w, d_y, y_dtype, y_stride, saved, d_workspace=None,
                       workspace_bytes=0, stream=0):
    _check(_lib().ags_mx_linear_save(d_x, dtype, rows, row_stride, ctypes.byref(w), d_y, y_dtype, y_stride,
                                     ctypes.byref(saved), d_workspace, workspace_bytes, stream))


def ags_mx_linear_backward_workspace(rows: int, n: int, k: int, need_dx: int) -> int:
    b = ctypes.c_size_t(0)
    _check(_lib().ags_mx_linear_backward_workspace(rows, n, k, need_dx, ctypes.byref(b)))
    return b.value


def ags_mx_linear_backward(d_dy, dtype, rows, n, row_stride, d_noise, noise_stride, saved, wt, d_dx, dx_stride,
                           d_dw, dw_dtype, dw_stride, accumulate=0, d_workspace=None, workspace_bytes=0,
                           stream=0):
    _check(_lib().ags_mx_linear_backward(d_dy, dtype, rows, n, row_stride, d_noise, noise_stride,
                                         ctypes.byref(saved), None if wt is None else ctypes.byref(wt), d_dx,
                                         dx_stride, d_dw, dw_dtype, dw_stride, accumulate, d_workspace,
                                         workspace_bytes, stream))


# ------------------------------------------------------- torch convenience --
# Device memory and streams come from torch; work goes on the current stream
# (choose another with torch.cuda.stream).

_torch = None


def _t():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _dtype(dtype):
    """(AGS_F32 or AGS_BF16, torch dtype) of "f32", "bf16" or a torch dtype."""
    t = _t()
    if dtype is t.bfloat16 or dtype == "bf16":
        return ags.AGS_BF16, t.bfloat16
    if dtype is t.float32 or dtype == "f32":
        return ags.AGS_F32, t.float32
    raise ValueError(f"dtype {dtype!r} is neither float32 nor bfloat16")


def _stream(device):
    """The current stream of the tensors' device, as an int (the raw query
    takes 0.1 us, a Stream object 2)."""
    t = _t()
    raw = getattr(t._C, "_cuda_getCurrentRawStream", None)
    if raw is not None and device.index is not None:
        return raw(device.index)
    return t.cuda.current_stream(device).cuda_stream


def _matrix(x, what, copy=False):
    """x as 2-D with unit column stride: (tensor, rows, cols, row stride).
    copy: rows that overlap or are not contiguous are copied, not refused."""
    if not x.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if x.dim() != 2:
        if x.dim() == 0:
            raise ValueError(f"{what} needs at least one dimension")
        x = x.reshape(math.prod(x.shape[:-1]), x.shape[-1])
    rows, cols = x.shape
    if cols > 1 and x.stride(1) != 1:
        if not copy:
            raise ValueError(f"{what} must be contiguous along its last axis")
        x = x.contiguous()
    stride = x.stride(0) if rows > 1 else cols
    if stride < cols:
        if not copy:
            raise ValueError(f"{what}'s rows overlap")
        x, stride = x.contiguous(), cols
    return x, rows, cols, stride


def _up(x, unit):
    return -(-x // unit) * unit


class MX4:
    """A [rows, cols] tensor held in 4 bits, blocked along its columns: one
    buffer with the codes, then the scales (the sizes ags_mx_bytes gives)."""

    __slots__ = ("data", "rows", "cols", "c")

    def __init__(self, rows, cols, device=None):
        t = _t()
        padded = _up(cols, AGS_MX_PAD)
        codes, scales = rows * padded // 2, _up(rows, AGS_MX_ROWS) * padded // AGS_MX_BLOCK
        dev = t.device("cuda", t.cuda.current_device()) if device is None else device
        self.data = t.empty(codes + scales, dtype=t.uint8, device=dev)
        self.rows, self.cols = int(rows), int(cols)
        p = self.data.data_ptr() or None
        # a row of codes is a multiple of 128 bytes, so the scales are aligned too
        self.c = ags_mx_tensor(p, p and p + codes, self.rows, self.cols)

    @property
    def codes(self):
        return self.data[:self.rows * _up(self.cols, AGS_MX_PAD) // 2]

    @property
    def scales(self):
        return self.data[self.rows * _up(self.cols, AGS_MX_PAD) // 2:]

    @property
    def shape(self):
        return self.rows, self.cols


def _noise(noise, rows, cols, what, copy=False):
    """(random bytes [rows, cols] or None, their address, row stride)."""
    if noise is None:
        return None, None, 0
    noise, r, c, stride = _matrix(noise, "noise", copy)
    if noise.dtype is not _t().uint8 or (r, c) != (rows, cols):
        raise ValueError(f"noise must hold one uint8 for each element of {what}")
    return noise, noise.data_ptr() or None, stride


def _transposed(x):
    return x.dim() == 2 and x.stride(1) != 1 and x.stride(0) == 1 and x.shape[1] > 1


def _quantize(x, noise, q, qt):
    if _transposed(x):
        # the two forms change places
        qt, q = _quantize(x.t(), None if noise is None else noise.t().contiguous(), qt, q)
        return q, qt
    x, rows, cols, stride = _matrix(x, "x")
    dt = _dtype(x.dtype)[0]
    noise, n_ptr, n_stride = _noise(noise, rows, cols, "x")
    if q is True:
        q = MX4(rows, cols, x.device)
    if qt is True:
        qt = MX4(cols, rows, x.device)
    ags_mx_quantize(x.data_ptr(), dt, rows, cols, stride, n_ptr, n_stride, q and q.c, qt and qt.c,
                    _stream(x.device))
    return q, qt


def quantize(x, noise=None, out=None):
    """x [..., cols] in 4 bits, blocked along its columns: an MX4 of
    [rows, cols].  x is contiguous along its last axis, or a transposed matrix.
    noise: random bytes (uint8, x's shape) for stochastic rounding.  out: an MX4
    to write."""
    return _quantize(x, noise, True if out is None else out, None)[0]


def quantize_t(x, noise=None, out=None):
    """x transposed, blocked along the rows of x: an MX4 of [cols, rows]."""
    return _quantize(x, noise, None, True if out is None else out)[1]


def quantize_both(x, noise=None):
    """(quantize(x), quantize_t(x)) in one pass over x."""
    return _quantize(x, noise, True, True)


def dequantize(q, dtype="f32"):
    """The values q stands for, [rows, cols]."""
    t = _t()
    code, dt = _dtype(dtype)
    out = t.empty((q.rows, q.cols), dtype=dt, device=q.data.device)
    ags_mx_dequantize(q.c, out.data_ptr() or None, code, max(q.cols, 1), _stream(out.device))
    return out


def _workspace(nbytes, device):
    return _t().empty(nbytes, dtype=_t().uint8, device=device) if nbytes else None


def _output(out, rows, cols, dtype, accumulate, what, device):
    """(tensor [rows, cols], its type's code, row stride): `out`, or a new one
    of `dtype`."""
    if out is None:
        if accumulate:
            raise ValueError(f"accumulate needs {what}")
        code, dt = _dtype(dtype)
        return _t().empty((rows, cols), dtype=dt, device=device), code, max(cols, 1)
    code = _dtype(out.dtype)[0]
    if tuple(out.shape) != (rows, cols):
        raise ValueError(f"{what} must be [{rows}, {cols}]")
    return out, code, max(_matrix(out, what)[3], 1)


def product(a, b, dtype="bf16", out=None, accumulate=False):
    """a [m, k] times b' [k, n] (MX4s blocked along k): [m, n] of `dtype`, or
    written to `out` (2-D, unit column stride), added to it with
    `accumulate`."""
    dev = a.data.device
    out, code, stride = _output(out, a.rows, b.rows, dtype, accumulate, "out", dev)
    nbytes = ags_mx_product_workspace(a.rows, b.rows, a.cols)
    ws = _workspace(nbytes, dev)
    ags_mx_product(a.c, b.c, out.data_ptr() or None, code, stride, int(accumulate),
                   None if ws is None else ws.data_ptr(), nbytes, _stream(dev))
    return out


class Weight:
    """A linear layer's weight w [n, k] in 4 bits, in the two forms its
    products need: blocked along k (`forward`) and, transposed, along n
    (`backward`).  :meth:`update` stores new values (after an optimizer
    step) in the same buffers."""

    def __init__(self, w, forward=True, backward=True):
        w, n, k, _ = _matrix(w, "w")
        self.n, self.k = n, k
        self.rows = MX4(n, k, w.device) if forward else None
        self.cols = MX4(k, n, w.device) if backward else None
        if not forward and not backward:
            raise ValueError("a weight needs a forward or a backward form")
        self.update(w)

    def update(self, w):
        w, n, k, _ = _matrix(w, "w")
        if (n, k) != (self.n, self.k):
            raise ValueError(f"w must be [{self.n}, {self.k}]")
        _quantize(w, None, self.rows, self.cols)


def linear(x, w, dtype=None, save=False):
    """y = x w' for x [..., k] and a Weight w [n, k]: [..., n] of `dtype` (x's
    unless given).  save=True returns (y, saved): what linear_backward takes
    in place of x, stored in the same pass over it.  An x whose rows are not
    contiguous (transposed, broadcast) is copied first.  Autograd does not see the
    call (linear_backward is its backward pass), so an x that requires a
    gradient is refused where gradients are recorded."""
    t = _t()
    if x.requires_grad and t.is_grad_enabled():
        raise ValueError("x requires a gradient, which linear does not record: detach it, or call under "
                         "torch.no_grad() and linear_backward for the gradients")
    if w.rows is None:
        raise ValueError("the weight has no forward form")
    x2, rows, cols, stride = _matrix(x, "x", copy=True)
    if cols != w.k:
        raise ValueError(f"x must have {w.k} columns")
    out_code, out_dt = _dtype(x.dtype if dtype is None else dtype)
    shape = (*x.shape[:-1], w.n)
    dev = x.device
    y = t.empty(shape, dtype=out_dt, device=dev)
    if save:
        saved = MX4(w.k, rows, dev)
        nbytes = ags_mx_linear_save_workspace(rows, w.n, w.k)
        ws = _workspace(nbytes, dev)
        ags_mx_linear_save(x2.data_ptr() or None, _dtype(x.dtype)[0], rows, max(stride, 1), w.rows.c,
                           y.data_ptr() or None, out_code, max(w.n, 1), saved.c,
                           None if ws is None else ws.data_ptr(), nbytes, _stream(dev))
        return y, saved
    nbytes = ags_mx_linear_workspace(rows, w.n, w.k)
    ws = _workspace(nbytes, x.device)
    ags_mx_linear(x2.data_ptr() or None, _dtype(x.dtype)[0], rows, max(stride, 1), w.rows.c,
                  y.data_ptr() or None, out_code, max(w.n, 1), None if ws is None else ws.data_ptr(), nbytes,
                  _stream(x.device))
    return y


def linear_backward(dy, x, w, noise=None, dw=None, dw_dtype="f32", accumulate=False, need_dx=True):
    """The gradients of y = x w' given dy [..., n]: (dx [..., k] of dy's type,
    dw [n, k]).  x: the layer's input, or what linear(save=True) returned.
    noise: random bytes for dy's rounding (uint8, dy's shape).  dw: written
    there (a view of a replica's row, say), added with `accumulate`; else a
    new tensor of `dw_dtype`.  need_dx=False returns None for dx.  Inputs may
    have any strides, as for linear."""
    if need_dx and w.cols is None:
        raise ValueError("the weight has no backward form")
    dy2, rows, n, stride = _matrix(dy, "dy", copy=True)
    if n != w.n:
        raise ValueError(f"dy must have {w.n} columns")
    code, dev, k = _dtype(dy.dtype)[0], dy.device, w.k
    noise, n_ptr, n_stride = _noise(noise, rows, n, "dy", copy=True)
    dw, dw_code, dw_stride = _output(dw, n, k, dw_dtype, accumulate, "dw", dev)
    xt = x if isinstance(x, MX4) else quantize_t(x if _transposed(x) else _matrix(x, "x", copy=True)[0])
    if xt.shape != (k, rows):
        raise ValueError(f"x and dy differ in rows, or x has not {k} columns")
    dx = _t().empty((*dy.shape[:-1], k), dtype=dy.dtype, device=dev) if need_dx else None
    nbytes = ags_mx_linear_backward_workspace(rows, n, k, 1 if need_dx else 0)
    ws = _workspace(nbytes, dev)
    ags_mx_linear_backward(dy2.data_ptr() or None, code, rows, n, max(stride, 1), n_ptr, n_stride, xt.c,
                           w.cols.c if need_dx else None, dx.data_ptr() or None if need_dx else None, max(k, 1),
                           dw.data_ptr() or None, dw_code, dw_stride, int(accumulate),
                           None if ws is None else ws.data_ptr(), nbytes, _stream(dev))
    return dx, dw
