"""Python binding of the libags gated feed-forward products
(include/ags_glu.h): argument marshalling only; everything runs in the HIP
kernels of the library.
"""
from __future__ import annotations

import ctypes

from . import ags
from .mx import _check, _dtype, _matrix, _output, _stream, _t, _workspace
from .norm import _recorded

AGS_GLU_SILU, AGS_GLU_GELU = 0, 1
EXPORTS = ("ags_glu_bytes", "ags_glu_store", "ags_glu_forward_workspace", "ags_glu_forward",
           "ags_glu_backward_workspace", "ags_glu_backward")


class ags_glu_weight(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64), ("k", ctypes.c_int64)]


_sig_done = False


def _lib():
    global _sig_done
    lib = ags.load_library()
    if not _sig_done:
        P, vp, c_int, i32, i64, sz = (ctypes.POINTER, ctypes.c_void_p, ctypes.c_int, ctypes.c_int32,
                                      ctypes.c_int64, ctypes.c_size_t)
        W = P(ags_glu_weight)
        sig = {
            "ags_glu_bytes": [i64, i64, P(sz)],
            "ags_glu_store": [vp, i64, vp, i64, c_int, W, vp],
            "ags_glu_forward_workspace": [i64, i64, i64, P(sz)],
            "ags_glu_forward": [vp, i64, i64, W, i32, vp, c_int, i64, vp, vp, sz, vp],
            "ags_glu_backward_workspace": [i64, i64, i64, P(sz)],
            "ags_glu_backward": [vp, i64, vp, i64, i64, vp, W, i32, vp, i64, vp, vp, c_int, i64, i32, vp, sz, vp],
        }
        for name, args in sig.items():
            f = getattr(lib, name)
            f.restype = c_int
            f.argtypes = args
        _sig_done = True
    return lib


# ------------------------------------------------------------ thin calls --
# Same names and arguments as the C functions; pointers are ints.


def _size(name, *args):
    b = ctypes.c_size_t(0)
    _check(getattr(_lib(), name)(*args, ctypes.byref(b)))
    return b.value


def ags_glu_bytes(n: int, k: int) -> int:
    return _size("ags_glu_bytes", n, k)


def ags_glu_store(d_gate, gate_stride, d_up, up_stride, dtype, w, stream=0):
    _check(_lib().ags_glu_store(d_gate, gate_stride, d_up, up_stride, dtype, ctypes.byref(w), stream))


def ags_glu_forward_workspace(rows: int, n: int, k: int) -> int:
    return _size("ags_glu_forward_workspace", rows, n, k)


def ags_glu_forward(d_x, rows, x_stride, w, act, d_h, h_dtype, h_stride, d_saved=None, d_workspace=None,
                    workspace_bytes=0, stream=0):
    _check(_lib().ags_glu_forward(d_x, rows, x_stride, ctypes.byref(w), act, d_h, h_dtype, h_stride, d_saved,
                                  d_workspace, workspace_bytes, stream))


def ags_glu_backward_workspace(rows: int, n: int, k: int) -> int:
    return _size("ags_glu_backward_workspace", rows, n, k)


def ags_glu_backward(d_dh, dh_stride, d_x, rows, x_stride, d_saved, w, act, d_dx, dx_stride, d_dgate, d_dup,
                     dw_dtype, dw_stride, accumulate=0, d_workspace=None, workspace_bytes=0, stream=0):
    _check(_lib().ags_glu_backward(d_dh, dh_stride, d_x, rows, x_stride, d_saved, ctypes.byref(w), act, d_dx,
                                   dx_stride, d_dgate, d_dup, dw_dtype, dw_stride, accumulate, d_workspace,
                                   workspace_bytes, stream))


# ------------------------------------------------------- torch convenience --
# Device memory and streams come from torch; work goes on the current stream
# (choose another with torch.cuda.stream).


def _act(act):
    if act not in ("silu", "gelu"):
        raise ValueError(f"act {act!r} is neither 'silu' nor 'gelu'")
    return AGS_GLU_SILU if act == "silu" else AGS_GLU_GELU


def _bf16(x, what, device=None):
    if x.dtype is not _t().bfloat16:
        raise ValueError(f"{what} must be bfloat16")
    if device is not None and x.device != device:
        raise ValueError(f"{what} is on another device than the weight")
    return _matrix(x, what, copy=True)


class Weight:
    """The two weights gate, up [n, k] of a gated block, in bf16, laid out for
    its products.  :meth:`update` stores new values (after an optimizer step)
    in the same buffer.  It is a copy that autograd does not see, of parameters
    that require a gradient too: gated_linear_backward returns theirs."""

    def __init__(self, gate, up):
        gate, self.n, self.k, _ = _matrix(gate, "gate")
        t = _t()
        self.data = t.empty(ags_glu_bytes(self.n, self.k) // 2, dtype=t.bfloat16, device=gate.device)
        self.c = ags_glu_weight(self.data.data_ptr() or None, self.n, self.k)
        self.update(gate, up)

    @property
    def lines(self):
        return 2 * (-(-self.n // 16) * 16)

    def update(self, gate, up):
        gate, n, k, g_stride = _matrix(gate, "gate")
        up, n2, k2, u_stride = _matrix(up, "up")
        if (n, k) != (self.n, self.k) or (n2, k2) != (n, k):
            raise ValueError(f"gate and up must be [{self.n}, {self.k}]")
        if gate.dtype is not up.dtype or gate.device != self.data.device or up.device != self.data.device:
            raise ValueError("gate and up differ in type, or are on another device than the weight")
        ags_glu_store(gate.data_ptr() or None, max(g_stride, 1), up.data_ptr() or None, max(u_stride, 1),
                      _dtype(gate.dtype)[0], self.c, _stream(self.data.device))


def gated_linear(x, w, act="silu", dtype=None, save=False):
    """h = act(x gate') * (x up') for x [..., k] (bf16) and a Weight of [n, k]:
    [..., n] of `dtype` (bf16 unless given).  save=True returns (h, saved): g and
    u in 24 bits each for the backward pass, 6 bytes a hidden unit and row.  An x whose
    rows are not contiguous is copied first.  Autograd does not see the call
    (gated_linear_backward is its backward pass), so an x that requires a
    gradient is refused where gradients are recorded."""
    t = _t()
    _recorded(x)
    act, dev = _act(act), w.data.device
    x2, rows, k, stride = _bf16(x, "x", dev)
    if k != w.k:
        raise ValueError(f"x must have {w.k} columns")
    code, dt = _dtype(t.bfloat16 if dtype is None else dtype)
    h = t.empty((*x.shape[:-1], w.n), dtype=dt, device=dev)
    saved = t.empty((rows, 3 * w.lines), dtype=t.uint8, device=dev) if save else None
    nbytes = ags_glu_forward_workspace(rows, w.n, k)
    ws = _workspace(nbytes, dev)
    ags_glu_forward(x2.data_ptr() or None, rows, max(stride, 1), w.c, act, h.data_ptr() or None, code, max(w.n, 1),
                    (saved.data_ptr() or None) if save else None, None if ws is None else ws.data_ptr(), nbytes,
                    _stream(dev))
    return (h, saved) if save else h


def gated_linear_backward(dh, x, w, saved=None, act="silu", dgate=None, dup=None, dw_dtype="bf16",
                          accumulate=False, need_dx=True, need_dw=True):
    """The gradients of gated_linear given dh [..., n] (bf16): (dx [..., k] in
    bf16, dgate [n, k], dup [n, k]), None in place of those not wanted.  saved:
    what gated_linear(save=True) returned; without it g and u are computed
    again.  dgate, dup: written there (views of a replica's row, say; equal
    types and strides), added with `accumulate`; else new tensors of
    `dw_dtype`.  Inputs may have any strides, as for gated_linear."""
    t = _t()
    act, dev = _act(act), w.data.device
    dh2, rows, n, dh_stride = _bf16(dh, "dh", dev)
    x2, x_rows, k, x_stride = _bf16(x, "x", dev)
    if n != w.n or k != w.k or rows != x_rows:
        raise ValueError(f"dh and x must have {w.n} and {w.k} columns and equal rows")
    if saved is not None and (tuple(saved.shape) != (rows, 3 * w.lines) or saved.dtype is not t.uint8 or
                              saved.device != dev or not saved.is_contiguous()):
        raise ValueError("saved is not what gated_linear returned for this x and w")
    if not need_dw and (dgate is not None or dup is not None):
        raise ValueError("dgate or dup is given but not wanted")
    code, dw_stride = ags.AGS_BF16, max(k, 1)
    if need_dw:
        if (dgate is None) != (dup is None):
            raise ValueError("dgate and dup go together")
        dgate, code, dw_stride = _output(dgate, n, k, dw_dtype, accumulate, "dgate", dev)
        dup, code2, stride2 = _output(dup, n, k, dw_dtype, accumulate, "dup", dev)
        if code != code2 or (n > 1 and dw_stride != stride2):
            raise ValueError("dgate and dup differ in type or row stride")
        if dgate.device != dev or dup.device != dev:
            raise ValueError("dgate or dup is on another device than the weight")
    dx = t.empty((*x.shape[:-1], k), dtype=t.bfloat16, device=dev) if need_dx else None
    if not (need_dx or need_dw):
        return None, None, None
    nbytes = ags_glu_backward_workspace(rows, n, k)
    ws = _workspace(nbytes, dev)
    if k and (rows or need_dw and n):
        ags_glu_backward(dh2.data_ptr() or None, max(dh_stride, 1), x2.data_ptr() or None, rows, max(x_stride, 1),
                         None if saved is None else saved.data_ptr() or None, w.c, act,
                         (dx.data_ptr() or None) if need_dx else None, max(k, 1),
                         (dgate.data_ptr() or None) if need_dw else None,
                         (dup.data_ptr() or None) if need_dw else None, code, dw_stride, int(accumulate),
                         None if ws is None else ws.data_ptr(), nbytes, _stream(dev))
    return dx, dgate, dup
