"""Python binding of the libags orthogonalised updates (include/ags_muon.h):
argument marshalling only; everything runs in the HIP kernels of the library.
"""
from __future__ import annotations

import ctypes
import functools
import math

from . import ags
from .mx import _check, _dtype, _stream, _t, _workspace

AGS_MUON_MAX_STEPS = 32
EXPORTS = ("ags_muon_orthogonalize_workspace", "ags_muon_orthogonalize", "ags_muon_workspace_bytes",
           "ags_muon_init", "ags_muon_step", "ags_muon_set_lr", "ags_muon_destroy")
#: singular values s -> a s + b s^3 + c s^5, the same for every step
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


class ags_muon_schedule(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("reserved", ctypes.c_int32), ("abc", ctypes.POINTER(ctypes.c_double)),
                ("eps", ctypes.c_double)]


class ags_muon_matrix(ctypes.Structure):
    _fields_ = [("offset", ctypes.c_int64), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("scale", ctypes.c_double)]


class ags_muon_config(ctypes.Structure):
    _fields_ = [("n_matrices", ctypes.c_int32), ("K", ctypes.c_int32),
                ("matrices", ctypes.POINTER(ags_muon_matrix)), ("n_flat", ctypes.c_int64),
                ("grad_dtype", ctypes.c_int32), ("nesterov", ctypes.c_int32), ("lr", ctypes.c_double),
                ("momentum", ctypes.c_double), ("weight_decay", ctypes.c_double), ("schedule", ags_muon_schedule)]


_sig_done = False


def _lib():
    global _sig_done
    lib = ags.load_library()
    if not _sig_done:
        P, vp, c_int, i64, sz, dbl = (ctypes.POINTER, ctypes.c_void_p, ctypes.c_int, ctypes.c_int64,
                                      ctypes.c_size_t, ctypes.c_double)
        S, C = P(ags_muon_schedule), P(ags_muon_config)
        sig = {
            "ags_muon_orthogonalize_workspace": [i64, i64, i64, P(sz)],
            "ags_muon_orthogonalize": [vp, c_int, i64, i64, i64, i64, i64, S, vp, c_int, i64, i64, vp, sz, vp],
            "ags_muon_workspace_bytes": [C, P(sz)],
            "ags_muon_init": [C, vp, vp, vp, P(vp)],
            "ags_muon_step": [vp, vp, i64, vp],
            "ags_muon_set_lr": [vp, dbl],
        }
        for name, args in sig.items():
            f = getattr(lib, name)
            f.restype = c_int
            f.argtypes = args
        lib.ags_muon_destroy.restype = None
        lib.ags_muon_destroy.argtypes = [vp]
        _sig_done = True
    return lib


def make_schedule(steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """The ctypes schedule: `coefficients` is one (a, b, c) for every step, or
    one for each."""
    rows = [tuple(c) for c in coefficients] if hasattr(coefficients[0], "__len__") else [tuple(coefficients)] * steps
    if len(rows) != steps or any(len(r) != 3 for r in rows):
        raise ValueError("coefficients must be one (a, b, c), or one for each step")
    flat = (ctypes.c_double * max(3 * steps, 1))(*[float(x) for r in rows for x in r])
    return ags_muon_schedule(int(steps), 0, flat, float(eps))


def make_config(matrices, n_flat, K, *, grad_dtype="f32", lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True,
                steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """The ctypes config for matrices [(offset, rows, cols, scale)]."""
    arr = (ags_muon_matrix * max(len(matrices), 1))(*[ags_muon_matrix(int(o), int(r), int(c), float(s))
                                                      for o, r, c, s in matrices])
    cfg = ags_muon_config(len(matrices), int(K), arr, int(n_flat),
                          {"f32": ags.AGS_F32, "bf16": ags.AGS_BF16}[grad_dtype], int(bool(nesterov)), float(lr),
                          float(momentum), float(weight_decay), make_schedule(steps, coefficients, eps))
    cfg._keepalive = arr
    return cfg


# ------------------------------------------------------------ thin calls --
# Same names and arguments as the C functions; pointers are ints.


def ags_muon_orthogonalize_workspace(batch: int, rows: int, cols: int) -> int:
    b = ctypes.c_size_t(0)
    _check(_lib().ags_muon_orthogonalize_workspace(batch, rows, cols, ctypes.byref(b)))
    return b.value


def ags_muon_orthogonalize(d_x, dtype, batch, rows, cols, x_batch_stride, x_stride, schedule, d_out, out_dtype,
                           out_batch_stride, out_stride, d_workspace=None, workspace_bytes=0, stream=0):
    _check(_lib().ags_muon_orthogonalize(d_x, dtype, batch, rows, cols, x_batch_stride, x_stride,
                                         ctypes.byref(schedule), d_out, out_dtype, out_batch_stride, out_stride,
                                         d_workspace, workspace_bytes, stream))


def ags_muon_workspace_bytes(cfg) -> int:
    b = ctypes.c_size_t(0)
    _check(_lib().ags_muon_workspace_bytes(ctypes.byref(cfg), ctypes.byref(b)))
    return b.value


def ags_muon_init(cfg, d_w: int, d_m: int, stream: int = 0):
    h = ctypes.c_void_p()
    _check(_lib().ags_muon_init(ctypes.byref(cfg), d_w, d_m, stream, ctypes.byref(h)))
    return h


def ags_muon_step(handle, d_grads: int, replica_stride: int, stream: int = 0):
    _check(_lib().ags_muon_step(handle, d_grads, replica_stride, stream))


def ags_muon_set_lr(handle, lr: float):
    _check(_lib().ags_muon_set_lr(handle, float(lr)))


def ags_muon_destroy(handle):
    if handle is not None and handle.value:
        _lib().ags_muon_destroy(handle)


# ------------------------------------------------------- torch convenience --
# Device memory and streams come from torch; work goes on the current stream
# (choose another with torch.cuda.stream).

_usual = functools.lru_cache(maxsize=64)(make_schedule)


def _schedule(steps, coefficients, eps):
    """make_schedule, made once for each number of steps of the usual coefficients."""
    if coefficients is COEFFICIENTS and type(steps) is int and type(eps) is float:
        return _usual(steps, COEFFICIENTS, eps)
    return make_schedule(steps, coefficients, eps)


def _rows(x, what):
    """x [rows, cols] or [batch, rows, cols] with unit column stride, rows and
    matrices that do not overlap: (tensor, batch, rows, cols, batch stride, row
    stride)."""
    if not x.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor")
    if x.dim() not in (2, 3):
        raise ValueError(f"{what} must be [rows, cols] or [batch, rows, cols]")
    batch, rows, cols = (1, *x.shape) if x.dim() == 2 else x.shape
    row = x.stride(-2) if rows > 1 else cols
    each = x.stride(0) if batch > 1 else 0
    if (cols > 1 and x.stride(-1) != 1) or row < cols or (batch > 1 and each < (rows - 1) * row + cols):
        return None, batch, rows, cols, rows * cols, cols
    return x, batch, rows, cols, each, row


def orthogonalize(x, steps=5, coefficients=COEFFICIENTS, eps=1e-7, dtype="bf16", out=None):
    """Newton-Schulz steps of x [rows, cols] or of each matrix of x [batch,
    rows, cols] (fp32 or bf16), divided by their norms first: a new tensor of
    `dtype`, or `out`.  coefficients: one (a, b, c) for every step, or one for
    each.  An x whose rows are not contiguous is copied first."""
    t = _t()
    if x.requires_grad and t.is_grad_enabled():
        raise ValueError("x requires a gradient, which this call does not record: detach it")
    code = _dtype(x.dtype)[0]
    x2, batch, rows, cols, x_batch, x_row = _rows(x, "x")
    if x2 is None:
        x2 = x.contiguous()
    if out is None:
        out_code, dt = _dtype(dtype)
        out = t.empty(x.shape, dtype=dt, device=x.device)
        o_batch, o_row = rows * cols, cols
    else:
        out_code = _dtype(out.dtype)[0]
        if out.shape != x.shape or out.device != x.device:
            raise ValueError("out and x differ in shape or device")
        o, _, _, _, o_batch, o_row = _rows(out, "out")
        if o is None:
            raise ValueError("out must be contiguous along its last axis, without overlaps")
    schedule = _schedule(steps, coefficients, eps)
    nbytes = ags_muon_orthogonalize_workspace(batch, rows, cols)
    ws = _workspace(nbytes, x.device)
    ags_muon_orthogonalize(x2.data_ptr() or None, code, batch, rows, cols, x_batch, x_row, schedule,
                           out.data_ptr() or None, out_code, o_batch, o_row,
                           None if ws is None else ws.data_ptr(), nbytes, _stream(x.device))
    return out


def spectral_scale(rows, cols):
    """The usual factor of an update: the root of rows / cols where that is more
    than 1 (an orthogonal update then changes outputs of the layer evenly)."""
    return math.sqrt(max(1.0, rows / cols))


class Muon:
    """A Muon handle over torch tensors (device memory and streams only), for
    the matrices of the flat buffers whose other layers an ``ags.AGS`` handle
    updates.

    layers: (offset, rows, cols) or (offset, rows, cols, scale) of each matrix;
    a scale that is not given is :func:`spectral_scale`.  ``w`` and ``m`` are
    contiguous fp32 CUDA tensors of equal size, updated in place by
    :meth:`step`; its gradients are a contiguous [K, stride] tensor of
    ``grad_dtype``, as for ``ags.AGS``.  Graphs that captured a handle's steps
    share its workspace: their replays must not overlap.
    """

    def __init__(self, layers, w, m, K, *, grad_dtype="f32", lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True,
                 steps=5, coefficients=COEFFICIENTS, eps=1e-7, stream=None):
        import torch
        self.torch = torch
        for name, t in (("w", w), ("m", m)):
            if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous float32 CUDA tensor")
        if w.numel() != m.numel() or w.device != m.device:
            raise ValueError("w and m differ in size or device")
        if grad_dtype not in ("f32", "bf16"):
            raise ValueError(f"grad_dtype {grad_dtype!r} is neither 'f32' nor 'bf16'")
        self.K, self.grad_dtype = int(K), grad_dtype
        self.w, self.m = w, m
        matrices = [(*x, spectral_scale(x[1], x[2]))[:4] if x[1] and x[2] else (*x, 1.0)[:4] for x in layers]
        self.cfg = make_config(matrices, w.numel(), K, grad_dtype=grad_dtype, lr=lr, momentum=momentum,
                               weight_decay=weight_decay, nesterov=nesterov, steps=steps, coefficients=coefficients,
                               eps=eps)
        self.handle = ags_muon_init(self.cfg, w.data_ptr() or None, m.data_ptr() or None, self._stream(stream))

    def _stream(self, stream):
        if stream is None:
            return _stream(self.w.device)
        return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)

    def step(self, grads, stream=None):
        """One update from the replica gradients."""
        want = self.torch.float32 if self.grad_dtype == "f32" else self.torch.bfloat16
        if grads.dtype != want or not grads.is_cuda or not grads.is_contiguous() or grads.dim() != 2:
            raise ValueError(f"grads must be a contiguous 2-D CUDA tensor of dtype {want}")
        if grads.shape[0] != self.K:
            raise ValueError(f"grads has {grads.shape[0]} replicas, the handle has K={self.K}")
        ags_muon_step(self.handle, grads.data_ptr(), grads.shape[1], self._stream(stream))

    def set_lr(self, lr):
        ags_muon_set_lr(self.handle, lr)

    def close(self):
        if getattr(self, "handle", None) is not None:
            ags_muon_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
