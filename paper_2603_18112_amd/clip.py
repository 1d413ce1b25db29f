"""Python binding of libags gradient clipping (include/ags_clip.h): argument
marshalling only; norms, coefficients and scaled gradients are computed by
the HIP kernels of the library.
"""
from __future__ import annotations

import array
import ctypes
from operator import attrgetter

import numpy as np

from . import ags

AGS_CLIP_L2, AGS_CLIP_L1, AGS_CLIP_MAX = 0, 1, 2
KINDS = {"l2": AGS_CLIP_L2, "l1": AGS_CLIP_L1, "max": AGS_CLIP_MAX}
EXPORTS = ("ags_clip_workspace_bytes", "ags_clip_init", "ags_clip_norm", "ags_clip_apply",
           "ags_clip_destroy")

#: one run of consecutive elements (ags_clip_segment)
SEGMENT = np.dtype([("numel", np.int64), ("in_offset", np.int64), ("out_offset", np.int64),
                    ("in_base", np.int32), ("out_base", np.int32), ("group", np.int32),
                    ("reserved", np.int32)])


class ags_clip_config(ctypes.Structure):
    _fields_ = [("n_segments", ctypes.c_int32), ("segments", ctypes.c_void_p),
                ("n_in", ctypes.c_int32), ("in_dtypes", ctypes.c_void_p),
                ("n_out", ctypes.c_int32), ("out_dtypes", ctypes.c_void_p),
                ("n_groups", ctypes.c_int32), ("kind", ctypes.c_int32), ("eps", ctypes.c_double)]


_sig_done = False


def _lib():
    global _sig_done
    lib = ags.load_library()
    if not _sig_done:
        P, vp, c_int = ctypes.POINTER, ctypes.c_void_p, ctypes.c_int
        sig = {
            "ags_clip_workspace_bytes": (c_int, [P(ags_clip_config), P(ctypes.c_size_t)]),
            "ags_clip_init": (c_int, [P(ags_clip_config), vp, P(vp)]),
            "ags_clip_norm": (c_int, [vp, vp, vp, vp]),
            "ags_clip_apply": (c_int, [vp, vp, vp, ctypes.c_double, vp, vp]),
            "ags_clip_destroy": (None, [vp]),
        }
        for name, (res, args) in sig.items():
            f = getattr(lib, name)
            f.restype = res
            f.argtypes = args
        _sig_done = True
    return lib


def _check(status):
    if status != ags.AGS_OK:
        raise ags.AGSError(status, ags.ags_last_error(None))


def make_config(segments, in_dtypes, out_dtypes=(), n_groups=1, kind="l2", eps=1e-6):
    """An ags_clip_config (the arrays it points to are kept alive on it).
    segments: records of SEGMENT, or tuples (numel, in_base, in_offset,
    group[, out_base, out_offset]); dtypes: "f32" or "bf16" per tensor."""
    if isinstance(segments, np.ndarray):
        seg = np.ascontiguousarray(segments, dtype=SEGMENT)
    else:
        rows = [tuple(int(v) for v in s) for s in segments]
        seg = np.zeros(len(rows), SEGMENT)
        for i, r in enumerate(rows):
            ob, oo = r[4:6] if len(r) > 4 else (0, 0)
            seg[i] = (r[0], r[2], oo, r[1], ob, r[3], 0)
    idt = np.array([ags.DTYPES[d] for d in in_dtypes], np.int32)
    odt = np.array([ags.DTYPES[d] for d in out_dtypes], np.int32)
    cfg = ags_clip_config(n_segments=len(seg), segments=seg.ctypes.data, n_in=len(idt),
                          in_dtypes=idt.ctypes.data, n_out=len(odt), out_dtypes=odt.ctypes.data,
                          n_groups=int(n_groups), kind=KINDS[kind], eps=float(eps))
    cfg._keepalive = (seg, idt, odt)
    return cfg


# ------------------------------------------------------------ thin calls --


def ags_clip_workspace_bytes(cfg) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib().ags_clip_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)))
    return int(out.value)


def ags_clip_init(cfg, stream: int = 0):
    h = ctypes.c_void_p(0)
    _check(_lib().ags_clip_init(ctypes.byref(cfg), stream, ctypes.byref(h)))
    return h


def ags_clip_norm(handle, d_in, d_norms: int, stream: int = 0):
    """d_in: host address of an array of device pointers (or a ctypes array)."""
    _check(_lib().ags_clip_norm(handle, d_in, d_norms, stream))


def ags_clip_apply(handle, d_in, d_out, max_norm: float, d_norms: int, stream: int = 0):
    """d_in, d_out: as in ags_clip_norm; d_out None: in place."""
    _check(_lib().ags_clip_apply(handle, d_in, d_out, float(max_norm), d_norms, stream))


def ags_clip_destroy(handle):
    if handle is not None and handle.value:
        _lib().ags_clip_destroy(handle)


# ------------------------------------------------------- torch convenience --


def _dense(t):
    """Do t's elements lie side by side, in whatever order of its axes?"""
    n = 1
    for stride, size in sorted(zip(t.stride(), t.shape)):
        if size != 1:
            if stride != n:
                return False
            n *= size
    return True


def _name(dtype):
    return str(dtype).replace("torch.", "").replace("float32", "f32").replace("bfloat16", "bf16")


class GradClip:
    """A clipping handle over torch tensors (device memory and streams only).

    The handle is made for tensors of given sizes, types and groups; every
    call takes the tensors anew.  :meth:`norm` returns the norm of each
    group, :meth:`clip` scales the gradients of a group whose norm exceeds
    the bound and returns the norms before that.
    """

    def __init__(self, segments, in_numels, in_dtypes, out_numels=(), out_dtypes=(), n_groups=1,
                 kind="l2", eps=1e-6, stream=None):
        import torch
        self.torch = torch
        names = {"f32": torch.float32, "bf16": torch.bfloat16}
        for d in (*in_dtypes, *out_dtypes):
            if d not in names:
                raise ValueError(f"dtype {d!r} is not one of {sorted(names)}")
        self.in_numels, self.out_numels = list(map(int, in_numels)), list(map(int, out_numels))
        self.in_dtypes = [names[d] for d in in_dtypes]
        self.out_dtypes = [names[d] for d in out_dtypes]
        if kind not in KINDS:
            raise ValueError(f"kind {kind!r} is not one of {sorted(KINDS)}")
        if len(self.in_numels) != len(self.in_dtypes) or len(self.out_numels) != len(self.out_dtypes):
            raise ValueError("one type for each tensor")
        self.n_groups = int(n_groups)
        self.cfg = make_config(segments, in_dtypes, out_dtypes, n_groups, kind, eps)
        seg = self.cfg._keepalive[0]
        # no segment reaches past the tensors the calls are given
        for base, off, sizes in (("in_base", "in_offset", self.in_numels),
                                 ("out_base", "out_offset", self.out_numels)):
            if not len(sizes) or not len(seg):
                continue
            if seg[base].min() < 0 or seg[base].max() >= len(sizes):
                raise ValueError(f"{base} out of range")
            if np.any((seg[off] + seg["numel"] > np.asarray(sizes)[seg[base]]) & (seg["numel"] > 0)):
                raise ValueError(f"a segment ends past its tensor ({off})")
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.handle = ags_clip_init(self.cfg, self._stream(stream))
        # every segment is a whole tensor: the order of its elements is free
        self.whole = bool(np.all((seg["in_offset"] == 0)
                                 & (seg["numel"] == np.asarray(self.in_numels, np.int64)[seg["in_base"]])))

    @classmethod
    def for_tensors(cls, tensors, *, groups=None, layers=None, out_dtype=None, kind="l2", eps=1e-6,
                    stream=None):
        """For tensors of these sizes and types: one group, or the group of
        each.  With `layers` ((offset, numel, flags) of a flat layout, one per
        tensor) :meth:`clip` can write them into a flat row of `out_dtype`
        (by default fp32) that reaches at least to the last layer's end; its
        tensors are contiguous then.  Norms and scaling in place take dense
        tensors whose axes lie in any order (channels last) too."""
        numels = [t.numel() for t in tensors]
        dtypes = [_name(t.dtype) for t in tensors]
        groups = [0] * len(numels) if groups is None else [int(g) for g in groups]
        if len(groups) != len(numels):
            raise ValueError("one group for each tensor")
        n_groups = max(groups, default=0) + 1
        if layers is None:
            segments = [(n, i, 0, g) for i, (n, g) in enumerate(zip(numels, groups))]
            return cls(segments, numels, dtypes, n_groups=n_groups, kind=kind, eps=eps, stream=stream)
        if [int(n) for _, n, _ in layers] != numels:
            raise ValueError("layers and tensors differ in size")
        segments = [(n, i, 0, g, 0, int(o))
                    for i, (n, g, (o, _, _)) in enumerate(zip(numels, groups, layers))]
        end = max((int(o) + int(n) for o, n, _ in layers), default=0)
        return cls(segments, numels, dtypes, [end], [out_dtype or "f32"], n_groups, kind, eps, stream)

    @classmethod
    def for_stack(cls, layers, K, stride, *, dtype="f32", out_dtype=None, kind="l2", eps=1e-6,
                  stream=None):
        """For a replica stack [K, stride]: a group for each replica over the
        elements of its layers (gaps between layers are never read).  With
        `out_dtype` the clipped rows go to a stack of that type, its gaps
        unwritten; without it they are scaled in place."""
        K, stride = int(K), int(stride)
        o = np.array([int(o) for o, _, _ in layers], np.int64)
        n = np.array([int(n) for _, n, _ in layers], np.int64)
        if len(o) and int((o + n).max()) > stride:
            raise ValueError("a layer ends past the row stride")
        seg = np.zeros((K, len(o)), SEGMENT)
        rows = np.arange(K, dtype=np.int64)[:, None] * stride
        seg["numel"], seg["in_offset"], seg["out_offset"] = n, o + rows, o + rows
        seg["group"] = np.arange(K)[:, None]
        total = [K * stride]
        outs = ([], []) if out_dtype is None else (total, [out_dtype])
        return cls(seg.reshape(-1), total, [dtype], outs[0], outs[1], K, kind, eps, stream)

    def _stream(self, stream):
        if stream is None:
            raw = getattr(self.torch._C, "_cuda_getCurrentRawStream", None)
            if raw is not None:  # 0.1 us instead of 2
                return raw(self.device.index)
            stream = self.torch.cuda.current_stream(self.device)
        return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)

    def _pointers(self, what, tensors, numels, dtypes, longer=False, any_order=False):
        """Host array of the tensors' addresses (the library checks that they
        lie in device memory).  any_order: a dense tensor whose axes lie in
        another order (channels last) will do.  One pass of a C function over the list for each
        property: written as a loop the checks of 161 tensors take longer than
        the kernels."""
        T = self.torch.Tensor
        sizes = list(map(T.numel, tensors))
        if sizes != numels and not (longer and len(sizes) == len(numels)
                                    and all(a >= b for a, b in zip(sizes, numels))):
            raise ValueError(f"{what} differ in number or size from the handle's")
        if list(map(attrgetter("dtype"), tensors)) != dtypes:
            raise ValueError(f"{what} differ in type from the handle's")
        if not all(map(T.is_contiguous, tensors)) and not (
                any_order and all(t.is_contiguous() or _dense(t) for t in tensors)):
            raise ValueError(f"{what} must be contiguous")
        return array.array("Q", map(T.data_ptr, tensors))

    def _norms(self, stream):
        t = self.torch
        if stream is None:
            return t.empty(self.n_groups, dtype=t.float32, device=self.device)
        # the allocator reuses a tensor's memory in the order of its own stream
        if not hasattr(stream, "cuda_stream"):
            stream = t.cuda.ExternalStream(int(stream), device=self.device)
        with t.cuda.stream(stream):
            return t.empty(self.n_groups, dtype=t.float32, device=self.device)

    def norm(self, tensors, stream=None):
        """The norm of each group, fp32 [n_groups] on the device."""
        p = self._pointers("the gradients", tensors, self.in_numels, self.in_dtypes, any_order=self.whole)
        norms = self._norms(stream)
        ags_clip_norm(self.handle, p.buffer_info()[0], norms.data_ptr(), self._stream(stream))
        return norms

    def clip(self, tensors, max_norm, out=None, stream=None):
        """Scale each group by min(1, max_norm / (norm + eps)), in place or
        into the tensors of `out`; returns the norms."""
        p = self._pointers("the gradients", tensors, self.in_numels, self.in_dtypes,
                           any_order=self.whole and out is None)
        q = None
        if out is not None:
            if not self.out_numels:
                raise ValueError("the handle was made without outputs")
            q = self._pointers("the outputs", out, self.out_numels, self.out_dtypes, True)
        norms = self._norms(stream)
        ags_clip_apply(self.handle, p.buffer_info()[0], None if q is None else q.buffer_info()[0], max_norm,
                       norms.data_ptr(), self._stream(stream))
        return norms

    def close(self):
        if getattr(self, "handle", None) is not None:
            ags_clip_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
