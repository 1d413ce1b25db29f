"""libags gradient clipping on the host: the binding's names, struct sizes and
argument checks (no GPU; only calls that fail before any HIP call)."""
import ctypes
import os
import re

import pytest

from paper_2603_18112_amd import _build, ags, clip

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB):
        _build.build()
    return clip._lib()


def test_header_declares_the_binding_names():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ags_clip.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ags_[a-z_]+)\s*\(", text))) == sorted(clip.EXPORTS)


def test_struct_sizes_match_the_header():
    assert clip.SEGMENT.itemsize == 3 * 8 + 4 * 4
    assert ctypes.sizeof(clip.ags_clip_config) == 8 + 8 + 8 + 8 + 8 + 8 + 4 + 4 + 8


def _status(segments, in_dtypes=("f32",), **kw):
    raw = {k: kw.pop(k) for k in ("kind_value", "dtype_value", "reserved") if k in kw}
    cfg = clip.make_config(segments, in_dtypes, **kw)
    if "kind_value" in raw:
        cfg.kind = raw["kind_value"]
    if "dtype_value" in raw:
        cfg._keepalive[1][0] = raw["dtype_value"]
    if "reserved" in raw:
        cfg._keepalive[0]["reserved"][0] = raw["reserved"]
    try:
        return ags.AGS_OK, clip.ags_clip_workspace_bytes(cfg)
    except ags.AGSError as e:
        return e.status, str(e)


def test_workspace_bytes(lib):
    st, n = _status([(100, 0, 0, 0)])
    assert st == ags.AGS_OK and 0 < n < 32768
    st, n = _status([(1 << 33, 0, 0, 0)])          # 8e9 elements: some 4096 pieces
    assert st == ags.AGS_OK and n < 1 << 20
    st, n = _status([])                              # nothing to read is no error
    assert st == ags.AGS_OK
    st, n = _status([(10, i, 0, 0) for i in range(3000)], ["f32"] * 3000)
    assert st == ags.AGS_OK


@pytest.mark.parametrize("segments,kw,status", [
    ([(10, 1, 0, 0)], {}, ags.AGS_E_ARG),                                 # no such tensor
    ([(10, -1, 0, 0)], {}, ags.AGS_E_ARG),
    ([(10, 0, 0, 1)], {}, ags.AGS_E_ARG),                                 # no such group
    ([(10, 0, 0, -1)], {}, ags.AGS_E_ARG),
    ([(-1, 0, 0, 0)], {}, ags.AGS_E_LAYOUT),
    ([(10, 0, -8, 0)], {}, ags.AGS_E_LAYOUT),
    ([(1 << 61, 0, 0, 0)], {}, ags.AGS_E_LAYOUT),
    ([(1 << 60, 0, 0, 0), (1 << 60, 0, 0, 0)], {}, ags.AGS_E_LAYOUT),    # the sum passes the limit
    ([(1 << 50, 0, 0, 0)], {}, ags.AGS_E_LAYOUT),                         # a piece of over 2^30 elements
    ([(10, 0, 0, 0)], dict(n_groups=0), ags.AGS_E_ARG),
    ([(10, 0, 0, 0)], dict(eps=-1.0), ags.AGS_E_ARG),
    ([(10, 0, 0, 0)], dict(eps=float("nan")), ags.AGS_E_ARG),
    ([(10, 0, 0, 0)], dict(kind_value=3), ags.AGS_E_ARG),
    ([(10, 0, 0, 0)], dict(dtype_value=2), ags.AGS_E_ARG),
    ([(10, 0, 0, 0)], dict(reserved=1), ags.AGS_E_ARG),
    ([(10, 0, 0, 0, 1, 0)], dict(out_dtypes=["f32"]), ags.AGS_E_ARG),     # no such output
    ([(10, 0, 0, 0, 0, -8)], dict(out_dtypes=["f32"]), ags.AGS_E_LAYOUT),
    ([(10, 0, 0, 0, 0, 0), (10, 0, 10, 0, 0, 9)], dict(out_dtypes=["f32"]), ags.AGS_E_LAYOUT),
])
def test_config_validation(lib, segments, kw, status):
    st, msg = _status(segments, **kw)
    assert st == status, msg
    assert ags.ags_last_error(None)


def test_null_arguments_are_errors(lib):
    n = ctypes.c_size_t()
    assert lib.ags_clip_workspace_bytes(None, ctypes.byref(n)) == ags.AGS_E_ARG
    cfg = clip.make_config([(10, 0, 0, 0)], ["f32"])
    assert lib.ags_clip_workspace_bytes(ctypes.byref(cfg), None) == ags.AGS_E_ARG
    assert lib.ags_clip_init(ctypes.byref(cfg), None, None) == ags.AGS_E_ARG
    cfg.segments = None
    assert lib.ags_clip_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)) == ags.AGS_E_ARG
    assert lib.ags_clip_norm(None, None, None, None) == ags.AGS_E_ARG
    assert lib.ags_clip_apply(None, None, None, 1.0, None, None) == ags.AGS_E_ARG
    lib.ags_clip_destroy(None)


def test_workspace_cap_gives_nomem_before_any_device_call(lib, monkeypatch):
    cfg = clip.make_config([(1 << 20, 0, 0, 0)], ["f32"])
    monkeypatch.setenv("AGS_MAX_WORKSPACE_BYTES", str(clip.ags_clip_workspace_bytes(cfg) - 1))
    with pytest.raises(ags.AGSError) as e:
        clip.ags_clip_init(cfg)
    assert e.value.status == ags.AGS_E_NOMEM


@pytest.mark.parametrize("n_groups", [(1 << 30) + 1, (1 << 31) - 1])
def test_group_numbers_that_a_kernel_could_not_count_to(lib, n_groups):
    # the kernels step over the groups in 32-bit numbers, up to 256 at a time
    st, msg = _status([(10, 0, 0, 0)], n_groups=n_groups)
    assert st == ags.AGS_E_LAYOUT and "groups" in msg
