"""Which eps the layer norm takes (no GPU; only calls that fail, or return, before any
HIP call)."""
import os

import pytest

from paper_2603_18112_amd import _build, ags, norm

X, Y = 0x1000000000, 0x2000000000       # never dereferenced


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(_build.LIB):
        _build.build()


@pytest.mark.parametrize("eps", [3.5e38, 1e39, 1e300, float("inf"), -float("inf"), float("nan"), -1e-300])
def test_refused(eps):
    for rows in (0, 4):
        with pytest.raises(ags.AGSError) as e:
            norm.ags_layer_norm(X, ags.AGS_F32, rows, 64, 64, None, None, ags.AGS_F32, eps, Y, ags.AGS_F32, 64)
        assert e.value.status == ags.AGS_E_ARG and "eps" in ags.ags_last_error(None)


@pytest.mark.parametrize("eps", [0.0, 1e-300, 1e-40, 1e-5, 3.4e38])
def test_taken(eps):
    norm.ags_layer_norm(None, ags.AGS_F32, 0, 64, 64, None, None, ags.AGS_F32, eps, None, ags.AGS_F32, 64)
