"""Workspaces of the orthogonalised updates (no GPU)."""
import os

import pytest

from paper_2603_18112_amd import _build, muon


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(_build.LIB):
        _build.build()


def _handle(matrices, n_flat, K=1):
    return muon.ags_muon_workspace_bytes(muon.make_config(matrices, n_flat, K))


@pytest.mark.parametrize("rows,cols", [(1_000_000, 1), (1, 1_000_000), (1 << 20, 16), (16, 100_000), (9, 2048), (1, 1)])
def test_thin_matrices_take_what_they_use(rows, cols):
    """Sums of products of each 128 of the longer side, in at most 256 parts of 2 KiB; a handle's
    U in fp32 before them, and a block's entry of 16 bytes in the tables of two launches."""
    parts = min(256, -(-max(rows, cols) // 128))
    assert muon.ags_muon_orthogonalize_workspace(1, rows, cols) <= max(65536, 2048 * parts)
    assert muon.ags_muon_orthogonalize_workspace(1, rows, cols) >= 2048 * -(-parts // 2)
    empty, n = _handle([], 1 << 25), rows * cols
    grown = _handle([(0, rows, cols, 1.0)], 1 << 25) - empty
    assert 4 * n + 2048 * -(-parts // 2) <= grown <= 4 * n + 2048 * parts + 16 * (parts + n // 4096 + 1) + 4096


@pytest.mark.parametrize("rows,cols", [(17, 64), (64, 17), (1000, 512), (4096, 4096), (2048, 4608)])
def test_others_take_what_the_header_says(rows, cols):
    pad = lambda x: -(-x // 64) * 64
    side = min(rows, cols)
    least = rows * pad(cols) * 8 + side * pad(side) * 4
    one = muon.ags_muon_orthogonalize_workspace(1, rows, cols)
    assert least <= one <= least + 8192 + 64
    grown = _handle([(0, rows, cols, 1.0)], 1 << 25) - _handle([], 1 << 25)
    assert least <= grown <= least + 2 ** 16 + 0.05 * least
