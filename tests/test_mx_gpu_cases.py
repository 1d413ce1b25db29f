"""What the GPU tests of 4-bit products take for granted, shown on the CPU:
that whole-number products are exact in fp32, and that the products meant to
be cut into parts are."""
import os

import numpy as np
import pytest

import test_gpu_mx as gpu
from paper_2603_18112_amd import _build, mx


def _gpu_cases(*names):
    return [c for name in names for mark in getattr(gpu, name).pytestmark if mark.name == "parametrize"
            for c in mark.args[1]]


@pytest.mark.parametrize("m,n,k", _gpu_cases("test_products_of_whole_numbers_are_exact",
                                             "test_products_ahead_of_memory",
                                             "test_parts_joined_over_rows_of_any_length"))
def test_whole_number_products_are_exact_in_fp32(m, n, k):
    """The products that the GPU tests compare exactly: multiples of 1/4 whose
    magnitudes sum to less than 2^22, so that fp32 holds every partial sum of
    every order."""
    a, b = gpu.whole(m, k, 1), gpu.whole(n, k, 2)
    assert np.array_equal(a * 2, np.rint(a * 2)) and np.array_equal(b * 2, np.rint(b * 2))
    assert (np.abs(a) @ np.abs(b).T).max() < 2 ** 22


@pytest.mark.parametrize("m,n,k", _gpu_cases("test_parts_joined_over_rows_of_any_length"))
def test_the_products_that_test_parts_are_in_parts(m, n, k):
    if not os.path.exists(_build.LIB):
        _build.build()
    assert mx.ags_mx_product_workspace(m, n, k) >= 2 * m * n * 4
