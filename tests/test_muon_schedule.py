"""Which schedules the orthogonalised updates take (no GPU): operands scaled for fp16
must stay in its range, the roundings of the steps before included."""
import math
import os
import random

import numpy as np
import pytest

from paper_2603_18112_amd import _build, ags, muon


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(_build.LIB):
        _build.build()


def _taken(abc):
    """An empty matrix: the schedule is all that is looked at."""
    try:
        muon.ags_muon_orthogonalize(None, ags.AGS_F32, 1, 0, 40, 0, 40,
                                    muon.make_schedule(steps=len(abc), coefficients=abc), None, ags.AGS_F32, 0, 40)
        return True
    except ags.AGSError as e:
        assert e.status == ags.AGS_E_ARG
        return False


def _half(x, scale):
    with np.errstate(over="ignore"):
        return float(np.float16(np.float32(x * scale))) / scale


def _fits(abc, n):
    """The steps of a row of n equal elements, the only one that is not zero, with the
    kernels' roundings: all of its elements are rounded the same way, and A and b A + c A A
    are one number each."""
    x = float(np.float32(n ** -0.5))
    for a, b, c in abc:
        xh = _half(x, 2.0 ** 15)
        gram = _half(float(np.float32(n * xh * xh)), 2.0 ** 15)
        p = _half(float(np.float32(b * gram + c * gram * gram)), 2.0 ** 14)
        if not (math.isfinite(xh) and math.isfinite(gram) and math.isfinite(p)):
            return False
        x = float(np.float32(a * x + p * xh))
    return True


# singular values near 1.4 whose rounding the next step's slope multiplies: A or b A + c A A
# passes 2^16
TOO_NEAR = [
    [(0.1853026011107958, -2.914232134960426, 4.100832248150128),
     (-0.62091932026449, -1.247276887631736, 1.1198445028567179),
     (3.724285890779864, 5.154794959443859, -3.2337261148991714)],
    [(2.468364920841308, -6.651318988511642, 5.548227161461792),
     (-0.4125069798169615, -0.16750163558087933, -0.08170701878952173),
     (1.1134822831592075, 7.194331653508671, -4.871086670279529)],
    [(0.4697663218418605, 4.986945886608942, -6.809187048087021),
     (0.6719559063378127, -1.2146550942420553, 0.7651985031158028),
     (3.343721628943147, 1.8038478244610259, -1.8919752846903382)],
]


@pytest.mark.parametrize("abc", TOO_NEAR)
def test_roundings_that_pass_the_range_are_refused(abc):
    assert not _fits(abc, 777)
    assert not _taken(abc)


@pytest.mark.parametrize("abc", [[(3.4445, -4.775, 2.0315)] * 32, [(1.5, -0.5, 0.0)] * 32, [(2.0, -1.5, 0.5)] * 32,
                                 [(1.875, -1.25, 0.375)] * 32, [(3.0, -3.2, 1.2)] * 10, [(4.0, 0.0, 0.0)],
                                 [(3.4445, -4.775, 2.0315)] * 4 + [(1.5, -0.5, 0.0)], [(1.0, 0.0, 0.0)] * 32])
def test_schedules_in_use_are_taken(abc):
    assert _taken(abc)
    assert all(_fits(abc, n) for n in (64, 777, 1000, 3001))


def test_no_schedule_that_is_taken_leaves_the_range():
    """Random steps scaled to come out near the range's end, as those above were found."""
    rng, taken = random.Random(7), 0
    for _ in range(20000):
        abc, top = [], 1.0
        for _ in range(rng.randint(2, 4)):
            a, b, c = rng.uniform(-6, 6), rng.uniform(-20, 20) / top ** 2, rng.uniform(-25, 25) / top ** 4
            s = [top * i / 200 for i in range(201)]
            most = max(abs(x * (a + b * x ** 2 + c * x ** 4)) for x in s)
            to = 1.41 * rng.uniform(0.93, 1.0) / most
            abc.append((a * to, b * to, c * to))
            top = most * to
            if max(abs(abc[-1][1] * x ** 2 + abc[-1][2] * x ** 4) for x in s) > 4.0:
                break
        else:
            if _taken(abc):
                taken += 1
                assert all(_fits(abc, n) for n in (64, 513, 777, 1000, 2047, 3001)), abc
    assert taken > 50
