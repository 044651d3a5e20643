"""A rotary magnitude is a number of fp32, in which the kernels hold it."""
import ctypes
import math

import pytest

S = pytest.importorskip("paper_2607_14557_gb300.seer")
P, INVALID = 1 << 20, 1           # a 16-byte aligned address that no refused call follows


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_14557_gb300 import build
    build.build()


@pytest.mark.parametrize("magnitude", [1e39, -1e39, 3.5e38, 1.7e308, math.inf, -math.inf, math.nan])
def test_magnitudes_that_fp32_does_not_hold_are_refused(magnitude):
    rot = ctypes.byref(S.make_rotary(1e4, 32, magnitude=magnitude))
    pages = ctypes.byref(S.seer_pages(P, P, 10, 16, 4, 2, 64))
    assert S.lib().seer_rotate(P, 256, 1, 4, 64, 8, None, P, rot, 2 * P, 256, None) == INVALID
    assert b"magnitude" in S.lib().seer_last_error()
    assert S.lib().seer_kv_append_rotary(P, 512, 1, 4, 8, None, P, P, P, P, 2, rot, 2 * P, 384, pages, None) == INVALID
    assert b"magnitude" in S.lib().seer_last_error()


@pytest.mark.parametrize("magnitude", [3.4028234663852886e38, -3.4028234663852886e38, 0.0, 1e-45])
def test_the_largest_and_smallest_magnitudes_are_taken(magnitude):
    rot = ctypes.byref(S.make_rotary(1e4, 32, magnitude=magnitude))
    assert S.lib().seer_rotate(None, 0, 1, 4, 64, 0, None, None, rot, None, 0, None) == 0    # no rows
