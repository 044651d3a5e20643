"""Calls of the paged cache for no rows: empty buffers may have no address, and nothing is launched, so
these run without a GPU."""
import ctypes
import math

import pytest

S = pytest.importorskip("paper_2607_14557_gb300.seer")
P = 1 << 20


@pytest.fixture(scope="module")
def L():
    from paper_2607_14557_gb300 import build
    build.build()
    return S.lib()


def pages():
    return ctypes.byref(S.seer_pages(P, P, 10, 16, 4, 2, 64))


def test_calls_for_no_rows_take_buffers_without_an_address(L):
    for dt in (0, 1, 2):
        assert L.seer_kv_append(None, 0, dt, 4, 0, None, None, None, 1e4, None, 0, pages(), None) == 0
        assert L.seer_attention_causal(None, 0, None, 0, None, 0, None, 0, dt, P, 2, 0, 4, 2, 64, None) == 0
        assert L.seer_attention_tree(None, 0, None, 0, dt, P, P, None, 2, 0, 4, 8, pages(), None, 0, None) == 0


def test_what_is_wrong_with_a_call_for_no_rows_is_refused(L):
    assert L.seer_kv_append(None, 0, 1, 4, 0, None, None, None, math.nan, None, 0, pages(), None) == 1
    assert L.seer_kv_append(None, 0, 1, 4, 0, None, None, None, 1e4, None, 0, None, None) == 1
    assert L.seer_attention_causal(None, 0, None, 0, None, 0, None, 0, 1, P, 2, 0, 5, 2, 64, None) == 1
    assert L.seer_attention_causal(None, 0, None, 0, None, 0, None, 0, 1, None, 2, 0, 4, 2, 64, None) == 1
    assert L.seer_attention_tree(None, 0, None, 0, 1, P, None, None, 2, 0, 4, 8, pages(), None, 0, None) == 1
