"""The sizes that one launch of the sequence operators takes, and what they say past them
(nothing here reaches the device)."""
import ctypes
import os

import pytest

from paper_2012_01170_amd import _lib as L

A = 1 << 42  # stand-in device addresses, never dereferenced
UNSUPPORTED = 8


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        from paper_2012_01170_amd import build
        build.build()
    return L.lib()


@pytest.mark.parametrize("n,heads,dv", [(1 << 22, 4, 1), (1 << 24, 1, 64), (1 << 23, 1, 65),
                                        ((1 << 31) - 1, 1, 1)])
def test_step_names_its_limit(lib, n, heads, dv):
    a = L.SbcAttention(n, 1, heads, 1, dv, 0, 1.0, A, None, None)
    h = lambda i, d: ctypes.byref(L.SbcHeads(i * A, heads * d, d))  # noqa: E731
    assert lib.sbc_linear_attention_step(ctypes.byref(a), h(2, 1), h(3, 1), h(4, dv), 5 * A, None,
                                         h(6, dv), 7 * A, None, None) == UNSUPPORTED
    assert b"ceil(dv / 64) must be below 2^24" in lib.sbc_last_error()


@pytest.mark.parametrize("n,d,interleaved", [((1 << 31) - 1, 16, 0), (1 << 29, 24, 1)])
def test_rotary_names_its_limit(lib, n, d, interleaved):
    assert n * (d + 8) > 1 << 33
    plan = L.SbcRotaryPlan(A, 1, 1, 2 * A, 1, (ctypes.c_int32 * 8)(d // 2), interleaved)
    h = lambda i: ctypes.byref(L.SbcHeads(i * A, d, d))  # noqa: E731
    assert lib.sbc_rotary(ctypes.byref(plan), h(3), 1, None, 0, 0, n, d, 0, h(4), None,
                          None) == UNSUPPORTED
    assert b"2^31 lanes" in lib.sbc_last_error()
