"""The C ABI of the sequence operators refuses outputs that lie on other arguments (nothing
here reaches the device)."""
import ctypes

import pytest

from paper_2012_01170_amd import _lib as L

A = 1 << 24  # stand-in device addresses, never dereferenced
INVALID = 1


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(L.LIB_PATH):
        from paper_2012_01170_amd import build
        build.build()
    return L.lib()


# names of the calls' arrays -> their addresses; a case puts one on (or into) another
def _put(names, case):
    at = {name: (i + 1) * A for i, name in enumerate(names)}
    name, (other, offset) = case
    at[name] = at[other] + offset
    return at


N, C = 10, 64
NORM_FWD = ("x", "w", "b", "y", "mean", "rstd")


@pytest.mark.parametrize("case", [
    ("y", ("w", 0)), ("y", ("b", 4)), ("mean", ("x", 64)), ("mean", ("w", 0)), ("rstd", ("b", 8)),
    ("rstd", ("mean", 4)), ("mean", ("y", 100)), ("y", ("x", 0)), ("rstd", ("x", (N * C - 1) * 4)),
])
def test_norm_forward(lib, case):
    at = _put(NORM_FWD, case)
    assert lib.sbc_layer_norm_forward(at["x"], C, at["w"], at["b"], 0, N, C, 1e-5, at["y"], C,
                                      at["mean"], at["rstd"], None) == INVALID


NORM_BWD = ("dy", "x", "w", "mean", "rstd", "dx", "dw", "db", "ws")


@pytest.mark.parametrize("case", [
    ("dx", ("w", 0)), ("dx", ("mean", 8)), ("dx", ("rstd", 0)), ("dw", ("w", 0)), ("dw", ("x", 4)),
    ("db", ("dy", 0)), ("db", ("mean", 0)), ("db", ("dw", 8)), ("dw", ("dx", 0)),
])
def test_norm_backward(lib, case):
    at = _put(NORM_BWD, case)
    assert lib.sbc_layer_norm_backward(at["dy"], C, at["x"], C, at["w"], at["mean"], at["rstd"], 0,
                                       N, C, at["dx"], C, at["dw"], at["db"], at["ws"], 1 << 20,
                                       None) == INVALID


@pytest.mark.parametrize("case", [
    ("qo", ("pos", 0)), ("ko", ("pos", 8)), ("qo", ("freqs", 0)), ("ko", ("freqs", 4)),
    ("qo", ("k", 0)), ("ko", ("qo", 256)),
])
def test_rotary(lib, case):
    at = _put(("pos", "freqs", "q", "k", "qo", "ko"), case)
    plan = L.SbcRotaryPlan(at["pos"], 3, 1, at["freqs"], 3, (ctypes.c_int32 * 8)(8, 4, 4), 0)
    h = lambda n: ctypes.byref(L.SbcHeads(at[n], 64, 32))  # noqa: E731
    assert lib.sbc_rotary(ctypes.byref(plan), h("q"), 2, h("k"), 2, 0, N, 32, 0, h("qo"), h("ko"),
                          None) == INVALID


DK, DV, H, B = 32, 16, 2, 3
ATTN = ("q", "k", "v", "rates", "splits", "t", "s_in", "t_in", "o", "s_out", "t_out", "ws")


def _attention(at):
    return L.SbcAttention(N, B, H, DK, DV, 0, 1.0, at["rates"], at.get("splits"), at["t"])


def _heads(at, name):
    d = DV if name in ("v", "o", "do", "dv") else DK
    return ctypes.byref(L.SbcHeads(at[name], H * d, d))


@pytest.mark.parametrize("case", [
    ("o", ("s_in", 0)), ("o", ("rates", 0)), ("o", ("splits", 4)), ("o", ("t", 0)),
    ("o", ("t_in", 0)), ("o", ("s_out", 64)), ("s_out", ("q", 0)), ("s_out", ("k", 128)),
    ("s_out", ("v", 0)), ("s_out", ("rates", 0)), ("s_out", ("t", 0)), ("s_out", ("s_in", 4)),
    ("t_out", ("t", 8)), ("t_out", ("splits", 0)), ("t_out", ("t_in", 0)), ("t_out", ("q", 0)),
    ("t_out", ("s_out", 0)), ("t_out", ("s_in", 0)), ("o", ("q", 0)),
])
def test_attention_forward(lib, case):
    at = _put(ATTN, case)
    assert lib.sbc_linear_attention_forward(
        ctypes.byref(_attention(at)), _heads(at, "q"), _heads(at, "k"), _heads(at, "v"), at["s_in"],
        at["t_in"], _heads(at, "o"), at["s_out"], at["t_out"], at["ws"], 1 << 22, None) == INVALID


@pytest.mark.parametrize("case", [
    ("o", ("s_in", 0)), ("o", ("rates", 0)), ("o", ("t", 0)), ("o", ("t_in", 0)),
    ("o", ("s_out", 64)), ("s_out", ("q", 0)), ("s_out", ("v", 128)), ("s_out", ("rates", 0)),
    ("s_out", ("t", 0)), ("s_out", ("s_in", 4)), ("t_out", ("t", 8)), ("t_out", ("t_in", 0)),
    ("t_out", ("q", 0)), ("t_out", ("s_out", 0)), ("t_out", ("s_in", 0)), ("o", ("k", 0)),
])
def test_attention_step(lib, case):
    at = _put(ATTN, case)
    assert lib.sbc_linear_attention_step(
        ctypes.byref(_attention(at)), _heads(at, "q"), _heads(at, "k"), _heads(at, "v"), at["s_in"],
        at["t_in"], _heads(at, "o"), at["s_out"], at["t_out"], None) == INVALID


@pytest.mark.parametrize("case", [
    ("dq", ("rates", 0)), ("dk", ("splits", 0)), ("dv", ("t", 4)), ("drates", ("rates", 0)),
    ("drates", ("q", 8)), ("drates", ("do", 0)), ("drates", ("dk", 0)), ("drates", ("t", 0)),
    ("dq", ("k", 0)), ("dv", ("dq", 0)),
])
def test_attention_backward(lib, case):
    at = _put(("do", "q", "k", "v", "rates", "splits", "t", "dq", "dk", "dv", "drates", "ws"), case)
    assert lib.sbc_linear_attention_backward(
        ctypes.byref(_attention(at)), *(_heads(at, n) for n in ("do", "q", "k", "v", "dq", "dk", "dv")),
        at["drates"], at["ws"], 1 << 22, None) == INVALID


# Rows of one array: outputs in them beside what they are made from are no overlap, so that
# the next check speaks (no workspace, 6).
def test_rows_that_share_memory(lib):
    e = 4
    at = {n: (i + 1) * A for i, n in enumerate(ATTN)}
    row = 2 * H * DK + 2 * H * DV + H * DK * DV  # q, k, v, o and, past them, a stream's state
    h = lambda off, d: ctypes.byref(L.SbcHeads(A + off * e, row, d))  # noqa: E731
    at["ws"] = None
    tokens = lambda o: (h(0, DK), h(H * DK, DK), h(2 * H * DK, DV), at["s_in"], at["t_in"],  # noqa: E731
                        h(o, DV), at["s_out"], at["t_out"], None, 0, None)
    a = _attention({**at, "rates": 50 * A})
    good = 2 * H * DK + H * DV
    assert lib.sbc_linear_attention_forward(ctypes.byref(a), *tokens(good)) == 6
    assert lib.sbc_linear_attention_forward(ctypes.byref(a), *tokens(good - 1)) == INVALID
    # a state between two tokens' rows, and one that reaches into the second
    a2 = L.SbcAttention(2, 1, H, DK, DV, 0, 1.0, 50 * A, None, None)
    for at_, want in ((good + H * DV, 6), (good + H * DV + 1, INVALID), (good + H * DV - 1, INVALID)):
        assert lib.sbc_linear_attention_forward(
            ctypes.byref(a2), h(0, DK), h(H * DK, DK), h(2 * H * DK, DV), None, None, h(good, DV),
            A + at_ * e, None, None, 0, None) == want
    # heads before tokens: q, k, v and o of a head beside each other
    def hm(i, d):
        return ctypes.byref(L.SbcHeads(A + i * N * DK * e, d, 4 * N * DK))
    assert lib.sbc_linear_attention_forward(
        ctypes.byref(a), hm(0, DK), hm(1, DK), hm(2, DV), None, None, hm(3, DV), None, None, None, 0,
        None) == 6
