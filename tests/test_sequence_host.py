"""The sequence operators without a GPU: size queries and refusals of the C ABI (nothing
here reaches the device), and the float64 reference's gradients against differences."""
import ctypes

import numpy as np
import pytest

from paper_2012_01170_amd import _lib as L
from tests import sequence_ref as R

A = 1 << 20  # stand-in device addresses, never dereferenced


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(L.LIB_PATH):
        from paper_2012_01170_amd import build
        build.build()
    return L.lib()


# ---------------------------------------------------------------- layer norm
def _norm_fwd(lib, **kw):
    a = dict(x=A, xs=64, w=None, b=None, dt=0, n=10, C=64, eps=1e-5, y=2 * A, ys=64)
    a.update(kw)
    return lib.sbc_layer_norm_forward(a["x"], a["xs"], a["w"], a["b"], a["dt"], a["n"], a["C"],
                                      a["eps"], a["y"], a["ys"], None, None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 1), (dict(C=0), 1), (dict(C=(1 << 24) + 1, xs=1 << 25, ys=1 << 25), 8),
    (dict(dt=7), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(xs=63), 1),
    (dict(ys=63), 1), (dict(x=None), 1), (dict(y=None), 1), (dict(y=A), 1),
    (dict(y=A + 9 * 64 * 4), 1), (dict(n=0, x=None, y=None), 0),
])
def test_norm_forward_refusals(lib, kw, status):
    assert _norm_fwd(lib, **kw) == status
    assert (lib.sbc_last_error() != b"") == (status != 0)


def _norm_bwd(lib, **kw):
    a = dict(dy=A, dys=64, x=2 * A, xs=64, w=None, m=3 * A, r=3 * A, dt=0, n=10, C=64, dx=4 * A,
             dxs=64, dw=5 * A, db=6 * A, ws=7 * A, wsb=1 << 30)
    a.update(kw)
    return lib.sbc_layer_norm_backward(a["dy"], a["dys"], a["x"], a["xs"], a["w"], a["m"], a["r"],
                                       a["dt"], a["n"], a["C"], a["dx"], a["dxs"], a["dw"],
                                       a["db"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 1), (dict(C=0), 1), (dict(dt=2), 1), (dict(dys=1), 1), (dict(xs=1), 1),
    (dict(dxs=1), 1), (dict(dy=None), 1), (dict(x=None), 1), (dict(m=None), 1), (dict(r=None), 1),
    (dict(dx=A), 1), (dict(dx=2 * A), 1), (dict(ws=None), 6), (dict(wsb=8), 6),
    (dict(dx=None, dw=None, db=None), 0),
])
def test_norm_backward_refusals(lib, kw, status):
    assert _norm_bwd(lib, **kw) == status


def test_norm_workspace(lib):
    assert lib.sbc_layer_norm_workspace_size(-1, 8) == 0
    assert lib.sbc_layer_norm_workspace_size(8, 0) == 0
    small, large = (lib.sbc_layer_norm_workspace_size(n, 64) for n in (1, 1_000_000))
    assert 0 < small < large and small >= 2 * 64 * 4
    # a tenth of the rows in bf16 at most
    assert large <= 0.1 * 3 * 1_000_000 * 64 * 2


# ---------------------------------------------------------------- rotary
def _rotary(lib, plan=(), q=(), k=(), **kw):
    p = dict(positions=A, position_stride=3, float_positions=1, freqs=A, n_axes=3,
             sections=(8, 4, 4), interleaved=0)
    p.update(plan)
    a = dict(qh=2, kh=2, dt=0, n=5, d=32, qo=(4 * A, 64, 32), ko=(5 * A, 64, 32))
    a.update(kw)
    q = dict(dict(data=2 * A, token_stride=64, head_stride=32), **dict(q))
    k = dict(dict(data=3 * A, token_stride=64, head_stride=32), **dict(k))
    pl = L.SbcRotaryPlan(p["positions"], p["position_stride"], p["float_positions"], p["freqs"],
                         p["n_axes"], (ctypes.c_int32 * 8)(*p["sections"]), p["interleaved"])
    h = lambda d: ctypes.byref(L.SbcHeads(*d)) if d else None  # noqa: E731
    return lib.sbc_rotary(ctypes.byref(pl), h(tuple(q.values())), a["qh"], h(tuple(k.values())),
                          a["kh"], a["dt"], a["n"], a["d"], 0, h(a["qo"]), h(a["ko"]), None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), 1), (dict(d=0), 1), (dict(dt=3), 1), (dict(plan=dict(n_axes=0)), 1),
    (dict(plan=dict(n_axes=9)), 1), (dict(plan=dict(sections=(8, -1, 4))), 1),
    (dict(plan=dict(sections=(8, 8, 4))), 1), (dict(plan=dict(sections=(0, 0, 0))), 1),
    (dict(plan=dict(position_stride=2)), 1), (dict(plan=dict(positions=None)), 1),
    (dict(plan=dict(freqs=None)), 1), (dict(qh=-1), 1), (dict(q=dict(data=None)), 1),
    (dict(q=dict(token_stride=-1)), 1), (dict(q=dict(data=2 * A + 2)), 1), (dict(qo=None), 1),
    (dict(qo=(4 * A, 32, 32)), 1),          # two tokens' heads in one place
    (dict(qo=(4 * A, 64, 16)), 1),          # two heads
    (dict(qo=(3 * A, 64, 32)), 1),          # q_out on k
    (dict(qo=(4 * A, 64, 32), ko=(4 * A + 64, 64, 32)), 1),
    (dict(qo=(2 * A + 64, 64, 32)), 1),     # on q, but not q itself
    (dict(n=0, q=dict(data=None)), 0), (dict(qh=0, kh=0), 0),
])
def test_rotary_refusals(lib, kw, status):
    assert _rotary(lib, **kw) == status


# ---------------------------------------------------------------- attention
def _heads(data, d, heads=2):
    return ctypes.byref(L.SbcHeads(data, heads * d, d))


def _attn(**kw):
    a = dict(n=10, n_batch=2, heads=2, dk=32, dv=16, dtype=0, scale=1.0, rates=A, splits=A, t=A)
    a.update(kw)
    return L.SbcAttention(*a.values())


def _fwd(lib, a, state_in=None, state_time=None, o=5 * A, state_out=None, time_out=None,
         q=2 * A, wsb=1 << 30, ws=9 * A):
    return lib.sbc_linear_attention_forward(
        ctypes.byref(a), _heads(q, a.dk), _heads(3 * A, a.dk), _heads(4 * A, a.dv), state_in,
        state_time, _heads(o, a.dv), state_out, time_out, ws, wsb, None)


@pytest.mark.parametrize("kw,call,status", [
    (dict(n=-1), {}, 1), (dict(n_batch=-1), {}, 1), (dict(n_batch=0), {}, 1),
    (dict(heads=0), {}, 1), (dict(dk=0), {}, 1), (dict(dv=0), {}, 1), (dict(dtype=4), {}, 1),
    (dict(dk=129), {}, 8), (dict(dv=129), {}, 8), (dict(rates=None), {}, 1),
    (dict(splits=None), {}, 1), (dict(), dict(q=None), 1), (dict(), dict(o=2 * A), 1),
    (dict(), dict(state_in=6 * A), 1),                       # no time
    (dict(), dict(state_out=6 * A), 1),                      # no time_out
    (dict(t=None), dict(state_in=6 * A, state_out=6 * A), 1),
    (dict(), dict(state_in=6 * A, state_time=7 * A, state_out=8 * A, time_out=7 * A), 1),
    (dict(), dict(ws=None), 6), (dict(), dict(wsb=16), 6), (dict(n=0), dict(q=None), 0),
])
def test_attention_forward_refusals(lib, kw, call, status):
    assert _fwd(lib, _attn(**kw), **call) == status


def _bwd(lib, a, do=A * 2, dq=6 * A, dk=7 * A, dv=8 * A, wsb=1 << 30, ws=9 * A):
    return lib.sbc_linear_attention_backward(
        ctypes.byref(a), _heads(do, a.dv), _heads(3 * A, a.dk), _heads(4 * A, a.dk),
        _heads(5 * A, a.dv), _heads(dq, a.dk), _heads(dk, a.dk), _heads(dv, a.dv), None, ws, wsb,
        None)


@pytest.mark.parametrize("kw,call,status", [
    (dict(dk=200), {}, 8), (dict(rates=None), {}, 1), (dict(), dict(do=None), 1),
    (dict(), dict(dq=None), 1), (dict(), dict(dq=3 * A), 1), (dict(), dict(dk=5 * A), 1),
    (dict(), dict(dv=7 * A), 1), (dict(), dict(ws=None), 6), (dict(), dict(wsb=0), 6),
    (dict(n=0), dict(do=None), 0),
])
def test_attention_backward_refusals(lib, kw, call, status):
    assert _bwd(lib, _attn(**kw), **call) == status


def _step(lib, a, state_in=6 * A, state_time=7 * A, state_out=8 * A, time_out=9 * A, o=5 * A):
    return lib.sbc_linear_attention_step(
        ctypes.byref(a), _heads(2 * A, a.dk), _heads(3 * A, a.dk), _heads(4 * A, a.dv), state_in,
        state_time, _heads(o, a.dv), state_out, time_out, None)


@pytest.mark.parametrize("kw,call,status", [
    (dict(dv=0), {}, 1), (dict(rates=None), {}, 1), (dict(), dict(state_in=None), 1),
    (dict(), dict(state_out=None), 1), (dict(), dict(state_time=None), 1),
    (dict(), dict(time_out=None), 1), (dict(), dict(time_out=7 * A), 1),
    (dict(), dict(state_out=6 * A + 16), 1), (dict(), dict(o=4 * A), 1), (dict(n=0), {}, 0),
])
def test_attention_step_refusals(lib, kw, call, status):
    assert _step(lib, _attn(**kw), **call) == status


def test_attention_workspaces(lib):
    f, b = lib.sbc_linear_attention_workspace_size, lib.sbc_linear_attention_backward_workspace_size
    for w in (f, b):
        assert w(-1, 1, 8, 8) == 0 and w(8, 0, 8, 8) == 0 and w(8, 1, 129, 8) == 0
        assert 0 < w(0, 1, 8, 8) <= w(100_000, 4, 64, 64) <= w(100_000, 4, 128, 128)


# ---------------------------------------------------------------- the reference's gradients
def _numeric(f, x, d, eps=1e-5):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


@pytest.mark.parametrize("times", [False, True])
def test_reference_gradients_against_differences(times):
    rng = np.random.default_rng(3)
    n, H, dk, dv, splits, scale = 23, 2, 5, 4, [0, 9, 9, 10, 23], 0.7
    q, k, v, do = (rng.standard_normal((n, H, d)) for d in (dk, dk, dv, dv))
    t = np.sort(rng.integers(0, 60, n)) if times else None
    rates = np.array([0.3, 0.02])
    f = lambda q, k, v, r: (R.attention(q, k, v, r, splits, t, scale)[0] * do).sum()  # noqa: E731
    got = R.attention_grad(do, q, k, v, rates, splits, t, scale)[0]
    for i, (name, x) in enumerate((("q", q), ("k", k), ("v", v), ("rates", rates))):
        args = [q, k, v, rates]
        for _ in range(3):
            d = rng.standard_normal(x.shape)

            def at(z):
                a = list(args)
                a[i] = z
                return f(*a)
            assert abs(_numeric(at, x, d) - (got[i] * d).sum()) < 1e-6 * (1 + abs((got[i] * d)).sum()), name


def test_reference_norm_gradients_against_differences():
    rng = np.random.default_rng(4)
    x, w, b, dy = (rng.standard_normal(s) for s in ((6, 9), 9, 9, (6, 9)))
    f = lambda x, w, b: (R.layer_norm(x, w, b, 1e-5)[0] * dy).sum()  # noqa: E731
    _, mean, rstd = R.layer_norm(x, w, b, 1e-5)
    got = R.layer_norm_grad(dy, x, w, mean, rstd)
    for i, a in enumerate((x, w, b)):
        d = rng.standard_normal(a.shape)

        def at(z):
            args = [x, w, b]
            args[i] = z
            return f(*args)
        assert abs(_numeric(at, a, d) - (got[i] * d).sum()) < 1e-6 * (1 + abs(got[i] * d).sum())


def test_reference_recursion_is_the_sum():
    """The state carried from one half of the sequences to the other."""
    rng = np.random.default_rng(5)
    n, H, dk, dv = 20, 2, 4, 3
    q, k, v = (rng.standard_normal((n, H, d)) for d in (dk, dk, dv))
    t = np.sort(rng.integers(0, 50, n))
    rates = np.array([0.1, 0.01])
    whole = R.attention(q, k, v, rates, [0, n], t, 0.5)
    o1, S, T, _ = R.attention(q[:8], k[:8], v[:8], rates, [0, 8], t[:8], 0.5)
    o2, S, T, _ = R.attention(q[8:], k[8:], v[8:], rates, [0, n - 8], t[8:], 0.5, S, T)
    assert np.allclose(np.concatenate([o1, o2]), whole[0], rtol=1e-12, atol=1e-12)
    assert np.allclose(S, whole[1], rtol=1e-12, atol=1e-12) and T[0] == t[-1]
