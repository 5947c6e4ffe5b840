"""Softmax attention, its cache and the norms with the rotation without a GPU: size queries and
refusals of the C ABI (nothing here reaches the device), and the float64 reference against
itself."""
import ctypes

import numpy as np
import pytest

from paper_2012_01170_amd import _lib as L
from tests import softmax_ref as S

A = 1 << 26  # stand-in device addresses, never dereferenced
INVALID, WORKSPACE, UNSUPPORTED = 1, 6, 8


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(L.LIB_PATH):
        from paper_2012_01170_amd import build
        build.build()
    return L.lib()


def _heads(x):
    return None if x is None else ctypes.byref(L.SbcHeads(*x))


# ---------------------------------------------------------------- norms and rotation
N, D = 10, 32
QK = ("pos", "freqs", "qw", "kw", "q", "k", "dq", "dk", "qo", "ko", "dqw", "dkw", "ws")


def _at(case=None):
    at = {name: (i + 1) * A for i, name in enumerate(QK)}
    if case:
        at[case[0]] = None if case[1] is None else at[case[1]] + case[2]
    return at


def _plan(at, **kw):
    a = dict(stride=3, axes=3, sections=(8, 4, 4), inter=0)
    a.update(kw)
    return ctypes.byref(L.SbcRotaryPlan(at["pos"], a["stride"], 1, at["freqs"], a["axes"],
                                        (ctypes.c_int32 * 8)(*a["sections"]), a["inter"]))


def _h(at, name, heads=2, d=D):
    return _heads((at[name], heads * d, d))


def _qk_fwd(lib, at, plan={}, heads=(2, 2), dt=0, n=N, d=D, eps=1e-5):
    return lib.sbc_qk_norm_rotary_forward(_plan(at, **plan), _h(at, "q", d=d), heads[0],
                                          _h(at, "k", d=d), heads[1], at["qw"], at["kw"], dt, n, d,
                                          eps, _h(at, "qo", d=d), _h(at, "ko", d=d), None)


def _qk_bwd(lib, at, plan={}, heads=(2, 2), dt=0, n=N, d=D, eps=1e-5, wsb=1 << 20):
    return lib.sbc_qk_norm_rotary_backward(
        _plan(at, **plan), _h(at, "dq"), _h(at, "dk"), _h(at, "q"), heads[0], _h(at, "k"), heads[1],
        at["qw"], at["kw"], dt, n, d, eps, _h(at, "qo"), _h(at, "ko"), at["dqw"], at["dkw"],
        at["ws"], wsb, None)


@pytest.mark.parametrize("call", [_qk_fwd, _qk_bwd])
@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(d=0), INVALID), (dict(dt=5), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(heads=(-1, 2)), INVALID),
    (dict(heads=(70000, 2)), UNSUPPORTED), (dict(plan=dict(axes=0)), INVALID),
    (dict(plan=dict(axes=9)), INVALID), (dict(plan=dict(sections=(8, -1, 4))), INVALID),
    (dict(plan=dict(sections=(8, 8, 4))), INVALID), (dict(plan=dict(sections=(0, 0, 0))), INVALID),
    (dict(plan=dict(stride=2)), INVALID), (dict(d=257), UNSUPPORTED),
    (dict(d=256, plan=dict(sections=(1, 0, 0))), UNSUPPORTED),
])
def test_qk_norm_refusals(lib, call, kw, status):
    assert call(lib, _at(), **kw) == status and lib.sbc_last_error() != b""


@pytest.mark.parametrize("case", [
    ("pos", None), ("freqs", None), ("q", None), ("qo", None), ("ko", "q", 0), ("qo", "k", 0),
    ("qo", "q", 64), ("qo", "pos", 0), ("ko", "freqs", 4), ("qo", "qw", 0), ("ko", "kw", 8),
    ("ko", "qo", 128), ("q", "q", 2),
])
def test_qk_norm_forward_arrays(lib, case):
    assert _qk_fwd(lib, _at(case)) == INVALID


@pytest.mark.parametrize("case", [
    ("dq", None), ("k", None), ("ko", None), ("qo", "q", 0), ("qo", "dq", 0), ("ko", "dk", 0),
    ("dqw", "qw", 0), ("dkw", "k", 8), ("dqw", "dkw", 0), ("qo", "ko", 256), ("dqw", "pos", 0),
])
def test_qk_norm_backward_arrays(lib, case):
    assert _qk_bwd(lib, _at(case)) == INVALID


def test_qk_norm_workspace(lib):
    assert _qk_bwd(lib, _at(("ws", None))) == WORKSPACE and _qk_bwd(lib, _at(), wsb=8) == WORKSPACE
    f = lib.sbc_qk_norm_rotary_workspace_size
    assert f(-1, 8) == 0 and f(8, 0) == 0 and f(8, 257) == 0
    assert 0 < f(0, 8) <= f(10, 64) <= f(10 ** 6, 64) <= 2 ** 20


# ---------------------------------------------------------------- attention
SOFT = ("q", "k", "v", "o", "lse", "splits", "k_splits", "do", "dq", "dk", "dv", "ws")
HQ, HK, DK, DV, M = 4, 2, 16, 8, 12


def _soft_at(case=None):
    at = {name: (i + 1) * A for i, name in enumerate(SOFT)}
    if case:
        at[case[0]] = None if case[1] is None else at[case[1]] + case[2]
    return at


def _soft(at, **kw):
    a = dict(n=N, m=M, n_batch=2, heads=HQ, kv_heads=HK, dk=DK, dv=DV, dtype=0, scale=1.0, causal=1,
             splits=at["splits"], k_splits=at["k_splits"])
    a.update(kw)
    return ctypes.byref(L.SbcSoftmaxAttention(*a.values()))


def _soft_h(at, name):
    heads = HK if name in ("k", "v", "dk", "dv") else HQ
    d = DV if name in ("v", "o", "do", "dv") else DK
    return _heads((at[name], heads * d, d))


def _soft_fwd(lib, at, wsb=1 << 24, **kw):
    return lib.sbc_softmax_attention_forward(_soft(at, **kw), *(_soft_h(at, x) for x in "qkvo"),
                                             at["lse"], at["ws"], wsb, None)


def _soft_bwd(lib, at, wsb=1 << 24, **kw):
    h = [_soft_h(at, x) for x in ("do", "q", "k", "v", "o")]
    g = [_soft_h(at, x) for x in ("dq", "dk", "dv")]
    return lib.sbc_softmax_attention_backward(_soft(at, **kw), *h, at["lse"], *g, at["ws"], wsb, None)


@pytest.mark.parametrize("call", [_soft_fwd, _soft_bwd])
@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(m=-1), INVALID), (dict(n_batch=-1), INVALID),
    (dict(n_batch=0), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID),
    (dict(kv_heads=3), INVALID), (dict(dk=0), INVALID), (dict(dv=0), INVALID),
    (dict(dtype=9), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=3e38), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(dk=129), UNSUPPORTED), (dict(dv=129), UNSUPPORTED), (dict(splits=None), INVALID),
    (dict(k_splits=None), INVALID), (dict(heads=65536), UNSUPPORTED),
    (dict(n=1 << 30), UNSUPPORTED), (dict(m=1 << 30), UNSUPPORTED),
    (dict(heads=1, kv_heads=1, n=2 ** 31 - 1000), UNSUPPORTED),
    (dict(heads=1, kv_heads=1, m=2 ** 31 - 1), UNSUPPORTED), (dict(wsb=8, n=4000, m=4000), WORKSPACE),
])
def test_attention_refusals(lib, call, kw, status):
    assert call(lib, _soft_at(), **kw) == status and lib.sbc_last_error() != b""


@pytest.mark.parametrize("case", [
    ("q", None), ("k", None), ("v", None), ("o", None), ("o", "q", 0), ("o", "k", 64),
    ("o", "v", 0), ("o", "lse", 0), ("lse", "q", 0), ("lse", "splits", 0), ("o", "k_splits", 4),
    ("q", "q", 2), ("lse", "v", 16),
])
def test_attention_forward_arrays(lib, case):
    assert _soft_fwd(lib, _soft_at(case)) == INVALID


@pytest.mark.parametrize("case", [
    ("do", None), ("o", None), ("lse", None), ("dq", None), ("dk", None), ("dv", None),
    ("dq", "q", 0), ("dk", "k", 0), ("dv", "v", 4), ("dq", "do", 0), ("dk", "o", 0),
    ("dv", "lse", 0), ("dk", "dq", 0), ("dv", "dk", 32), ("dq", "splits", 0), ("dk", "k_splits", 0),
])
def test_attention_backward_arrays(lib, case):
    assert _soft_bwd(lib, _soft_at(case)) == INVALID


def test_attention_workspaces(lib):
    at = _soft_at()
    for f in (lib.sbc_softmax_attention_workspace_size,
              lib.sbc_softmax_attention_backward_workspace_size):
        assert f(None) == 0 and f(_soft(at, dk=129)) == 0
        for n in (1, 1000, 100_000):  # no scores are kept
            size = f(_soft(at, n=n, m=n, heads=8, kv_heads=8, dk=64, dv=64))
            assert 0 <= size <= (1 << 25) + 40 * n * 8 * 128 * 4
    f = lib.sbc_softmax_attention_paged_workspace_size
    assert f(_soft(at), 0, 4) == 0 and f(_soft(at), 16, -1) == 0
    assert 0 == f(_soft(at, n=1, n_batch=1), 16, 0) < f(_soft(at, n=1, n_batch=1), 16, 10_000)
    assert f(_soft(at, n=1, n_batch=1), 1 << 30, 1 << 30) > 0


# ---------------------------------------------------------------- a cache in pages
CACHE = ("q", "k", "v", "o", "lse", "splits", "table", "lengths", "ws")
N_PAGES, PAGE, WIDTH = 6, 4, 3


def _pages(at, name, d, stride=None):
    if at[name] is None:
        return None
    s = (PAGE * HK * d, HK * d, d) if stride is None else stride
    return ctypes.byref(L.SbcPages(at[name], *s))


def _paged(lib, at, n_pages=N_PAGES, page=PAGE, width=WIDTH, wsb=1 << 24, k_stride=None, **kw):
    h = lambda x, d: _heads((at[x], HQ * d, d))  # noqa: E731
    a = dict(dict(m=0, k_splits=None), **kw)
    return lib.sbc_softmax_attention_paged(
        _soft(at, **a), h("q", DK), _pages(at, "k", DK, k_stride), _pages(at, "v", DV), n_pages,
        page, at["table"], width, at["lengths"], h("o", DV), at["lse"], at["ws"], wsb, None)


def _cache_at(case=None):
    at = {name: (i + 1) * A for i, name in enumerate(CACHE)}
    at["k_splits"] = None
    if case:
        at[case[0]] = None if case[1] is None else at[case[1]] + case[2]
    return at


@pytest.mark.parametrize("kw,status", [
    (dict(n_pages=-1), INVALID), (dict(page=0), INVALID), (dict(width=-1), INVALID),
    (dict(splits=None), INVALID), (dict(n_batch=0), INVALID), (dict(scale=0.0), INVALID),
    (dict(k_stride=(-1, 32, 16)), INVALID), (dict(dk=200), UNSUPPORTED),
    (dict(wsb=8, width=1000), WORKSPACE),
    (dict(n=0), 0),
])
def test_paged_refusals(lib, kw, status):
    assert _paged(lib, _cache_at(), **kw) == status


@pytest.mark.parametrize("case", [
    ("q", None), ("k", None), ("v", None), ("o", None), ("table", None), ("lengths", None),
    ("o", "k", 0), ("o", "v", 512), ("o", "table", 0), ("lse", "lengths", 0), ("o", "q", 0),
    ("lse", "splits", 8),
])
def test_paged_arrays(lib, case):
    assert _paged(lib, _cache_at(case)) == INVALID


@pytest.mark.parametrize("m", [-7, 2 ** 31 - 1])
def test_paged_reads_no_fields_of_packed_keys(lib, m):
    """m, causal and k_splits may hold anything, in the call and in its size query."""
    at = _cache_at()
    odd = dict(m=m, causal=m, k_splits=at["q"] + 1)
    assert _paged(lib, at, n=0, **odd) == 0
    assert _paged(lib, at, wsb=8, width=1000, **odd) == WORKSPACE  # past the checks
    f = lib.sbc_softmax_attention_paged_workspace_size
    size = f(_soft(at, n=1, n_batch=1, m=0, causal=0, k_splits=None), 16, 10_000)
    assert size > 0 and f(_soft(at, n=1, n_batch=1, **odd), 16, 10_000) == size


SLOTS = ("lengths", "splits", "table", "free", "out", "slots", "after", "needed", "ws")


def _slots(lib, case=None, n=9, n_batch=5, width=WIDTH, page=PAGE, n_free=4, wsb=1 << 20):
    at = {name: (i + 1) * A for i, name in enumerate(SLOTS)}
    if case:
        at[case[0]] = None if case[1] is None else at[case[1]] + case[2]
    return lib.sbc_cache_slots(at["lengths"], at["splits"], n, n_batch, at["table"], width, page,
                               at["free"], n_free, at["out"], at["slots"], at["after"],
                               at["needed"], at["ws"], wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(n_batch=-1), INVALID), (dict(width=-1), INVALID),
    (dict(page=0), INVALID), (dict(n_free=-1), INVALID), (dict(case=("splits", None)), INVALID),
    (dict(width=1 << 30), UNSUPPORTED), (dict(n_batch=5000, case=("ws", None)), WORKSPACE),
    (dict(n_batch=5000, wsb=256), WORKSPACE),
])
def test_cache_slots_refusals(lib, kw, status):
    assert _slots(lib, **kw) == status


@pytest.mark.parametrize("case", [
    ("lengths", None), ("table", None), ("free", None), ("out", None), ("slots", None),
    ("after", None), ("needed", None), ("out", "table", 4), ("out", "free", 0), ("out", "lengths", 0),
    ("after", "lengths", 0), ("slots", "table", 8), ("needed", "after", 0), ("needed", "free", 4),
    ("slots", "splits", 0), ("after", "out", 8),
])
def test_cache_slots_arrays(lib, case):
    assert _slots(lib, case) == INVALID


def _append(lib, n=9, heads=HK, dk=DK, dv=DV, dt=0, page=PAGE, n_pages=N_PAGES, k_stride=None,
            case=None):
    at = {name: (i + 1) * A for i, name in enumerate(("k", "v", "slots", "kp", "vp"))}
    if case:
        at[case[0]] = None if case[1] is None else at[case[1]] + case[2]
    h = lambda x, d: None if at[x] is None else _heads((at[x], HK * d, d))  # noqa: E731
    return lib.sbc_cache_append(h("k", DK), h("v", DV), n, heads, dk, dv, dt, at["slots"],
                                _pages(at, "kp", DK, k_stride), _pages(at, "vp", DV), n_pages, page,
                                None)


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(heads=0), INVALID), (dict(dk=0), INVALID), (dict(dv=-2), INVALID),
    (dict(dt=3), INVALID), (dict(page=0), INVALID), (dict(n_pages=-1), INVALID),
    (dict(k_stride=(0, 32, 16)), INVALID), (dict(k_stride=(128, 16, 16)), INVALID),
    (dict(k_stride=(128, 32, 8)), INVALID), (dict(case=("k", None)), INVALID),
    (dict(case=("vp", None)), INVALID), (dict(case=("slots", None)), INVALID),
    (dict(case=("kp", "k", 0)), INVALID), (dict(case=("vp", "slots", 0)), INVALID),
    (dict(case=("vp", "kp", 64)), INVALID), (dict(n=0), 0),
    (dict(n_pages=0), 0),
])
def test_cache_append_refusals(lib, kw, status):
    assert _append(lib, **kw) == status


def test_cache_append_layouts(lib):
    """Heads first, and keys beside values in each page, are layouts without overlaps."""
    stride = (PAGE * HK * DK, DK, PAGE * DK)
    assert _append(lib, n_pages=0, k_stride=stride) == 0
    at = {"kp": A, "vp": A + 4 * PAGE * HK * DK}
    both = PAGE * HK * (DK + DV)
    k = ctypes.byref(L.SbcPages(at["kp"], both, HK * DK, DK))
    v = ctypes.byref(L.SbcPages(at["vp"], both, HK * DV, DV))
    rows = lambda x, d: _heads((x, HK * d, d))  # noqa: E731
    call = lambda v: lib.sbc_cache_append(rows(4 * A, DK), rows(5 * A, DV), 1 << 29, HK, DK, DV, 0,  # noqa: E731
                                          6 * A, k, v, N_PAGES, PAGE, None)
    assert call(v) == UNSUPPORTED  # past the overlaps, at the number of rows
    assert call(ctypes.byref(L.SbcPages(at["vp"] - 4, both, HK * DV, DV))) == INVALID


def _elements(base, strides, dims, d):
    """Of a cache: the places of all its elements"""
    at = np.full(1, base)
    for n, s in (*zip(dims, strides), (d, 1)):
        at = (at[:, None] + s * np.arange(n)).ravel()
    return at


def _append_places(lib, k, v, dims, dk, dv, dt):
    """The status of caches at elements and strides k and v, past their checks of overlaps
    UNSUPPORTED, by the number of rows"""
    e = 4 if dt == 0 else 2
    n_pages, page, heads = dims
    pages = [ctypes.byref(L.SbcPages(A + e * at, *strides)) for at, strides in (k, v)]
    rows = lambda x, d: _heads((x, heads * d, d))  # noqa: E731
    return lib.sbc_cache_append(rows(8 * A, dk), rows(9 * A, dv), 2 ** 31 - 1, heads, dk, dv, dt,
                                10 * A, *pages, n_pages, page, None)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("dims", [(5, 4, 3), (1, 4, 3), (5, 1, 3), (5, 4, 1), (1, 1, 2), (2, 1, 1)])
@pytest.mark.parametrize("dk,dv", [(16, 16), (16, 8), (9, 7)])
def test_cache_append_one_pool(lib, dims, dk, dv, dt):
    """Keys and values beside each other in a page, a token, a head's channels, heads before or
    behind tokens: taken; one element into each other: refused."""
    pages, page, G = dims
    both = G * (dk + dv)
    layouts = [
        ((0, (page * both, G * dk, dk)), (page * G * dk, (page * both, G * dv, dv))),  # of a page
        ((0, (page * both, both, dk)), (G * dk, (page * both, both, dv))),             # of a token
        ((0, (page * both, both, dk + dv)), (dk, (page * both, both, dk + dv))),       # of a head
        ((0, (page * both, dk, page * dk)),
         (page * G * dk, (page * both, dv, page * dv))),                               # heads first
        ((0, (page * both, dk + dv, page * (dk + dv))),
         (dk, (page * both, dk + dv, page * (dk + dv)))),                              # and of a head
        ((0, (page * G * dk, G * dk, dk)),
         (pages * page * G * dk, (page * G * dv, G * dv, dv))),                        # apart
        ((0, (both, pages * both, dk)), (G * dk, (both, pages * both, dv))),           # pages inside
    ]
    for k, v in layouts:
        assert _append_places(lib, k, v, dims, dk, dv, dt) == UNSUPPORTED, (k, v)
        assert _append_places(lib, v, k, dims, dv, dk, dt) == UNSUPPORTED, (k, v)
        assert _append_places(lib, k, (v[0] - 1, v[1]), dims, dk, dv, dt) == INVALID, (k, v)


def test_cache_append_overlaps_are_found(lib):
    """No two caches of any strides are taken that share an element."""
    rng = np.random.default_rng(5)
    kinds = {True: set(), False: set()}
    for _ in range(4000):
        dims, dk, dv = rng.integers(1, 4, 3), int(rng.integers(1, 7)), int(rng.integers(1, 7))
        two = []
        for d in (dk, dv):
            order, step, strides = rng.permutation(3), d + int(rng.integers(0, 7)), [0, 0, 0]
            for axis in order:
                strides[axis] = step
                step = step * (dims[axis] + int(rng.integers(0, 2))) + int(rng.integers(0, 2)) * 3
            two.append(strides)
        if rng.random() < 0.7:
            two[1] = list(two[0])
        off = int(rng.integers(0, 60))
        places = [_elements(at, st, dims, d) for at, st, d in ((0, two[0], dk), (off, two[1], dv))]
        if any(len(np.unique(x)) < len(x) for x in places):
            continue  # (refused by itself)
        share = len(np.intersect1d(*places)) > 0
        status = _append_places(lib, (0, two[0]), (off, two[1]), tuple(int(x) for x in dims), dk, dv, 0)
        kinds[share].add(status)
    assert kinds[True] == {INVALID} and UNSUPPORTED in kinds[False]


# ---------------------------------------------------------------- the reference
def _numeric(f, x, d, eps=1e-5):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


@pytest.mark.parametrize("causal", [False, True])
def test_reference_gradients_against_differences(causal):
    rng = np.random.default_rng(3)
    sq, sk, scale = [0, 7, 7, 15], [0, 4, 6, 20], 0.6
    q, do = rng.standard_normal((15, 4, 5)), rng.standard_normal((15, 4, 3))
    k, v = rng.standard_normal((20, 2, 5)), rng.standard_normal((20, 2, 3))
    f = lambda q, k, v: S.attention(q, k, v, sq, sk, scale, causal)  # noqa: E731
    o, lse, *_ = f(q, k, v)
    assert (lse[:3] == -np.inf).all() == causal and (o[:3] == 0).all() == causal
    grads, _ = S.attention_grad(do, q, k, v, o, lse, sq, sk, scale, causal)
    for i, g in enumerate(grads):
        for _ in range(3):
            d = rng.standard_normal(g.shape)

            def at(z):
                a = [q, k, v]
                a[i] = z
                return (f(*a)[0] * do).sum()
            assert abs(_numeric(at, (q, k, v)[i], d) - (g * d).sum()) < 1e-6 * (1 + abs(g * d).sum())


def test_reference_norm_gradients_against_differences():
    rng = np.random.default_rng(4)
    x, dy, w = rng.standard_normal((6, 2, 9)), rng.standard_normal((6, 2, 9)), rng.standard_normal(9)
    args = (rng.standard_normal((6, 2)), rng.standard_normal(4), (3, 1), True, 1e-5)
    dx, dw, *_ = S.qk_norm_grad(dy, x, w, *args)
    f = lambda x, w: (S.qk_norm(x, w, *args)[0] * dy).sum()  # noqa: E731
    d = rng.standard_normal(x.shape)
    assert abs(_numeric(lambda z: f(z, w), x, d) - (dx * d).sum()) < 1e-6 * (1 + abs(dx * d).sum())
    d = rng.standard_normal(9)
    assert abs(_numeric(lambda z: f(x, z), w, d) - (dw * d).sum()) < 1e-6 * (1 + abs(dw * d).sum())


def test_reference_places():
    table, slots, lengths, needed = S.cache_slots(np.array([3, 0, 4]), np.array([[5, -1], [-1, -1],
                                                  [6, -1]]), [9, 2], 4, np.array([0, 2, 4, 5]))
    assert table.tolist() == [[5, 9], [2, -1], [6, -1]] and needed == 3
    assert slots.tolist() == [23, 36, 8, 9, -1] and lengths.tolist() == [5, 2, 5]
