"""Softmax attention on the GPU against plain float64 (tests/softmax_ref.py), whose functions
derive the tolerances; outputs of bf16 are rounded once more, by half a unit of 2^-8."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2012_01170_amd as sbc
from paper_2012_01170_amd import _lib as L
from tests import softmax_ref as S

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}  # half a unit


def _rand(rng, shape, dtype=F32, size=1.0):
    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * np.float32(size))
    return x.to(DEV).to(dtype)


def _np(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _close(got, ref, tol, what):
    got = _np(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    same = got == ref  # (infinities)
    bad = np.where(same, 0.0, np.abs(np.where(same, 0, got) - np.where(same, 0, ref)) - tol)
    assert not np.isnan(bad).any(), f"{what}: NaN"
    assert bad.max(initial=0.0) <= 0, f"{what}: {bad.max()} over"


def _splits(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def _inputs(rng, n, m, hq, hk, dk, dv, dtype):
    return (_rand(rng, (n, hq, dk), dtype, 1.5), _rand(rng, (m, hk, dk), dtype),
            _rand(rng, (m, hk, dv), dtype), _rand(rng, (n, hq, dv), dtype))


def _check(q, k, v, do, lq, lk, causal, scale=None):
    """Forward and backward against the reference; lk None: the keys' lengths are lq"""
    dtype = q.dtype
    u = U[dtype] if dtype == BF16 else 0.0
    sq = _splits(lq)
    sk = sq if lk is None else _splits(lk)
    c = q.shape[2] ** -0.5 if scale is None else scale
    kw = dict(splits=_ints(sq), k_splits=None if lk is None else _ints(sk), scale=scale,
              causal=causal)
    o, lse = sbc.softmax_attention_forward(q, k, v, **kw)
    assert o.dtype == dtype and lse.dtype == F32
    qn, kn, vn = _np(q), _np(k), _np(v)
    ro, rl, to, tl = S.attention(qn, kn, vn, sq, sk, c, causal, u)
    _close(o, ro, to + U[dtype] * np.abs(ro), "o")
    _close(lse, rl, tl, "lse")
    grads = sbc.softmax_attention_backward(do, q, k, v, o, lse, **kw)
    ref, tol = S.attention_grad(_np(do), qn, kn, vn, _np(o), _np(lse), sq, sk, c, causal, u)
    for name, g, x, r, t in zip(("dq", "dk", "dv"), grads, (q, k, v), ref, tol):
        assert g.dtype == dtype and g.shape == x.shape
        _close(g, r, t + U[dtype] * np.abs(r), name)
    return o, lse, grads


# lengths, heads, channels: one token to several tiles, sizes next to 32, 64 and 128, empty
# sequences, heads in groups (of an odd number), channels of each tile and odd ones
CASES = [
    ([1], None, 1, 1, 16, 16),
    ([1], [300], 4, 1, 64, 64),
    ([3, 0, 1, 70], None, 2, 2, 32, 32),
    ([64], None, 1, 1, 64, 64),
    ([129], None, 2, 1, 64, 64),
    ([31, 33, 65, 127], None, 3, 1, 40, 72),
    ([200, 0, 57], [57, 10, 200], 4, 2, 64, 64),
    ([0, 40, 9], [30, 0, 300], 6, 3, 33, 31),
    ([257], [257], 8, 2, 128, 128),
    ([5, 300], None, 2, 2, 96, 96),
    ([130, 20], [20, 130], 12, 2, 128, 64),
    ([90], None, 16, 1, 7, 100),
    ([2] * 40 + [17], [3] * 40 + [100], 2, 1, 16, 16),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, causal, dtype):
    lq, lk, hq, hk, dk, dv = CASES[case]
    print(f"[softmax] {CASES[case]} causal {causal} {dtype}", flush=True)
    rng = np.random.default_rng(100 + case)
    n, m = sum(lq), sum(lq if lk is None else lk)
    _check(*_inputs(rng, n, m, hq, hk, dk, dv, dtype), lq, lk, causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [20, 64, 90, 128])
def test_attention_many_tiles(d, dtype):
    """Enough rows for workgroups of 128 (few rows take others), and so many row tiles that the
    gradients of keys come in parts"""
    print(f"[softmax tiles] {d} {dtype}", flush=True)
    rng = np.random.default_rng(d)
    lq = [700, 0, 431, 1, 520]
    n = sum(lq)
    for heads, causal, lk in (((12, 12), True, None), ((16, 8), False, [300, 40, 1000, 7, 60])):
        m = n if lk is None else sum(lk)
        _check(*_inputs(rng, n, m, *heads, d, d, dtype), lq, lk, causal)


def test_attention_without_splits():
    rng = np.random.default_rng(1)
    q, k, v, do = _inputs(rng, 50, 80, 4, 2, 32, 48, F32)
    o, lse = sbc.softmax_attention_forward(q, k, v, causal=True)
    o2, lse2 = sbc.softmax_attention_forward(q, k, v, splits=_ints([0, 50]),
                                             k_splits=_ints([0, 80]), scale=32 ** -0.5, causal=True)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    g = sbc.softmax_attention_backward(do, q, k, v, o, lse, causal=True)
    g2 = sbc.softmax_attention_backward(do, q, k, v, o, lse, splits=_ints([0, 50]),
                                        k_splits=_ints([0, 80]), causal=True)
    assert all(torch.equal(a, b) for a, b in zip(g, g2))


@pytest.mark.parametrize("n,m", [(0, 0), (0, 5), (5, 0)])
def test_attention_of_nothing(n, m):
    rng = np.random.default_rng(2)
    q, k, v, do = _inputs(rng, n, m, 2, 1, 16, 16, F32)
    o, lse = sbc.softmax_attention_forward(q, k, v)
    assert o.shape == (n, 2, 16) and not o.any() and bool((lse == -math.inf).all())
    dq, dk, dv = sbc.softmax_attention_backward(do, q, k, v, o, lse)
    assert not dq.any() and not dk.any() and not dv.any()
    assert dk.shape == k.shape


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_scores(dtype):
    """Scores of some hundreds: the maximum moves along the keys, most weights are zero."""
    rng = np.random.default_rng(3)
    q, k, v, do = _inputs(rng, 300, 300, 2, 2, 64, 64, dtype)
    k *= torch.linspace(0.1, 20, 300, device=DEV)[:, None, None].to(dtype)
    _check(q, k, v, do, [300], None, True, scale=0.5)
    _check(q, k.flip(0).contiguous(), v, do, [300], None, False, scale=0.5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,n", [((2, 1), 150), ((16, 8), 1100)])
def test_views(dtype, heads, n):
    """Parts of one projection, at odd offsets, with NaN between them; a shared key head by stride
    0 gives what its copies give; outputs and gradients do not read a row's neighbours."""
    rng = np.random.default_rng(4)
    (hq, hk), d = heads, 40
    wide = torch.full((n, hq + 2 * hk + 1, d + 3), math.nan, dtype=dtype, device=DEV)
    q, k, v = wide[:, :hq, 1:1 + d], wide[:, hq:hq + hk, 1:1 + d], wide[:, hq + hk:-1, 2:2 + d]
    for x in (q, k, v):
        x.copy_(_rand(rng, x.shape, dtype))
    do = _rand(rng, (hq, n, d), dtype).transpose(0, 1)
    got = sbc.softmax_attention_forward(q, k, v, causal=True)
    c = [x.contiguous() for x in (q, k, v)]
    ref = sbc.softmax_attention_forward(*c, causal=True)
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    g = sbc.softmax_attention_backward(do, q, k, v, *got, causal=True)
    r = sbc.softmax_attention_backward(do.contiguous(), *c, *got, causal=True)
    assert all(torch.equal(a, b) and bool(torch.isfinite(a.float()).all()) for a, b in zip(g, r))
    one_k, one_v = k[:, :1].expand(-1, hk, -1), v[:, :1].expand(-1, hk, -1)
    a = sbc.softmax_attention_forward(q, one_k, one_v, causal=True)
    b = sbc.softmax_attention_forward(q, one_k.contiguous(), one_v.contiguous(), causal=True)
    assert torch.equal(a[0], b[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,n", [((8, 4), 40), ((24, 8), 1300)])
def test_layouts(dtype, d, heads, n):
    """Heads before tokens, parts of a projection on and off 16 bytes, tokens in every second
    row: as contiguous ones, bit by bit."""
    rng = np.random.default_rng(14)
    hq, hk = heads
    c = [_rand(rng, (n, h, d), dtype) for h in (hq, hk, hk, hq)]

    def passes(q, k, v, do):
        o, lse = sbc.softmax_attention_forward(q, k, v, causal=True)
        return (o, lse, *sbc.softmax_attention_backward(do, q, k, v, o, lse, causal=True))

    want = passes(*c)
    heads_first = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in c]
    spread = []
    for x in c:
        y = torch.full((n, 2, x.shape[1], d), math.nan, dtype=dtype, device=DEV)
        y[:, 1] = x
        spread.append(y[:, 1])
    layouts = [heads_first, spread]
    for off in (8, 1):
        wide = torch.full((n, 2 * hq + 2 * hk, d + 16), math.nan, dtype=dtype, device=DEV)
        at, part = 0, []
        for x in c:
            part.append(wide[:, at:at + x.shape[1], off:off + d])
            part[-1].copy_(x)
            at += x.shape[1]
        layouts.append(part)
    for x in layouts:
        got = passes(*x)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 3e38])
@pytest.mark.parametrize("heads,n", [((2, 1), 100), ((32, 16), 600)])
def test_hidden_values_reach_no_row(dtype, value, heads, n):
    """Keys and values that are not finite, or whose scores are: rows that do not see them, in
    the same tiles, are as without them."""
    rng = np.random.default_rng(5)
    (hq, hk), d, at = heads, 64, [33, n - 30, n - 1]
    lq = [n, 50]
    q, k, v, _ = _inputs(rng, n + 50, n + 50, hq, hk, d, d, dtype)
    clean = sbc.softmax_attention_forward(q, k, v, splits=_ints(_splits(lq)), causal=True)
    for i in at:
        k2, v2 = k.clone(), v.clone()
        k2[i, :, 5], v2[i, :, 7] = value, value
        for kk, vv in ((k2, v), (k, v2)):
            o, lse = sbc.softmax_attention_forward(q, kk, vv, splits=_ints(_splits(lq)),
                                                   causal=True)
            for x, y in ((o, clean[0]), (lse, clean[1])):
                assert bool(torch.isfinite(x[:i].float()).all()), i
                # (keys one by one are summed in another order)
                assert bool(((x[:i].float() - y[:i].float()).abs()
                             <= 2.0 ** -7 * (1 + y[:i].float().abs())).all()), i
                assert torch.equal(x[n:], y[n:]), i
        if not math.isfinite(value):  # (and it does reach those that do)
            assert not bool(torch.isfinite(o[i, :, 7].float()).any())


def test_scores_of_minus_infinity():
    """bf16 keys of -inf have no weight (of float32 ones the smaller parts are NaN); a row that
    sees no others is 0, its sum -inf."""
    rng = np.random.default_rng(6)
    q, k, v, do = _inputs(rng, 40, 40, 1, 1, 16, 16, BF16)
    q = (q.abs() + 0.125).to(BF16)
    k[3:20] = -math.inf
    o, lse = sbc.softmax_attention_forward(q, k, v)
    keep = [0, 1, 2, *range(20, 40)]
    ref, rl = sbc.softmax_attention_forward(q, k[keep].contiguous(), v[keep].contiguous())
    assert bool(((o - ref).abs() <= 2.0 ** -6).all()) and bool(((lse - rl).abs() <= 2.0 ** -18).all())
    o, lse = sbc.softmax_attention_forward(q[:17], k[3:20], v[3:20], causal=True)
    assert not o.any() and bool((lse == -math.inf).all())
    dv = sbc.softmax_attention_backward(do[:17], q[:17], k[3:20], v[3:20], o, lse, causal=True)[2]
    assert not dv.any()


def test_gradients_against_differences():
    """Of the kernels' own outputs: <o, dO> in float32 along random directions."""
    rng = np.random.default_rng(7)
    q, k, v, do = _inputs(rng, 60, 60, 4, 2, 32, 32, F32)
    kw = dict(splits=_ints([0, 25, 60]), causal=True)
    o, lse = sbc.softmax_attention_forward(q, k, v, **kw)
    grads = sbc.softmax_attention_backward(do, q, k, v, o, lse, **kw)
    for i, g in enumerate(grads):
        for _ in range(3):
            d = _rand(rng, g.shape)
            h = 2.0 ** -6
            args = [[x + s * h * d if j == i else x for j, x in enumerate((q, k, v))]
                    for s in (1, -1)]
            up, down = (float((sbc.softmax_attention_forward(*a, **kw)[0].double()
                               * do.double()).sum()) for a in args)
            got, want = float((g.double() * d.double()).sum()), (up - down) / (2 * h)
            # third derivatives times h^2 / 6 (of 60 x 4 rows), and 2^-18 of the sum over 2 h
            assert abs(got - want) < 2.0 ** -12 * 10 * (1 + float((g * d).abs().sum())), i


def test_results_repeat():
    rng = np.random.default_rng(8)
    q, k, v, do = _inputs(rng, 2000, 2000, 8, 2, 64, 64, BF16)
    first = None
    for _ in range(3):
        o, lse = sbc.softmax_attention_forward(q, k, v, causal=True)
        out = (o, lse, *sbc.softmax_attention_backward(do, q, k, v, o, lse, causal=True))
        if first is None:
            first = out
        assert all(torch.equal(a, b) for a, b in zip(out, first))


def test_rows_in_no_sequence_stay():
    """The C ABI on arrays longer than the sequences: rows before the first and behind the last
    are left as they were."""
    rng = np.random.default_rng(9)
    for hq, n in ((2, 90), (64, 600)):
        q, k, v, do = _inputs(rng, n, n, hq, hq, 32, 32, BF16)
        splits = _ints([7, 7, n - 30])
        a = L.SbcSoftmaxAttention(n, n, 2, hq, hq, 32, 32, L.SBC_BF16, 0.2, 1, splits.data_ptr(), None)
        o, dq, dk, dv = (torch.full_like(q, 5.0) for _ in range(4))
        lse = torch.full((n, hq), 5.0, device=DEV)
        h = lambda x: ctypes.byref(L.SbcHeads(x.data_ptr(), x.stride(0), x.stride(1)))  # noqa: E731
        lib = L.lib()
        size = max(lib.sbc_softmax_attention_workspace_size(ctypes.byref(a)),
                   lib.sbc_softmax_attention_backward_workspace_size(ctypes.byref(a)))
        ws = torch.empty(size, dtype=torch.uint8, device=DEV)
        stream = torch.cuda.current_stream().cuda_stream
        L.check(lib.sbc_softmax_attention_forward(ctypes.byref(a), h(q), h(k), h(v), h(o),
                                                  lse.data_ptr(), ws.data_ptr(), size, stream))
        L.check(lib.sbc_softmax_attention_backward(ctypes.byref(a), h(do), h(q), h(k), h(v), h(o),
                                                   lse.data_ptr(), h(dq), h(dk), h(dv),
                                                   ws.data_ptr(), size, stream))
        torch.cuda.synchronize()
        for x in (o, lse, dq, dk, dv):
            assert bool((x[:7] == 5).all()) and bool((x[n - 30:] == 5).all())
            assert not bool((x[7:n - 30] == 5).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_other_stream_and_graph(dtype):
    """On a stream of its own, and captured: two graphs with their own workspaces, replayed in
    turn with eager calls between."""
    rng = np.random.default_rng(10)
    q, k, v, do = _inputs(rng, 400, 400, 8, 4, 64, 64, dtype)
    splits = _ints([0, 100, 400])

    def passes(q):
        o, lse = sbc.softmax_attention_forward(q, k, v, splits=splits, causal=True)
        return (o, lse, *sbc.softmax_attention_backward(do, q, k, v, o, lse, splits=splits,
                                                        causal=True))

    q2 = q.clone()
    want = [passes(q), passes(q2 * 2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = passes(q)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graphs, outs, ins = [], [], [q.clone(), q.clone()]
    for x in ins:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(passes(x))
        graphs.append(graph)
    for turn in range(3):
        for i in range(2):
            ins[i].copy_(q if (turn + i) % 2 == 0 else q2 * 2)
        for i in range(2):
            graphs[i].replay()
        passes(q)
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[(turn + i) % 2]))


def test_refusals():
    q, k, v = (torch.zeros(6, h, 16, device=DEV) for h in (4, 2, 2))
    f = sbc.softmax_attention_forward
    s = _ints([0, 6])
    for bad in (lambda: f(q[..., 0], k, v), lambda: f(q, k[..., :8], v), lambda: f(q, k, v[:5]),
                lambda: f(q, k.to(BF16), v), lambda: f(q.transpose(1, 2), k, v),
                lambda: f(q, k, v, splits=s.long()), lambda: f(q, k, v, k_splits=s),
                lambda: f(q, k, v, splits=s, k_splits=_ints([0, 3, 6])),
                lambda: f(q.half(), k.half(), v.half()),
                lambda: sbc.softmax_attention_backward(q, q, k, v, q, torch.zeros(6, 3, device=DEV)),
                lambda: sbc.softmax_attention_backward(q[:5], q, k, v, q, torch.zeros(6, 4, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: f(q, torch.zeros(6, 3, 16, device=DEV), torch.zeros(6, 3, 16, device=DEV)),
                lambda: f(q, k, v, scale=0.0), lambda: f(q, k, v, scale=math.inf),
                lambda: f(q[:5], k, v, splits=s)):
        with pytest.raises(L.SbcError):
            bad()
    wide = torch.zeros(2, 1, 129, device=DEV)
    with pytest.raises(L.SbcError):
        f(wide, wide, wide)
