"""The sequence operators on the GPU against plain float64 (tests/sequence_ref.py).

Tolerances, from the terms' magnitudes (`size`): float32 sums of up to some 2^8
roundings of 2^-24, most of which cancel, and products of operands split to 2^-22:
2^-18 of size.  Of bf16 inputs, what is computed is split to 2^-17 twice (the products of
a chunk and the state): 2^-15 of size, and the output's rounding, 2^-8 of itself.  The
state, the gradients of the rates and the norm's sums are float32 for either type.
"""
import numpy as np
import pytest
import torch

import paper_2012_01170_amd as sbc
from tests import sequence_ref as R

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -8       # half a unit of bf16


def _rand(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DEV).to(dtype)


def _np(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def _close(got, ref, tol, what):
    got = _np(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.isfinite(got).all(), what
    bad = np.abs(got - ref) - tol
    assert bad.max(initial=0.0) <= 0, f"{what}: {np.abs(got - ref).max()} off, {bad.max()} over"


# ---------------------------------------------------------------- layer norm
NORM_SHAPES = [(1, 1), (3, 1), (1, 7), (5, 8), (300, 32), (257, 33), (64, 64), (100, 100),
               (129, 127), (33, 256), (40, 513), (19, 1001), (9, 2048), (7, 2049), (6, 4099),
               (5, 8192), (3, 8193), (2, 20001), (4099, 16)]


def _norm_tol(x, w, b, mean, rstd, dtype):
    xn = (x - mean[:, None]) * rstd[:, None]
    w = np.ones(x.shape[1]) if w is None else np.abs(w)
    size = w * (rstd[:, None] * (np.abs(x) + np.abs(x).mean(1, keepdims=True)) + np.abs(xn))
    y = 2.0 ** -20 * (size + (0 if b is None else np.abs(b)))
    return y


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", NORM_SHAPES)
def test_layer_norm(n, c, dtype):
    print(f"[norm] {n} x {c} {dtype}", flush=True)
    rng = np.random.default_rng(n * 7 + c)
    x = (_rand(rng, (n, c), F32) * 2 + 0.5 * _rand(rng, (c,), F32)).to(dtype)
    w, b = 1 + 0.3 * _rand(rng, (c,), F32), _rand(rng, (c,), F32)
    dy = _rand(rng, (n, c), dtype)
    for ww, bb in ((w, b), (None, None)):
        y, mean, rstd = sbc.layer_norm_forward(x, ww, bb, eps=1e-5)
        wn, bn = (None if v is None else _np(v) for v in (ww, bb))
        ry, rm, rr = R.layer_norm(_np(x), wn, bn, 1e-5)
        tol = _norm_tol(_np(x), wn, bn, rm, rr, dtype)
        _close(y, ry, tol + (U * np.abs(ry) if dtype == BF16 else 0), "y")
        _close(mean, rm, 2.0 ** -20 * np.abs(_np(x)).mean(1) + 1e-30, "mean")
        _close(rstd, rr, 2.0 ** -18 * rr, "rstd")
        assert y.dtype == dtype and mean.dtype == F32
        dx, dw, db = sbc.layer_norm_backward(dy, x, ww, mean, rstd)
        rdx, rdw, rdb = R.layer_norm_grad(_np(dy), _np(x), wn, _np(mean), _np(rstd))
        # dx's three terms, with the means of magnitudes
        xn = np.abs((_np(x) - _np(mean)[:, None]) * _np(rstd)[:, None]) \
            + 2.0 ** -3 * np.abs(_np(mean) * _np(rstd))[:, None]
        g = np.abs(_np(dy) * (1 if wn is None else wn))
        size = _np(rstd)[:, None] * (g + g.mean(1, keepdims=True)
                                     + xn * (g * xn).mean(1, keepdims=True))
        _close(dx, rdx, 2.0 ** -19 * size + (U * np.abs(rdx) if dtype == BF16 else 0), "dx")
        _close(dw, rdw, 2.0 ** -19 * (np.abs(_np(dy)) * xn).sum(0) + 1e-30, "dw")
        _close(db, rdb, 2.0 ** -19 * np.abs(_np(dy)).sum(0), "db")


def test_layer_norm_many_rows():
    """More rows than a pass of all workgroups takes."""
    n, c = 70_001, 24
    x = torch.randn(n, c, device=DEV, dtype=F32)
    dy = torch.randn(n, c, device=DEV, dtype=F32)
    w = torch.randn(c, device=DEV)
    y, mean, rstd = sbc.layer_norm_forward(x, w)
    dx, dw, db = sbc.layer_norm_backward(dy, x, w, mean, rstd)
    rdx, rdw, rdb = R.layer_norm_grad(_np(dy), _np(x), _np(w), _np(mean), _np(rstd))
    _close(dw, rdw, 2.0 ** -19 * np.abs(_np(dy) * _np(x)).sum(0), "dw")
    _close(db, rdb, 2.0 ** -19 * np.abs(_np(dy)).sum(0), "db")
    again = sbc.layer_norm_backward(dy, x, w, mean, rstd)
    for a, b in zip((dx, dw, db), again):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layer_norm_views_and_parts(dtype):
    """Rows of a wider array that start off 16 bytes, with NaN between them; outputs left out."""
    rng = np.random.default_rng(5)
    n, c = 61, 45
    wide = torch.full((n, 101), float("nan"), dtype=dtype, device=DEV)
    x = wide[:, 3:3 + c]
    x.copy_(_rand(rng, (n, c), dtype))
    dyw = torch.full((n, 77), float("nan"), dtype=dtype, device=DEV)
    dy = dyw[:, 1:1 + c]
    dy.copy_(_rand(rng, (n, c), dtype))
    w = _rand(rng, (c,), F32)
    y, mean, rstd = sbc.layer_norm_forward(x, w)
    y2, _, _ = sbc.layer_norm_forward(x.contiguous(), w)
    assert torch.equal(y, y2) and bool(torch.isfinite(y.float()).all())
    full = sbc.layer_norm_backward(dy.contiguous(), x.contiguous(), w, mean, rstd)
    part = sbc.layer_norm_backward(dy, x, w, mean, rstd)
    for a, b in zip(full, part):
        assert torch.equal(a, b)
    dx, dw, db = sbc.layer_norm_backward(dy, x, w, mean, rstd, need_dbias=False)
    assert db is None and torch.equal(dw, full[1]) and torch.equal(dx, full[0])
    dx, dw, db = sbc.layer_norm_backward(dy, x, w, mean, rstd, need_dx=False)
    assert dx is None and torch.equal(dw, full[1]) and torch.equal(db, full[2])
    assert sbc.layer_norm_forward(x, w, stats=False)[1] is None


def test_layer_norm_of_nothing_and_of_a_broken_row():
    x = torch.empty(0, 16, device=DEV)
    y, mean, rstd = sbc.layer_norm_forward(x)
    assert y.shape == (0, 16) and mean.numel() == 0
    dx, dw, db = sbc.layer_norm_backward(x, x, None, mean, rstd)
    assert dx.shape == (0, 16) and not dw.any() and not db.any()
    x = torch.randn(40, 24, device=DEV)
    x[7, 3], x[9, 0] = float("nan"), float("inf")
    y, mean, rstd = sbc.layer_norm_forward(x)
    bad = torch.zeros(40, dtype=torch.bool, device=DEV)
    bad[7] = bad[9] = True
    assert torch.isfinite(y[~bad]).all() and not torch.isfinite(y[bad]).any()
    # a constant row has no spread: zero, not a division by zero
    y, _, rstd = sbc.layer_norm_forward(torch.full((3, 24), 5.0, device=DEV))
    assert not y.any() and torch.isfinite(rstd).all()


# ---------------------------------------------------------------- rotary
def _rotary_tol(x, ref, dtype):
    pair = np.abs(x).max(axis=-1, keepdims=True)
    return 2.0 ** -21 * pair + (U * np.abs(ref) if dtype == BF16 else 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,hq,hk,d,sections,kind", [
    (1, 1, 1, 2, (1,), "int"), (77, 4, 4, 64, (16, 8, 8), "int"), (40, 2, 1, 64, (11, 11, 10), "float"),
    (33, 3, 0, 40, (7, 0, 6), "float"), (29, 0, 2, 33, (5, 5, 5, 1), "int"),
    (513, 1, 2, 18, (3, 3, 3), "float"), (12, 2, 2, 128, (64,), "big"), (9, 1, 1, 7, (2, 1), "big"),
])
def test_rotary(n, hq, hk, d, sections, kind, interleaved, dtype):
    print(f"[rotary] {n} {hq} {hk} {d} {sections} {kind} {interleaved} {dtype}", flush=True)
    rng = np.random.default_rng(n + d)
    a = len(sections)
    if kind == "float":
        pos = torch.from_numpy(rng.uniform(-3, 3, (n, a)).astype(np.float32)).to(DEV)
    else:
        hi = 1 << 30 if kind == "big" else 1000
        pos = torch.from_numpy(rng.integers(-hi, hi, (n, a)).astype(np.int32)).to(DEV)
    freqs = torch.from_numpy(rng.uniform(0.001, 2, sum(sections)).astype(np.float32)).to(DEV)
    q = _rand(rng, (n, hq, d), dtype) if hq else None
    k = _rand(rng, (n, hk, d), dtype) if hk else None
    pn, fn = pos.cpu().numpy(), freqs.cpu().numpy()
    for call, sign in ((sbc.rotary_forward, 1.0), (sbc.rotary_backward, -1.0)):
        got = call(q, k, pos, freqs, sections, interleaved=interleaved)
        for x, y in zip((q, k), got):
            if x is None:
                assert y is None
                continue
            ref = R.rotary(_np(x), pn, fn, sections, interleaved, sign)
            _close(y, ref, _rotary_tol(_np(x), ref, dtype), "rotary")
            m = sum(sections)
            assert torch.equal(y[..., 2 * m:], x[..., 2 * m:])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rotary_of_a_projection_in_place(dtype, interleaved):
    """q and k as parts of one projection, turned in place; the values beside them stay."""
    rng = np.random.default_rng(8)
    n, h, d, sections = 50, 3, 20, (4, 3, 2)
    qkv = _rand(rng, (n, 3 * h * d + 1), dtype)
    before = qkv.clone()
    q, k = (qkv[:, 1 + i * h * d:1 + (i + 1) * h * d].view(n, h, d) for i in (0, 1))
    pos = torch.from_numpy(rng.uniform(-3, 3, (n, 5)).astype(np.float32)).to(DEV)[:, 1:4]
    freqs = torch.rand(9, device=DEV)
    want = sbc.rotary_forward(q.contiguous(), k.contiguous(), pos.contiguous(), freqs, sections,
                              interleaved=interleaved)
    got = sbc.rotary_forward(q, k, pos, freqs, sections, interleaved=interleaved, inplace=True)
    assert got[0].data_ptr() == q.data_ptr()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(qkv[:, 1 + 2 * h * d:], before[:, 1 + 2 * h * d:])
    assert torch.equal(qkv[:, 0], before[:, 0])
    # turned back
    back = sbc.rotary_backward(q.contiguous(), None, pos, freqs, sections, interleaved=interleaved)
    ref = _np(before[:, 1:1 + h * d].reshape(n, h, d))
    tol = 2.0 ** -20 * np.abs(ref).max() + (2 * U * np.abs(ref).max() if dtype == BF16 else 0)
    _close(back[0], ref, tol, "back")


# ---------------------------------------------------------------- linear attention
# (n, splits, heads, dk, dv)
ATTN = [
    (1, [0, 1], 1, 1, 1), (2, [0, 1, 2], 2, 8, 8), (63, [0, 63], 1, 32, 32),
    (64, [0, 64], 1, 32, 64), (65, [0, 65], 2, 64, 64), (200, [0, 0, 130, 130, 200, 200], 2, 64, 64),
    (300, [0, 1, 2, 70, 299, 300], 1, 40, 72), (513, [0, 256, 513], 1, 33, 31),
    (700, [0, 700], 2, 64, 48), (640, [0, 100, 600, 640], 1, 128, 128), (257, [0, 257], 1, 5, 128),
    (1100, [0, 255, 256, 1100], 1, 96, 100),
]
RATES = [0.15, 0.002, 0.0, 3.0]


def _attn_inputs(n, h, dk, dv, dtype, seed, times):
    rng = np.random.default_rng(seed)
    q, k = _rand(rng, (n, h, dk), dtype), _rand(rng, (n, h, dk), dtype)
    v, do = _rand(rng, (n, h, dv), dtype), _rand(rng, (n, h, dv), dtype)
    rates = torch.tensor([RATES[i % 4] for i in range(h)], device=DEV) * (0.3 if times else 1)
    t = None
    if times:  # runs of equal times and gaps
        t = torch.from_numpy(np.cumsum(rng.integers(0, 3, n) * rng.integers(0, 4, n)).astype(np.int32)
                             + 1000).to(DEV)
    return q, k, v, do, rates, t


def _tol(ref, size, dtype):
    return 2.0 ** -18 * size + 1e-30 if dtype == F32 else 2.0 ** -15 * size + U * np.abs(ref) + 1e-30


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("times", [False, True])
@pytest.mark.parametrize("with_state", [False, True])
@pytest.mark.parametrize("n,splits,h,dk,dv", ATTN)
def test_attention_forward(n, splits, h, dk, dv, with_state, times, dtype):
    print(f"[attn] {n} {splits} {h} {dk} {dv} {with_state} {times} {dtype}", flush=True)
    q, k, v, _, rates, t = _attn_inputs(n, h, dk, dv, dtype, n + dk, times)
    sp = torch.tensor(splits, dtype=torch.int32, device=DEV)
    b, scale = len(splits) - 1, 0.25
    state = time = None
    if with_state:
        state = torch.randn(b, h, dk, dv, device=DEV)
        time = torch.full((b,), 990, dtype=torch.int32, device=DEV) if times else None
    o, S, T = sbc.linear_attention_forward(q, k, v, rates, splits=sp, t=t, scale=scale,
                                           state=state, state_time=time, return_state=True)
    n_ = lambda x: None if x is None else _np(x)  # noqa: E731
    tn = None if t is None else t.cpu().numpy()
    args = (splits, tn, scale)
    ro, rS, rT, size = R.attention(_np(q), _np(k), _np(v), _np(rates), *args, n_(state), n_(time))
    sS = R.attention(abs(_np(q)), abs(_np(k)), abs(_np(v)), _np(rates), *args,
                     None if state is None else abs(_np(state)), n_(time))[1]
    _close(o, ro, _tol(ro, size, dtype), "o")
    _close(S, rS, 2.0 ** -18 * sS + 1e-30, "state")
    if times:
        assert np.array_equal(T.cpu().numpy(), rT)
    else:
        assert T is None
    o2 = sbc.linear_attention_forward(q, k, v, rates, splits=sp, t=t, scale=scale, state=state,
                                      state_time=time)
    assert torch.equal(o, o2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("times", [False, True])
@pytest.mark.parametrize("n,splits,h,dk,dv", ATTN)
def test_attention_backward(n, splits, h, dk, dv, times, dtype):
    print(f"[attn grad] {n} {splits} {h} {dk} {dv} {times} {dtype}", flush=True)
    q, k, v, do, rates, t = _attn_inputs(n, h, dk, dv, dtype, n + dv, times)
    sp = torch.tensor(splits, dtype=torch.int32, device=DEV)
    scale = 0.5
    got = sbc.linear_attention_backward(do, q, k, v, rates, splits=sp, t=t, scale=scale)
    tn = None if t is None else t.cpu().numpy()
    ref, size, total = R.attention_grad(_np(do), _np(q), _np(k), _np(v), _np(rates), splits, tn,
                                        scale)
    for name, g, r, s in zip(("dq", "dk", "dv"), got, ref, size):
        _close(g, r, _tol(r, s, dtype), name)
    # the rates: sums of token's terms (2^-21 of their magnitudes, most of which cancel) times
    # times within a segment
    tt = np.arange(n) if t is None else tn
    span = max(tt[min(i + 511, n - 1)] - tt[i] for i in range(n))
    _close(got[3], ref[3], 2.0 ** -18 * size[3] + 2.0 ** -21 * span * total + 1e-30, "drates")
    again = sbc.linear_attention_backward(do, q, k, v, rates, splits=sp, t=t, scale=scale)
    for a, b in zip(got, again):
        assert torch.equal(a, b)
    less = sbc.linear_attention_backward(do, q, k, v, rates, splits=sp, t=t, scale=scale,
                                         need_rates=False)
    assert less[3] is None and all(torch.equal(a, b) for a, b in zip(got[:3], less[:3]))


@pytest.mark.parametrize("times", [False, True])
def test_attention_gradients_against_differences(times):
    """The kernels' gradients along random directions against the float64 forward's
    differences; the differences' own error is below 1e-6 of the terms."""
    n, h, dk, dv, splits, scale = 150, 2, 24, 20, [0, 40, 150], 0.3
    q, k, v, do, rates, t = _attn_inputs(n, h, dk, dv, F32, 77, times)
    got = sbc.linear_attention_backward(do, q, k, v, rates, t=t, scale=scale,
                                        splits=torch.tensor(splits, dtype=torch.int32, device=DEV))
    tn = None if t is None else t.cpu().numpy()
    base = [_np(x) for x in (q, k, v, rates)]
    ref, size, total = R.attention_grad(_np(do), *base, splits, tn, scale)
    rng = np.random.default_rng(1)
    for i in range(4):
        d = rng.standard_normal(base[i].shape)
        f = []
        for s in (1e-5, -1e-5):
            a = list(base)
            a[i] = a[i] + s * d
            f.append((R.attention(*a, splits, tn, scale)[0] * _np(do)).sum())
        slope = (f[0] - f[1]) / 2e-5
        span = (n if t is None else tn[-1] - tn[0])
        sz = size[i] + (2.0 ** -3 * span * total if i == 3 else 0)
        assert abs(slope - (_np(got[i]) * d).sum()) <= 2.0 ** -17 * (sz * abs(d)).sum(), i


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_segments_meet(dtype):
    """One long sequence, and one beside short ones, over many segments."""
    for n, splits in ((9001, [0, 9001]), (6007, [0, 3, 5, 4000, 4000, 6007])):
        h, dk, dv = 2, 32, 32
        q, k, v, do, _, t = _attn_inputs(n, h, dk, dv, dtype, n, True)
        rates = torch.tensor([0.0005, 0.05], device=DEV)
        sp = torch.tensor(splits, dtype=torch.int32, device=DEV)
        tn = t.cpu().numpy()
        args = (_np(rates), splits, tn, 0.2)
        o, S, T = sbc.linear_attention_forward(q, k, v, rates, splits=sp, t=t, scale=0.2,
                                               return_state=True)
        ro, rS, _, size = R.attention(_np(q), _np(k), _np(v), *args)
        sS = R.attention(abs(_np(q)), abs(_np(k)), abs(_np(v)), *args)[1]
        _close(o, ro, _tol(ro, size, dtype), "o")
        _close(S, rS, 2.0 ** -18 * sS + 1e-30, "state")
        got = sbc.linear_attention_backward(do, q, k, v, rates, splits=sp, t=t, scale=0.2)
        ref, sz, total = R.attention_grad(_np(do), _np(q), _np(k), _np(v), *args)
        for name, g, r, s in zip(("dq", "dk", "dv"), got, ref, sz):
            _close(g, r, _tol(r, s, dtype), name)
        span = max(tn[min(i + 511, n - 1)] - tn[i] for i in range(n))
        _close(got[3], ref[3], 2.0 ** -18 * sz[3] + 2.0 ** -21 * span * total, "drates")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_views(dtype):
    """Parts of one projection (rows off 16 bytes, NaN beside them), heads before tokens, and
    one head of keys and values shared by all."""
    n, h, d = 210, 3, 24
    rng = np.random.default_rng(2)
    rates = torch.tensor([0.1, 0.01, 0.5], device=DEV)
    wide = torch.full((n, 3 * h * d + 5), float("nan"), dtype=dtype, device=DEV)
    parts = [wide[:, 1 + i * h * d:1 + (i + 1) * h * d].view(n, h, d) for i in range(3)]
    for p in parts:
        p.copy_(_rand(rng, (n, h, d), dtype))
    do = _rand(rng, (n, h, d), dtype)
    dense = [p.contiguous() for p in parts]
    o = sbc.linear_attention_forward(*parts, rates)
    want = sbc.linear_attention_forward(*dense, rates)
    assert torch.equal(o, want) and torch.isfinite(o.float()).all()
    g = sbc.linear_attention_backward(do, *parts, rates)
    gw = sbc.linear_attention_backward(do, *dense, rates)
    assert all(torch.equal(a, b) for a, b in zip(g, gw))
    first = [p.transpose(0, 1).contiguous().transpose(0, 1) for p in dense]
    assert first[0].stride(0) == d
    assert torch.equal(sbc.linear_attention_forward(*first, rates), want)
    k1, v1 = dense[1][:, :1].expand(n, h, d), dense[2][:, :1].expand(n, h, d)
    assert torch.equal(sbc.linear_attention_forward(dense[0], k1, v1, rates),
                       sbc.linear_attention_forward(dense[0], k1.contiguous(), v1.contiguous(),
                                                    rates))


def test_attention_long_gaps_and_a_clock_that_wraps():
    """Gaps that pass 2^24 and times that pass 2^31: differences stay exact."""
    n, h, d = 190, 2, 32
    q, k, v, do, _, _ = _attn_inputs(n, h, d, d, F32, 4, False)
    rates = torch.tensor([0.05, 1e-9], device=DEV)
    rng = np.random.default_rng(0)
    t = np.cumsum(np.where(rng.random(n) < 0.05, 150_000_000, rng.integers(0, 5, n))).astype(np.int64)
    t += 2_000_000_000 - t[90]
    assert t[-1] > 2 ** 31 and t[-1] - t[0] < 2 ** 32
    wrapped = torch.from_numpy(((t + 2 ** 31) % 2 ** 32 - 2 ** 31).astype(np.int32)).to(DEV)
    args = (_np(rates), [0, n], t, 1.0)
    ro, _, _, size = R.attention(_np(q), _np(k), _np(v), *args)
    _close(sbc.linear_attention_forward(q, k, v, rates, t=wrapped), ro, _tol(ro, size, F32), "o")
    ref, sz, _ = R.attention_grad(_np(do), _np(q), _np(k), _np(v), *args)
    got = sbc.linear_attention_backward(do, q, k, v, rates, t=wrapped)
    for name, g, r, s in zip(("dq", "dk", "dv"), got, ref, sz):
        _close(g, r, _tol(r, s, F32), name)


def test_attention_of_other_sequences_stays_apart():
    """A NaN in one sequence reaches no other, and no token before its chunk of 64."""
    n, h, d = 400, 1, 32
    q, k, v, do, rates, _ = _attn_inputs(n, h, d, d, F32, 6, False)
    sp = torch.tensor([0, 100, 101, 400], dtype=torch.int32, device=DEV)
    v[100, 0, 0] = float("nan")
    q[100, 0, 1] = float("inf")
    o = sbc.linear_attention_forward(q, k, v, rates, splits=sp)
    g = sbc.linear_attention_backward(do, q, k, v, rates, splits=sp)
    for x in (o, *g[:3]):
        rest = torch.cat([x[:100], x[101:]])
        assert torch.isfinite(rest).all()
    k[300, 0, 0] = float("nan")
    o = sbc.linear_attention_forward(q, k, v, rates, splits=sp)
    assert torch.isfinite(o[101:300]).all() and not torch.isfinite(o[300:]).all()


def test_attention_of_nothing():
    z = torch.empty(0, 2, 8, device=DEV)
    rates = torch.ones(2, device=DEV)
    assert sbc.linear_attention_forward(z, z, z, rates).shape == (0, 2, 8)
    sp = torch.zeros(4, dtype=torch.int32, device=DEV)
    state = torch.randn(3, 2, 8, 8, device=DEV)
    o, S, _ = sbc.linear_attention_forward(z, z, z, rates, splits=sp, state=state, return_state=True)
    assert torch.equal(S, state)
    _, S, _ = sbc.linear_attention_forward(z, z, z, rates, splits=sp, return_state=True)
    assert not S.any()
    dq, dk, dv, dr = sbc.linear_attention_backward(z, z, z, z, rates, splits=sp)
    assert dq.shape == (0, 2, 8) and not dr.any()


# ---------------------------------------------------------------- the step
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("times", [False, True])
@pytest.mark.parametrize("b,h,dk,dv", [(1, 1, 1, 1), (1, 4, 64, 64), (3, 2, 33, 31), (5, 1, 40, 72),
                                       (65, 2, 128, 128), (2, 3, 64, 130 - 2)])
def test_step(b, h, dk, dv, times, dtype):
    print(f"[step] {b} {h} {dk} {dv} {times} {dtype}", flush=True)
    rng = np.random.default_rng(b + dk)
    q, k, v = (_rand(rng, (b, h, d), dtype) for d in (dk, dk, dv))
    rates = torch.rand(h, device=DEV) * 0.1
    state = _rand(rng, (b, h, dk, dv), F32)
    t = time = None
    if times:
        time = torch.randint(0, 100, (b,), device=DEV, dtype=torch.int32)
        t = time + torch.randint(0, 50, (b,), device=DEV, dtype=torch.int32)
    args = (_np(rates), list(range(b + 1)), None if t is None else t.cpu().numpy(), 0.3)
    n_ = lambda x: None if x is None else _np(x)  # noqa: E731
    ro, rS, _, size = R.attention(_np(q), _np(k), _np(v), *args, _np(state), n_(time))
    sS = R.attention(abs(_np(q)), abs(_np(k)), abs(_np(v)), *args, abs(_np(state)), n_(time))[1]
    o, S, T = sbc.linear_attention_step(q, k, v, rates, state, t=t, state_time=time, scale=0.3)
    tol = 2.0 ** -18 * size + (U * np.abs(ro) if dtype == BF16 else 0)
    _close(o, ro, tol, "o")
    _close(S, rS, 2.0 ** -21 * sS, "state")
    assert T is None if t is None else torch.equal(T, t)
    # in place, from strided tokens
    wide = torch.full((b, h * (2 * dk + dv) + 3), float("nan"), dtype=dtype, device=DEV)
    cut = np.cumsum([1, h * dk, h * dk, h * dv])
    views = [wide[:, a:z].view(b, h, -1) for a, z in zip(cut, cut[1:])]
    for x, y in zip(views, (q, k, v)):
        x.copy_(y)
    o2, S2, _ = sbc.linear_attention_step(*views, rates, state, t=t, state_time=time, scale=0.3,
                                          out_state=state)
    assert S2 is state and torch.equal(S2, S) and torch.equal(o2, o)


def test_prompt_then_steps_is_the_whole():
    n, b, h, d = 90, 2, 2, 32
    q, k, v, _, rates, t = _attn_inputs(n * b, h, d, d, F32, 21, True)
    sp = torch.tensor([0, n, 2 * n], dtype=torch.int32, device=DEV)
    tn = t.cpu().numpy()
    ro, rS, _, size = R.attention(_np(q), _np(k), _np(v), _np(rates), [0, n, 2 * n], tn, 1.0)
    cut = n - 5
    at = torch.cat([torch.arange(cut), n + torch.arange(cut)]).to(DEV)
    o, S, T = sbc.linear_attention_forward(
        q[at], k[at], v[at], rates, t=t[at], return_state=True,
        splits=torch.tensor([0, cut, 2 * cut], dtype=torch.int32, device=DEV))
    for i in range(cut, n):
        at = torch.tensor([i, n + i], device=DEV)
        o, S, T = sbc.linear_attention_step(q[at], k[at], v[at], rates, S, t=t[at], state_time=T)
        r = at.cpu().numpy()
        _close(o, ro[r], 2.0 ** -17 * size[r], f"token {i}")


# ---------------------------------------------------------------- streams and graphs
def _layer(x, w, pos, freqs, rates, t, dy):
    y, mean, rstd = sbc.layer_norm_forward(x, w)
    n, c = x.shape
    q, k = sbc.rotary_forward(y.view(n, 2, c // 2), y.view(n, 2, c // 2), pos, freqs, (4, 2, 2))
    v = y.view(n, 2, c // 2)
    o, S, T = sbc.linear_attention_forward(q, k, v, rates, t=t, return_state=True)
    dq, dk, dv, dr = sbc.linear_attention_backward(dy.view(n, 2, c // 2), q, k, v, rates, t=t)
    dq, dk = sbc.rotary_backward(dq, dk, pos, freqs, (4, 2, 2))
    dx, dw, db = sbc.layer_norm_backward(dq.view(n, c), x, w, mean, rstd)
    step = sbc.linear_attention_step(q[:1], k[:1], v[:1], rates, S, t=t[:1], state_time=T)
    return y, o, S, T, dk, dv, dr, dx, dw, db, *step


def _layer_inputs(n=900, c=64):
    rng = np.random.default_rng(12)
    x, dy, w = _rand(rng, (n, c), BF16), _rand(rng, (n, c), BF16), _rand(rng, (c,), F32)
    pos = torch.from_numpy(rng.integers(0, 99, (n, 3)).astype(np.int32)).to(DEV)
    t = torch.arange(n, dtype=torch.int32, device=DEV)
    return x, w, pos, torch.rand(8, device=DEV), torch.tensor([0.01, 0.2], device=DEV), t, dy


def test_graph_replays_match_eager():
    args = _layer_inputs()
    eager = [x.clone() for x in _layer(*args)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for a, b in zip(eager, _layer(*args)):  # and on a stream of one's own
            assert torch.equal(a, b)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = _layer(*args)
    for r in range(3):
        junk = torch.randn(1 << 16, device=DEV).sum()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, outs):
            assert torch.equal(a, b), f"replay {r} differs"


def test_binding_refusals():
    x = torch.zeros(4, 2, 8, device=DEV)
    rates = torch.ones(2, device=DEV)
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    state = torch.zeros(1, 2, 8, 8, device=DEV)
    f = sbc.linear_attention_forward
    for call in (
        lambda: f(x.cpu(), x, x, rates), lambda: f(x, x.bfloat16(), x, rates),
        lambda: f(x, x[:, :1], x, rates), lambda: f(x, x, x[:3], rates),
        lambda: f(x, x, x, rates[:1]), lambda: f(x, x, x, rates.double()),
        lambda: f(x, x, x, rates, t=t.long()), lambda: f(x, x, x, rates, t=t[:2]),
        lambda: f(x.transpose(1, 2).contiguous().transpose(1, 2), x, x, rates),
        lambda: f(x.half(), x.half(), x.half(), rates),
        lambda: f(x, x, x, rates, state=state[..., :4].contiguous()),
        lambda: f(x, x, x, rates, t=t, state=state),
        lambda: f(x, x, x, rates, splits=t.float()),
        lambda: sbc.linear_attention_step(x, x, x, rates, None),
        lambda: sbc.linear_attention_backward(x[:2], x, x, x, rates),
        lambda: sbc.rotary_forward(None, None, t.view(4, 1), rates, (2,)),
        lambda: sbc.rotary_forward(x, None, t.view(4, 1), rates, (2, 1)),
        lambda: sbc.rotary_forward(x, None, t.view(4, 1), rates, (3,)),
        lambda: sbc.rotary_forward(x, x[:2], t.view(4, 1), rates, (2,)),
        lambda: sbc.layer_norm_forward(x), lambda: sbc.layer_norm_forward(x[0], rates),
        lambda: sbc.layer_norm_backward(x[0], x[1][:, :4], None, rates, rates),
        lambda: sbc.layer_norm_backward(x[0], x[1], None, rates[:1], rates),
    ):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(sbc.ops.L.SbcError, match="UNSUPPORTED"):
        big = torch.zeros(2, 1, 129, device=DEV)
        f(big, big, big, rates[:1])
    with pytest.raises(sbc.ops.L.SbcError, match="INVALID_ARG"):
        sbc.layer_norm_forward(x[0], eps=-1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("h,dk,dv", [(8, 64, 64), (8, 32, 24), (7, 96, 72), (8, 40, 128)])
def test_attention_of_many_workgroups(h, dk, dv, dtype):
    """Enough segments and heads that the passes of the gradients are launched one by one
    (fewer share a launch), and that CUs take several workgroups."""
    n, splits = 7100, [0, 900, 901, 901, 3000, 4500, 7100]
    print(f"[attn many] {h} {dk} {dv} {dtype}", flush=True)
    q, k, v, do, _, t = _attn_inputs(n, h, dk, dv, dtype, 31, True)
    rates = torch.tensor([0.0005, 0.05, 0.2, 0.01, 0.003, 1.0, 0.0, 0.1], device=DEV)[:h].clone()
    sp = torch.tensor(splits, dtype=torch.int32, device=DEV)
    tn = t.cpu().numpy()
    args = (_np(rates), splits, tn, 0.2)
    o, S, T = sbc.linear_attention_forward(q, k, v, rates, splits=sp, t=t, scale=0.2,
                                           return_state=True)
    ro, rS, _, size = R.attention(_np(q), _np(k), _np(v), *args)
    sS = R.attention(abs(_np(q)), abs(_np(k)), abs(_np(v)), *args)[1]
    _close(o, ro, _tol(ro, size, dtype), "o")
    _close(S, rS, 2.0 ** -18 * sS + 1e-30, "state")
    got = sbc.linear_attention_backward(do, q, k, v, rates, splits=sp, t=t, scale=0.2)
    ref, sz, total = R.attention_grad(_np(do), _np(q), _np(k), _np(v), *args)
    for name, g, r, s in zip(("dq", "dk", "dv"), got, ref, sz):
        _close(g, r, _tol(r, s, dtype), name)
    span = max(tn[min(i + 511, n - 1)] - tn[i] for i in range(n))
    _close(got[3], ref[3], 2.0 ** -18 * sz[3] + 2.0 ** -21 * span * total, "drates")
    less = sbc.linear_attention_backward(do, q, k, v, rates, splits=sp, t=t, scale=0.2,
                                         need_rates=False)
    assert all(torch.equal(a, b) for a, b in zip(got[:3], less[:3]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,dv", [(64, 64), (40, 72), (33, 31)])
def test_attention_forward_keeps_broken_values_from_earlier_tokens(d, dv, dtype):
    """Infinities and NaN in q, k and v: earlier tokens, earlier and later sequences are what
    they are without them, bit by bit or within the chunk's rounding."""
    n, splits = 500, [0, 120, 500]
    q, k, v, _, _, _ = _attn_inputs(n, 1, d, dv, dtype, 3, False)
    rates = torch.tensor([0.01], device=DEV)
    sp = torch.tensor(splits, dtype=torch.int32, device=DEV)
    want, S0, _ = sbc.linear_attention_forward(q, k, v, rates, splits=sp, return_state=True)
    ro, _, _, size = R.attention(_np(q), _np(k), _np(v), _np(rates), splits, None, 1.0)
    for which, at, value in ((v, 37, float("nan")), (v, 400, float("inf")), (v, 499, -float("inf")),
                             (k, 201, float("nan")), (q, 300, float("nan"))):
        kept = which[at, 0, 1].item()
        which[at, 0, 1] = value
        o, S, _ = sbc.linear_attention_forward(q, k, v, rates, splits=sp, return_state=True)
        b = 0 if at < 120 else 1
        clean = torch.ones(n, dtype=torch.bool, device=DEV)
        clean[at:splits[b + 1]] = False
        m = clean.cpu().numpy()
        _close(o[clean], ro[m], _tol(ro, size, dtype)[m], "earlier tokens")
        hit = o[at, 0] if which is not v else o[at, 0, 1:2]
        assert not torch.isfinite(hit.float()).any()
        assert torch.equal(S[1 - b], S0[1 - b])
        if which is v:    # the other columns know nothing of it
            assert torch.isfinite(o[at:, 0, 2:].float()).all()
        which[at, 0, 1] = kept
    assert torch.equal(sbc.linear_attention_forward(q, k, v, rates, splits=sp), want)
