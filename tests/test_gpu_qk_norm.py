"""Norms of queries and keys with the rotation on the GPU against plain float64
(tests/softmax_ref.py).

Tolerances: a mean square of up to 256 float32 terms and its root are off by less than 2^-20, an
output by that of its pair's two terms, and bf16 outputs by half a unit, 2^-8, more; gradients
by 2^-19 of their terms' magnitudes, as the layer norm's."""
import math

import numpy as np
import pytest
import torch

import paper_2012_01170_amd as sbc
from paper_2012_01170_amd import _lib as L
from tests import softmax_ref as S
from tests.test_gpu_softmax import BF16, DEV, F32, _close, _np, _rand

pytestmark = pytest.mark.gpu

EPS = 1e-5
# tokens, heads, key heads, channels, sections
SHAPES = [(1, 1, 1, 2, (1,)), (3, 2, 1, 16, (3, 2, 2)), (70, 4, 4, 64, (16, 8, 8)),
          (33, 8, 2, 96, (11, 11, 10)), (257, 3, 1, 33, (5, 4, 3)), (19, 2, 2, 256, (64, 64)),
          (40, 1, 5, 128, (1, 0, 7)), (5, 2, 0, 40, (20,)), (9, 0, 3, 7, (1, 1)),
          (1, 16, 1, 240, (1,)), (3001, 2, 1, 80, (20, 10))]


def _make(rng, n, d, sections, dtype, hq, hk, ints):
    axes = len(sections)
    if ints:
        positions = torch.from_numpy(rng.integers(-10 ** 6, 10 ** 6, (n, axes)).astype(np.int32)).to(DEV)
    else:
        positions = _rand(rng, (n, axes), F32, 100.0)
    freqs = _rand(rng, (sum(sections),)).abs() + 1e-3
    x = [_rand(rng, (n, h, d), dtype, 2.0) if h else None for h in (hq, hk)]
    dy = [_rand(rng, (n, h, d), dtype) if h else None for h in (hq, hk)]
    w = [1 + 0.3 * _rand(rng, (d,)) for _ in range(2)]
    return positions, freqs, x, dy, w


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_qk_norm_rotary(shape, interleaved, dtype):
    print(f"[qk norm] {shape} {interleaved} {dtype}", flush=True)
    n, hq, hk, d, sections = shape
    rng = np.random.default_rng(n + d)
    for ints, weights in ((True, True), (False, False)):
        positions, freqs, x, dy, w = _make(rng, n, d, sections, dtype, hq, hk, ints)
        ww = w if weights else [None, None]
        args = (*ww, positions, freqs, sections)
        y = sbc.qk_norm_rotary_forward(*x, *args, interleaved=interleaved, eps=EPS)
        g = sbc.qk_norm_rotary_backward(*dy, *x, *args, interleaved=interleaved, eps=EPS)
        u = 2.0 ** -8 if dtype == BF16 else 0.0
        for i in range(2):
            if x[i] is None:
                assert y[i] is None and g[i] is None and g[2 + i] is None
                continue
            wn = None if ww[i] is None else _np(ww[i])
            pn = positions.cpu().numpy().astype(np.float64)
            ry, size = S.qk_norm(_np(x[i]), wn, pn, _np(freqs), sections, interleaved, EPS)
            _close(y[i], ry, 2.0 ** -20 * size + u * np.abs(ry), "y")
            rdx, rdw, sx, sw = S.qk_norm_grad(_np(dy[i]), _np(x[i]), wn, pn, _np(freqs), sections,
                                              interleaved, EPS)
            _close(g[i], rdx, 2.0 ** -19 * sx + u * np.abs(rdx), "dx")
            _close(g[2 + i], rdw, 2.0 ** -19 * sw, "dw")
            assert y[i].dtype == dtype and g[2 + i].dtype == F32


def test_against_norm_and_rotation():
    """Zero rows, rows far below eps, and without rotation the norm alone; in place."""
    rng = np.random.default_rng(1)
    positions, freqs, x, dy, w = _make(rng, 50, 64, (16, 16), F32, 4, 2, False)
    x[0][3] = 0
    x[0][4] *= 1e-20
    zero = torch.zeros_like(positions)
    y, _ = sbc.qk_norm_rotary_forward(x[0], x[1], *w, zero, freqs, (16, 16))
    ref = (x[0].double() / (x[0].double().pow(2).mean(-1, keepdim=True) + 1e-5).sqrt()
           * w[0].double())
    assert bool(((y - ref).abs() <= 2.0 ** -20 * ref.abs()).all())
    q, k = sbc.qk_norm_rotary_forward(*x, *w, positions, freqs, (16, 16))
    a, b = x[0].clone(), x[1].clone()
    q2, k2 = sbc.qk_norm_rotary_forward(a, b, *w, positions, freqs, (16, 16), inplace=True)
    assert q2 is a and torch.equal(a, q) and torch.equal(b, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_views_and_repeats(dtype):
    """Parts of one projection at odd offsets, NaN between; the sums repeat; many tokens"""
    rng = np.random.default_rng(2)
    n, d = 20_011, 48
    wide = torch.full((n, 5, d + 3), math.nan, dtype=dtype, device=DEV)
    q, k = wide[:, :3, 1:1 + d], wide[:, 3:4, 3:3 + d]
    for x in (q, k):
        x.copy_(_rand(rng, x.shape, dtype))
    positions, freqs, _, dy, w = _make(rng, n, d, (8, 8), dtype, 3, 1, True)
    c = q.contiguous(), k.contiguous()
    args = (*w, positions, freqs, (8, 8))
    for a, b in zip(sbc.qk_norm_rotary_forward(q, k, *args), sbc.qk_norm_rotary_forward(*c, *args)):
        assert torch.equal(a, b)
    g = sbc.qk_norm_rotary_backward(*dy, q, k, *args)
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(g, sbc.qk_norm_rotary_backward(*dy, *c, *args)))
    part = sbc.qk_norm_rotary_backward(*dy, q, k, *args, need_weights=False)
    assert part[2] is None and torch.equal(part[0], g[0])
    pn = positions.cpu().numpy().astype(np.float64)
    _, rdw, _, sw = S.qk_norm_grad(_np(dy[0]), _np(q), _np(w[0]), pn, _np(freqs), (8, 8), False, EPS)
    _close(g[2], rdw, 2.0 ** -19 * sw, "dw")


def test_no_tokens():
    positions, freqs = torch.zeros(0, 1, device=DEV), torch.ones(4, device=DEV)
    x = torch.zeros(0, 2, 8, device=DEV)
    w = torch.ones(8, device=DEV)
    q, k = sbc.qk_norm_rotary_forward(x, x.clone(), w, w, positions, freqs, (4,))
    assert q.shape == (0, 2, 8)
    g = sbc.qk_norm_rotary_backward(x, x, x, x, w, w, positions, freqs, (4,))
    assert not g[2].any() and not g[3].any()


def test_gradients_against_differences():
    rng = np.random.default_rng(3)
    positions, freqs, (x, _), (dy, _), (w, _) = _make(rng, 40, 32, (8, 4), F32, 3, 1, False)
    f = lambda x, w: float((sbc.qk_norm_rotary_forward(  # noqa: E731
        x, None, w, None, positions, freqs, (8, 4))[0].double() * dy.double()).sum())
    dx, _, dw, _ = sbc.qk_norm_rotary_backward(dy, None, x, None, w, None, positions, freqs, (8, 4))
    h = 2.0 ** -8
    for i, g in enumerate((dx, dw)):
        d = _rand(rng, g.shape)
        up, down = (f(x + s * h * d, w) if i == 0 else f(x, w + s * h * d) for s in (1, -1))
        got = float((g.double() * d.double()).sum())
        # h^2 of third derivatives, of the order of the terms, and 2^-20 of <y, dy> over h
        assert abs(got - (up - down) / (2 * h)) < 2.0 ** -10 * (1 + float((g * d).abs().sum()))


def test_graph():
    rng = np.random.default_rng(4)
    positions, freqs, x, dy, w = _make(rng, 300, 64, (16, 8), BF16, 4, 2, True)
    args = (*w, positions, freqs, (16, 8))
    run = lambda: (*sbc.qk_norm_rotary_forward(*x, *args),  # noqa: E731
                   *sbc.qk_norm_rotary_backward(*dy, *x, *args))
    want = run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(3):
        graph.replay()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    x, w = torch.zeros(5, 2, 16, device=DEV), torch.zeros(16, device=DEV)
    p, fr = torch.zeros(5, 1, device=DEV), torch.zeros(8, device=DEV)
    f, b = sbc.qk_norm_rotary_forward, sbc.qk_norm_rotary_backward
    for bad in (lambda: f(None, None, w, w, p, fr, (8,)), lambda: f(x, x, w[:8], w, p, fr, (8,)),
                lambda: f(x, x.to(BF16), w, w, p, fr, (8,)), lambda: f(x, x, w, w, p, fr, (7,)),
                lambda: f(x, x, w, w.to(BF16), p, fr, (8,)), lambda: f(x, x, w, w, p[:4], fr, (8,)),
                lambda: b(x, None, x, x, w, w, p, fr, (8,)),
                lambda: b(x[:4], x, x, x, w, w, p, fr, (8,))):
        with pytest.raises(ValueError):
            bad()
    wide = torch.zeros(2, 1, 258, device=DEV)
    for bad in (lambda: f(x, None, w, None, p, fr, (8,), eps=-1.0),
                lambda: f(x, x, w, w, p, fr, (8,), inplace=True),
                lambda: f(wide, None, None, None, p[:2], fr, (8,))):
        with pytest.raises(L.SbcError):
            bad()
