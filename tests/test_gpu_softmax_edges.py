"""Softmax attention on the GPU where its arithmetic can go wrong: splits out of order, sizes next
to 2^31, values next to the largest, and the paths that only larger batches take."""
import ctypes

import math

import numpy as np
import pytest
import torch

import paper_2012_01170_amd as sbc
from paper_2012_01170_amd import _lib as L
from tests import softmax_ref as S
from tests.test_gpu_softmax import (BF16, DEV, F32, U, _check, _close, _inputs, _ints, _np, _rand,
                                     _splits)
from tests.test_gpu_softmax_cache import _cache, _check as _check_paged

pytestmark = pytest.mark.gpu


def _heads(x):
    return ctypes.byref(L.SbcHeads(x.data_ptr(), x.stride(0), x.stride(1)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,splits", [((2, 1), [0, 640, 0, 0, 0, 1000]),
                                          ((16, 8), [0, 900, 3, 0, 1000, 0, 700, 1000]),
                                          ((2, 2), [1000, 0, 2000, -5, 500])])
def test_splits_out_of_order(heads, splits, dtype):
    """Whatever the splits hold, no row in front of or behind the arrays is written."""
    print(f"[splits] {heads} {splits} {dtype}", flush=True)
    rng = np.random.default_rng(20)
    (hq, hk), n, d, edge = heads, 1000, 64, 300

    def guarded(h):
        return torch.full((n + 2 * edge, h, d), 5.0, dtype=dtype, device=DEV)

    q, do, k, v = (_rand(rng, (n, h, d), dtype) for h in (hq, hq, hk, hk))
    outs = [guarded(h) for h in (hq, hq, hk, hk)]
    o, dq, dk, dv = (x[edge:edge + n] for x in outs)
    lse_all = torch.full((n + 2 * edge, hq), 5.0, device=DEV)
    lse = lse_all[edge:edge + n]
    lib = L.lib()
    at = _ints(splits)
    for causal in (0, 1):
        a = L.SbcSoftmaxAttention(n, n, len(splits) - 1, hq, hk, d, d,
                                  L.SBC_F32 if dtype == F32 else L.SBC_BF16, 0.2, causal,
                                  at.data_ptr(), None)
        ref = ctypes.byref(a)
        size = max(lib.sbc_softmax_attention_workspace_size(ref),
                   lib.sbc_softmax_attention_backward_workspace_size(ref))
        # (rows that lie in no sequence leave their places in the workspace unwritten)
        ws = torch.zeros(size + 512, dtype=torch.uint8, device=DEV)
        stream = torch.cuda.current_stream().cuda_stream
        L.check(lib.sbc_softmax_attention_forward(ref, _heads(q), _heads(k), _heads(v), _heads(o),
                                                  lse.data_ptr(), ws.data_ptr(), size, stream))
        L.check(lib.sbc_softmax_attention_backward(
            ref, _heads(do), _heads(q), _heads(k), _heads(v), _heads(o), lse.data_ptr(), _heads(dq),
            _heads(dk), _heads(dv), ws.data_ptr(), size, stream))
        torch.cuda.synchronize()
        for x in (*outs, lse_all):
            assert bool((x[:edge] == 5).all()) and bool((x[edge + n:] == 5).all())
        assert not bool(ws[size:].any())


MOST = 2 ** 31 - 1024  # keys that a call takes


@pytest.mark.parametrize("m", [MOST])
def test_most_keys(m):
    """The same key and value over and over (stride 0): one row's lse counts them all.  A lane's
    sum is below 2^24 ones, and exact."""
    print(f"[most keys] {m}", flush=True)
    q = torch.full((1, 1, 16), 0.5, device=DEV, dtype=BF16)
    k = torch.full((1, 1, 16), 0.25, device=DEV, dtype=BF16).expand(m, 1, 16)
    v = torch.linspace(-1, 1, 17, device=DEV)[1:].to(BF16)[None, None].expand(m, 1, 16)
    o, lse = sbc.softmax_attention_forward(q, k, v, scale=1.0)
    want = 16 * 0.5 * 0.25 + math.log(m)
    # (float32's half unit of lse and of its parts, in units of log 2: 2^-19 each)
    assert abs(float(lse[0, 0]) - want) < 2.0 ** -17


@pytest.mark.parametrize("m", [1_500_000_000, 2_120_000_000, MOST])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_most_keys_values(m, dtype):
    """Their mean is the value itself: of each wave's sums (exact, of ones times a value of 8 bits)
    and their joins a few roundings are left, of 2^-24, and the output's."""
    print(f"[most keys, values] {m} {dtype}", flush=True)
    one = torch.full((1, 1, 16), 0.25, device=DEV, dtype=dtype)
    v = torch.linspace(-1, 1, 17, device=DEV)[1:].to(dtype)[None, None].expand(m, 1, 16)
    o, lse = sbc.softmax_attention_forward(2 * one, one.expand(m, 1, 16), v, scale=1.0)
    assert bool(((o - v[:1]).float().abs() <= 2.0 ** -20 * v[:1].float().abs()).all())
    assert abs(float(lse[0, 0]) - 2 - math.log(m)) < 2.0 ** -17


def test_most_kept_tokens():
    """A stream whose table names one page over and over"""
    page, width = 1 << 20, 1 << 11
    print(f"[most kept] {page} {width}", flush=True)
    k = torch.full((1, 1, 1, 16), 0.25, device=DEV, dtype=BF16).expand(1, page, 1, 16)
    v = torch.linspace(-1, 1, 17, device=DEV)[1:].to(BF16)[None, None, None].expand(1, page, 1, 16)
    q = torch.full((1, 1, 16), 0.5, device=DEV, dtype=BF16)
    table = torch.zeros((1, width), dtype=torch.int32, device=DEV)
    for n in (2_120_000_000, MOST, 2 ** 31 - 1):
        o = sbc.softmax_attention_paged(q, k, v, table, _ints([n]), scale=1.0)
        assert torch.equal(o, v[0, :1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", ["page", "token", "head", "heads first"])
def test_keys_and_values_in_one_pool(layout, dtype):
    """Appended to, and read, as caches of their own, bit by bit; other places keep what they held."""
    rng = np.random.default_rng(21)
    n_pages, page, g, d, lengths = 9, 16, 2, 64, [70, 37]
    shape = {"page": (n_pages, 2, page, g, d), "token": (n_pages, page, 2, g, d),
             "head": (n_pages, page, g, 2, d), "heads first": (n_pages, 2, g, page, d)}[layout]
    pool = torch.full((2, *shape), 5.0, dtype=dtype, device=DEV)
    kv = pool[0].unbind(shape.index(2))
    if layout == "heads first":
        kv = [x.transpose(1, 2) for x in kv]
    own = [torch.full((n_pages, page, g, d), 5.0, dtype=dtype, device=DEV) for _ in range(2)]
    table = torch.full((2, 5), -1, dtype=torch.int32, device=DEV)
    free = torch.randperm(n_pages, device=DEV).to(torch.int32)
    splits = _ints([0, *np.cumsum(lengths)])
    k, v = (_rand(rng, (sum(lengths), g, d), dtype) for _ in range(2))
    table, slots, after, _ = sbc.cache_slots(_ints([0, 0]), table, free, page, splits=splits,
                                             n=sum(lengths))
    for pages in (kv, own):
        sbc.cache_append(k, v, *pages, slots)
    for x, y in zip(kv, own):
        assert torch.equal(x, y)
    assert bool((pool[1] == 5).all())
    q = _rand(rng, (2, 4, d), dtype)
    assert torch.equal(sbc.softmax_attention_paged(q, *kv, table, after),
                       sbc.softmax_attention_paged(q, *own, table, after))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,n,paged", [((2, 1), 100, False), ((1, 1), 3000, False),
                                           ((32, 16), 600, False), ((2, 1), 300, True),
                                           ((32, 16), 600, True)])
def test_large_values(heads, n, paged, dtype):
    """Values up to the stated bound, 2^119 / keys, that rows see behind a tile of lower scores, whose
    maximum the weights refer to: a score 5.5 above it is a weight of 2^7.9."""
    print(f"[large values] {heads} {n} {paged} {dtype}", flush=True)
    rng = np.random.default_rng(22)
    (hq, hk), d = heads, 64
    new = n if hq > 2 else 3
    q = torch.zeros(new, hq, d, dtype=dtype, device=DEV)
    k = torch.zeros(n, hk, d, dtype=dtype, device=DEV)
    q[:, :, 0], k[64:, :, 0] = 1.0, 5.5
    v = (1 - 0.5 * torch.rand(n, hk, d, device=DEV)) * (2.0 ** 119 / n)
    v = (v * torch.where(_rand(rng, (1, hk, d)) > 0.5, -1.0, 1.0)).to(dtype)  # (nothing cancels)
    if paged:
        page = 32
        pages = [torch.zeros(-(-n // page), page, hk, d, dtype=dtype, device=DEV) for _ in range(2)]
        for x, y in zip((k, v), pages):
            y.view(-1, hk, d)[:n] = x
        table = torch.arange(len(pages[0]), dtype=torch.int32, device=DEV)[None].contiguous()
        o = sbc.softmax_attention_paged(q, *pages, table, _ints([n]), splits=_ints([0, new]), scale=1.0)
    else:
        o, _ = sbc.softmax_attention_forward(q, k, v, scale=1.0, causal=True)
    u = U[dtype] if dtype == BF16 else 0.0
    ro, _, to, _ = S.attention(_np(q), _np(k), _np(v), [0, new], [0, n], 1.0, True, u)
    _close(o, ro, to + U[dtype] * np.abs(ro), "o")


@pytest.mark.parametrize("lengths,new,page,heads,dk,dv", [
    ([1000, 5, 64, 0], [1, 1, 1, 1], 16, (8, 2), 128, 128), ([4095], [1], 48, (4, 4), 64, 64),
    ([300, 77], [16, 3], 5, (2, 1), 33, 31), ([40, 700], [8, 8], 64, (16, 2), 96, 40)])
def test_tokens_over_a_cache_are_rounded_once(lengths, new, page, heads, dk, dv):
    """bf16: weights have two parts of 8 bits there (2^-17), so o is as far from its exact value as
    float32 sums and its own rounding allow."""
    print(f"[rounded once] {lengths} {new} {heads} {dk} {dv}", flush=True)
    rng = np.random.default_rng(24)
    (kp, vp), table, _ = _cache(rng, lengths, page, heads[1], dk, dv, BF16)
    splits = _splits(new)
    q = _rand(rng, (int(splits[-1]), heads[0], dk), BF16, 1.5)
    o = sbc.softmax_attention_paged(q, kp, vp, _ints(table), _ints(lengths), splits=_ints(splits))
    K, ks = S.gather_pages(_np(kp), table, np.asarray(lengths))
    V, _ = S.gather_pages(_np(vp), table, np.asarray(lengths))
    ro, _, to, _ = S.attention(_np(q), K, V, splits, ks, dk ** -0.5, True, 2.0 ** -17)
    _close(o, ro, to + U[BF16] * np.abs(ro), "o")


# ---------------------------------------------------------------- batches that fill the card
# (Keys are in one part there: outputs are stored by the kernels that make the sums.)
FULL = 64  # sequences


def _lengths(rng, empty):
    lens = rng.integers(100, 230, FULL)
    lens[empty], lens[empty + 1] = 0, 1
    return lens


def _full_call(lq, heads, dk, dv, dtype, causal, lk=None):
    n = int(sum(lq))
    m = n if lk is None else int(sum(lk))
    return L.SbcSoftmaxAttention(n, m, FULL, *heads, dk, dv, L.SBC_F32 if dtype == F32 else L.SBC_BF16,
                                 dk ** -0.5, int(causal), 256, None if lk is None else 256)


def _one_part(a):
    """Whether the size queries tell of one part: no sums for the forward pass, and the backward's
    two numbers of each row alone, which it has where it takes more than one launch"""
    lib, rows = L.lib(), 4 * a.n * a.heads
    size = lib.sbc_softmax_attention_backward_workspace_size(ctypes.byref(a))
    return (lib.sbc_softmax_attention_workspace_size(ctypes.byref(a)) == 0
            and 2 * rows <= size <= 2 * rows + 1024)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,dk,dv", [((8, 8), 33, 33), ((8, 8), 40, 40), ((16, 8), 64, 64),
                                         ((8, 8), 96, 96), ((16, 8), 128, 128), ((8, 8), 128, 64),
                                         ((24, 8), 20, 24)])
def test_full_batches(heads, dk, dv, causal, dtype):
    print(f"[full] {heads} {dk} {dv} {causal} {dtype}", flush=True)
    rng = np.random.default_rng(dk + dv + causal)
    lq = _lengths(rng, 5)
    lk = None if causal else _lengths(rng, 30)
    assert _one_part(_full_call(lq, heads, dk, dv, dtype, causal, lk))
    n, m = int(sum(lq)), int(sum(lq if lk is None else lk))
    _check(*_inputs(rng, n, m, *heads, dk, dv, dtype), lq, lk, causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [64, 128])
def test_full_batches_of_views(d, dtype):
    """Rows off 16 bytes, with NaN between them: as contiguous ones, bit by bit"""
    rng = np.random.default_rng(d)
    lq = _lengths(rng, 0)
    n, splits = int(sum(lq)), _ints(_splits(lq))
    assert _one_part(_full_call(lq, (8, 8), d, d, dtype, True))
    wide = torch.full((n, 32, d + 3), math.nan, dtype=dtype, device=DEV)
    views = [wide[:, 8 * i:8 * i + 8, 1:1 + d] for i in range(4)]
    for x in views:
        x.copy_(_rand(rng, x.shape, dtype))

    def passes(q, k, v, do):
        o, lse = sbc.softmax_attention_forward(q, k, v, splits=splits, causal=True)
        return (o, lse, *sbc.softmax_attention_backward(do, q, k, v, o, lse, splits=splits, causal=True))

    for a, b in zip(passes(*views), passes(*(x.contiguous() for x in views))):
        assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_full_batches_leave_other_rows(dtype):
    rng = np.random.default_rng(23)
    lq, h, d = _lengths(rng, 9), 8, 64
    n = 7 + int(sum(lq)) + 30
    splits = _ints(7 + _splits(lq))
    a = _full_call(lq, (h, h), d, d, dtype, True)
    a.n, a.m, a.splits = n, n, splits.data_ptr()
    assert _one_part(a)
    q, k, v, do = _inputs(rng, n, n, h, h, d, d, dtype)
    o, dq, dk, dv = (torch.full_like(q, 5.0) for _ in range(4))
    lse = torch.full((n, h), 5.0, device=DEV)
    lib, ref = L.lib(), ctypes.byref(a)
    size = lib.sbc_softmax_attention_backward_workspace_size(ref)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    L.check(lib.sbc_softmax_attention_forward(ref, _heads(q), _heads(k), _heads(v), _heads(o),
                                              lse.data_ptr(), None, 0, stream))
    L.check(lib.sbc_softmax_attention_backward(
        ref, _heads(do), _heads(q), _heads(k), _heads(v), _heads(o), lse.data_ptr(), _heads(dq),
        _heads(dk), _heads(dv), ws.data_ptr(), size, stream))
    torch.cuda.synchronize()
    own = slice(7, n - 30)
    ro, rl = sbc.softmax_attention_forward(q[own], k[own], v[own], splits=_ints(_splits(lq)), causal=True)
    grads = sbc.softmax_attention_backward(do[own], q[own], k[own], v[own], ro, rl,
                                           splits=_ints(_splits(lq)), causal=True)
    for x, r in zip((o, lse, dq, dk, dv), (ro, rl, *grads)):
        assert bool((x[:7] == 5).all()) and bool((x[n - 30:] == 5).all())
        assert torch.equal(x[own], r)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,layout", [(33, 0), (40, 1), (64, 0), (64, 2), (96, 0), (128, 0), (128, 1)])
def test_full_batches_in_pages(d, layout, dtype):
    print(f"[full, paged] {d} {layout} {dtype}", flush=True)
    rng = np.random.default_rng(d + layout)
    new = _lengths(rng, 3)
    lengths = new + rng.integers(0, 90, FULL)
    page, heads = 48, (8, 8)
    a = _full_call(new, heads, d, d, dtype, True)
    width = int(-(-lengths.max() // page)) + 1
    assert L.lib().sbc_softmax_attention_paged_workspace_size(ctypes.byref(a), page, width) == 0
    assert a.n > 64 * FULL  # (workgroups of 128 rows)
    _check_paged(rng, lengths, new, page, *heads, d, d, dtype, layout)
