"""A cache in pages, and attention over it, on the GPU: places against a plain program, outputs
against plain float64 (tests/softmax_ref.py derives the tolerances)."""
import math

import numpy as np
import pytest
import torch

import paper_2012_01170_amd as sbc
from paper_2012_01170_amd import _lib as L
from tests import softmax_ref as S
from tests.test_gpu_softmax import BF16, DEV, F32, U, _close, _ints, _np, _rand, _splits

pytestmark = pytest.mark.gpu


def _cache(rng, lengths, page, hk, dk, dv, dtype, layout=0, room=1, spare=2):
    """Pages of random rows and a table for streams of these lengths"""
    held = [-(-int(n) // page) for n in lengths]
    width = max(held) + room
    n_pages = sum(held) + spare
    pages = []
    for d in (dk, dv):
        if layout == 0:
            x = _rand(rng, (n_pages, page, hk, d), dtype)
        elif layout == 1:  # a head's tokens behind each other
            x = _rand(rng, (n_pages, hk, page, d), dtype).transpose(1, 2)
        else:              # every second place of wider rows
            x = _rand(rng, (n_pages, 2, page, hk, d + 5), dtype)[:, 1, :, :, 1:1 + d]
        pages.append(x)
    order = rng.permutation(n_pages)
    table = np.full((len(lengths), width), -1, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    return pages, table, order[at:].astype(np.int32)


def _check(rng, lengths, new, page, hq, hk, dk, dv, dtype, layout=0, room=1):
    lengths, new = np.asarray(lengths), np.asarray(new)
    (kp, vp), table, _ = _cache(rng, lengths, page, hk, dk, dv, dtype, layout, room)
    splits = _splits(new)
    q = _rand(rng, (int(splits[-1]), hq, dk), dtype, 1.5)
    one = bool((new == 1).all())
    o = sbc.softmax_attention_paged(q, kp, vp, _ints(table), _ints(lengths),
                                    splits=None if one else _ints(splits))
    K, ks = S.gather_pages(_np(kp), table, lengths)
    V, _ = S.gather_pages(_np(vp), table, lengths)
    ro, _, to, _ = S.attention(_np(q), K, V, splits, ks, dk ** -0.5, True,
                               U[dtype] if dtype == BF16 else 0.0)
    _close(o, ro, to + U[dtype] * np.abs(ro), "o")


# kept with the new, new, page, heads, channels
PAGED = [
    ([1], [1], 16, 1, 1, 16, 16),
    ([4095], [1], 16, 8, 2, 128, 128),
    ([0, 5, 300, 64], [1, 1, 1, 1], 64, 4, 4, 64, 64),
    ([700, 1, 33], [1, 1, 1], 1, 12, 2, 64, 64),
    ([500, 31, 128], [1, 1, 1], 5, 3, 1, 40, 72),
    ([129, 200, 7, 0], [5, 0, 7, 0], 48, 6, 3, 33, 31),
    ([900, 300], [300, 299], 48, 4, 4, 64, 64),
    ([5000, 77], [2, 77], 256, 16, 1, 96, 96),
    ([20, 400], [40, 3], 16, 2, 1, 128, 64),     # more new tokens than the stream has
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", range(len(PAGED)))
def test_paged(case, dtype):
    print(f"[paged] {PAGED[case]} {dtype}", flush=True)
    _check(np.random.default_rng(case), *PAGED[case], dtype, layout=case % 3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
def test_paged_many_rows(d, dtype):
    """Enough new tokens for workgroups of 128 rows"""
    rng = np.random.default_rng(d)
    _check(rng, [700, 130, 1200, 66], [500, 130, 300, 65], 48, 32, 16, d, d, dtype)


def test_paged_wide_table():
    """A table with room for far more tokens than there are, and lengths past its room"""
    _check(np.random.default_rng(1), [50, 1000], [1, 1], 16, 4, 2, 64, 64, BF16, room=5000)
    rng = np.random.default_rng(2)
    (kp, vp), table, _ = _cache(rng, [64], 16, 1, 32, 32, F32, room=0)
    q = _rand(rng, (1, 1, 32))
    full, over = (sbc.softmax_attention_paged(q, kp, vp, _ints(table), _ints([n])) for n in (64, 900))
    assert torch.equal(full, over)
    none = sbc.softmax_attention_paged(q, kp, vp, _ints(table), _ints([-3]))
    assert not none.any()


@pytest.mark.parametrize("new,hq", [(1, 2), (150, 32)])
def test_pages_that_do_not_exist(new, hq):
    """Keys on pages outside the pool are left out; the others count, and NaN on pages of nobody
    or past a stream's end reach nothing."""
    rng = np.random.default_rng(3)
    lengths, page = [400, 260], 32
    (kp, vp), table, free = _cache(rng, lengths, page, 2 if hq == 2 else 16, 64, 64, F32)
    hk = kp.shape[2]
    n_pages = kp.shape[0]
    for x in (kp, vp):
        x[torch.from_numpy(free.astype(np.int64)).to(DEV)] = math.nan
        for b, n in enumerate(lengths):
            if n % page:
                x[int(table[b, n // page]), n % page:] = math.nan
    bad = table.copy()
    bad[0, 3], bad[0, 4], bad[1, 0] = -1, n_pages, 2 ** 31 - 1
    splits = _splits([new, new])
    q = _rand(rng, (2 * new, hq, 64))
    o = sbc.softmax_attention_paged(q, kp, vp, _ints(bad), _ints(lengths), splits=_ints(splits))
    K, ks = S.gather_pages(_np(kp), table, lengths)
    V, _ = S.gather_pages(_np(vp), table, lengths)
    keep = np.ones(len(K), bool)
    keep[3 * page:5 * page] = False
    keep[ks[1]:ks[1] + page] = False
    for b in range(2):
        for h in (0, hq - 1):
            for i in (0, new - 1):
                t, upto = int(splits[b]) + i, lengths[b] - new + i + 1
                rows = np.arange(ks[b], ks[b] + upto)
                rows = rows[keep[rows]]
                ro, _, to, _ = S.attention(_np(q)[t:t + 1, h:h + 1], K[rows][:, [h * hk // hq]],
                                           V[rows][:, [h * hk // hq]], [0, 1], [0, len(rows)], 0.125,
                                           False)
                _close(o[t:t + 1, h:h + 1], ro, to + U[F32] * np.abs(ro), "o")


def test_far_offsets():
    """Pages past 2^31 elements of the pool"""
    page, hk, d = 64, 2, 128
    n_pages = 2 ** 31 // (page * hk * d) + 40
    kp = torch.empty(n_pages, page, hk, d, dtype=BF16, device=DEV)
    vp = torch.empty(n_pages, page, hk, d, dtype=BF16, device=DEV)
    rng = np.random.default_rng(4)
    lengths = np.array([1000, 130])
    ids = np.concatenate([np.arange(n_pages - 16, n_pages), [2, n_pages - 30, 0]]).astype(np.int32)
    table = np.full((2, 16), -1, np.int32)
    table[0], table[1, :3] = ids[:16], ids[16:]
    where = torch.from_numpy(ids.astype(np.int64)).to(DEV)
    kp[where], vp[where] = (_rand(rng, (19, page, hk, d), BF16) for _ in range(2))
    # the last token of each stream appended far out
    k, v = (_rand(rng, (2, hk, d), BF16) for _ in range(2))
    free = torch.zeros(0, dtype=torch.int32, device=DEV)
    t2, slots, after, needed = sbc.cache_slots(_ints(lengths - 1), _ints(table), free, page)
    assert int(needed) == 0 and torch.equal(t2, _ints(table))
    sbc.cache_append(k, v, kp, vp, slots)
    assert torch.equal(kp[n_pages - 1, 999 % page], k[0]) and torch.equal(vp[0, 129 % page], v[1])
    q = _rand(rng, (2, 8, d), BF16)
    o = sbc.softmax_attention_paged(q, kp, vp, t2, after)
    small = {int(g): i for i, g in enumerate(ids)}
    local = np.vectorize(lambda g: small.get(int(g), -1))(table)
    K, ks = S.gather_pages(_np(kp[where]), local, lengths)
    V, _ = S.gather_pages(_np(vp[where]), local, lengths)
    ro, _, to, _ = S.attention(_np(q), K, V, [0, 1, 2], ks, d ** -0.5, True, U[BF16])
    _close(o, ro, to + U[BF16] * np.abs(ro), "o")


# ---------------------------------------------------------------- places
@pytest.mark.parametrize("page", [1, 5, 16, 256])
@pytest.mark.parametrize("b", [1, 7, 256, 1024, 1025, 5000])
def test_cache_slots(b, page):
    rng = np.random.default_rng(b + page)
    lengths = rng.integers(0, 40, b)
    new = rng.integers(0, 12, b)
    new[rng.integers(0, b)] = 60
    held = -(-lengths // page)
    after = -(-(lengths + new) // page)
    width = int(after.max()) + 1
    order = rng.permutation(int(after.sum()) + 3).astype(np.int32)
    table = np.full((b, width), -1, np.int32)
    at = 0
    for i in range(b):
        table[i, :held[i]] = order[at:at + held[i]]
        at += held[i]
    splits, free = _splits(new), order[at:]
    most = int((after - held).sum())
    for f, t in ((free, table), (free[:most // 2], table), (free[:0], table),
                 (free, table[:, :max(1, width // 2)].copy())):
        rt, rs, rl, rn = S.cache_slots(lengths, t, f, page, splits)
        for in_place in (False, True):
            dev = _ints(t)
            got = sbc.cache_slots(_ints(lengths), dev, _ints(f), page, splits=_ints(splits),
                                  n=int(splits[-1]), out_table=dev if in_place else None)
            assert (got[0].data_ptr() == dev.data_ptr()) == in_place
            assert np.array_equal(got[0].cpu().numpy(), rt)
            assert np.array_equal(got[1].cpu().numpy(), rs)
            assert np.array_equal(got[2].cpu().numpy(), rl) and int(got[3]) == rn
            if not in_place:
                assert torch.equal(dev, _ints(t))


def test_cache_slots_edges():
    """Tokens in no stream, no streams, a table without room"""
    free = _ints([4, 5, 6])
    t, s, n, need = sbc.cache_slots(_ints([3]), _ints([[0, -1]]), free, 4, splits=_ints([2, 4]), n=6)
    assert s.tolist() == [-1, -1, 3, 16, -1, -1] and t.tolist() == [[0, 4]] and int(need) == 1
    assert n.tolist() == [5]
    empty = torch.zeros(0, 3, dtype=torch.int32, device=DEV)
    t, s, n, need = sbc.cache_slots(_ints([]), empty, free, 4)
    assert t.shape == (0, 3) and s.numel() == 0 and int(need) == 0
    t, s, n, need = sbc.cache_slots(_ints([2, 9]), torch.zeros(2, 0, dtype=torch.int32, device=DEV),
                                    free, 4)
    assert s.tolist() == [-1, -1] and int(need) == 0 and n.tolist() == [3, 10]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk,dv,layout", [(64, 64, 0), (33, 31, 1), (40, 8, 2), (128, 100, 2)])
def test_cache_append(dk, dv, layout, dtype):
    rng = np.random.default_rng(dk)
    n, hk, page = 70, 3, 5
    (kp, vp), _, _ = _cache(rng, [100], page, hk, dk, dv, dtype, layout)
    wide = _rand(rng, (n, 2 * hk, dk + dv + 1), dtype)
    k, v = wide[:, :hk, 1:1 + dk], wide[:, hk:, 1 + dk:]
    total = kp.shape[0] * page
    slots = rng.permutation(total)[:n].astype(np.int64)
    slots[5], slots[6], slots[7] = -1, total, 2 ** 40
    want = []
    for x, rows in ((kp, k), (vp, v)):
        y = _np(x)
        for i, s in enumerate(slots):
            if 0 <= s < total:
                y[s // page, s % page] = _np(rows)[i]
        want.append(y)
    dev = torch.from_numpy(slots).to(DEV)
    first = kp.clone()
    sbc.cache_append(None, v, None, vp, dev)
    assert torch.equal(kp, first) and np.array_equal(_np(vp), want[1])
    sbc.cache_append(k, v, kp, vp, dev)
    assert np.array_equal(_np(kp), want[0]) and np.array_equal(_np(vp), want[1])


# ---------------------------------------------------------------- together
SECTIONS = (8, 4, 4)


def _layer(q, k, w, positions, freqs):
    return sbc.qk_norm_rotary_forward(q, k, w, w, positions, freqs, SECTIONS)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompt_then_tokens(dtype):
    """A layer over whole sequences, and the same in chunks and single tokens through the cache,
    captured into a graph for the tokens."""
    rng = np.random.default_rng(11)
    lens, hq, hk, d, page = [90, 41, 120], 4, 2, 64, 16
    n = sum(lens)
    splits = _splits(lens)
    positions = _ints(np.stack([np.arange(n) % 61, *rng.integers(0, 128, (2, n))], 1))
    freqs = torch.rand(16, device=DEV) + 0.01
    w = 1 + 0.2 * _rand(rng, (d,))
    q, k, v = _rand(rng, (n, hq, d), dtype), _rand(rng, (n, hk, d), dtype), _rand(rng, (n, hk, d), dtype)
    qr, kr = _layer(q, k, w, positions, freqs)
    whole, _ = sbc.softmax_attention_forward(qr, kr, v, splits=_ints(splits), causal=True)
    n_pages = 40
    kp, vp = (torch.full((n_pages, page, hk, d), math.nan, dtype=dtype, device=DEV) for _ in range(2))
    table = torch.full((3, 10), -1, dtype=torch.int32, device=DEV)
    lengths = torch.zeros(3, dtype=torch.int32, device=DEV)
    free = torch.randperm(n_pages, device=DEV).to(torch.int32)
    done = np.zeros(3, int)

    def rows_of(counts):
        return np.concatenate([np.arange(splits[b] + done[b], splits[b] + done[b] + c)
                               for b, c in enumerate(counts)])

    def step(x, splits, table, lengths, free, count):
        qs, ks = _layer(x[0], x[1], w, x[3], freqs)
        table, slots, lengths, needed = sbc.cache_slots(lengths, table, free, page, splits=splits,
                                                        n=count, out_table=table)
        sbc.cache_append(ks, x[2], kp, vp, slots)
        return sbc.softmax_attention_paged(qs, kp, vp, table, lengths, splits=splits), lengths, needed

    def check(o, rows):
        # both are off by what the references allow: weights, sums and the output's rounding
        a, b = o.float(), whole[torch.from_numpy(rows).to(DEV)].float()
        tol = 2.0 ** -15 if dtype == F32 else 2.0 ** -5
        assert bool(((a - b).abs() <= tol * (1 + b.abs())).all())

    for counts in ([80, 0, 100], [1, 37, 5]):
        r = rows_of(counts)
        i = torch.from_numpy(r).to(DEV)
        o, lengths, needed = step([q[i], k[i], v[i], positions[i]], _ints(_splits(counts)), table,
                                  lengths, free, len(r))
        free = free[int(needed):].contiguous()
        check(o, r)
        done += counts
    # single tokens: the call is captured once and replayed with the next token's inputs
    ins = [torch.empty(3, h, d, dtype=dtype, device=DEV) for h in (hq, hk, hk)]
    ins.append(torch.empty(3, 3, dtype=torch.int32, device=DEV))
    kept, pool = lengths.clone(), free.clone()
    graph = None
    for turn in range(4):
        r = rows_of([1, 1, 1])
        i = torch.from_numpy(r).to(DEV)
        for x, y in zip(ins, (q, k, v, positions)):
            x.copy_(y[i])
        if graph is None:
            state = kp.clone(), vp.clone(), table.clone()
            step(ins, None, table, kept, pool, None)  # (a first call, undone)
            for x, y in zip((kp, vp, table), state):
                x.copy_(y)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out, after, needed = step(ins, None, table, kept, pool, None)
        graph.replay()
        torch.cuda.synchronize()
        check(out, r)
        used = int(needed)
        kept.copy_(after)
        pool.copy_(torch.cat([pool[used:], pool[:used]]))
        done += 1


def test_refusals():
    kp = torch.zeros(4, 8, 2, 16, device=DEV)
    q, table, lens = torch.zeros(2, 4, 16, device=DEV), _ints([[0], [1]]), _ints([3, 4])
    f = sbc.softmax_attention_paged
    for bad in (lambda: f(q, kp[..., :8], kp, table, lens), lambda: f(q, kp, kp[:3], table, lens),
                lambda: f(q, kp, kp, table, lens[:1]), lambda: f(q[:1], kp, kp, table, lens),
                lambda: f(q, kp, kp, table.long(), lens), lambda: f(q, kp.to(BF16), kp, table, lens),
                lambda: f(q, kp, kp, table, lens, splits=_ints([0, 2])),
                lambda: sbc.cache_slots(lens, table[:1], lens, 8),
                lambda: sbc.cache_slots(lens, table, lens.long(), 8),
                lambda: sbc.cache_slots(lens, table, lens, 8, splits=_ints([0, 1, 2])),
                lambda: sbc.cache_slots(lens, table, lens, 8, out_table=_ints([[0, 1]])),
                lambda: sbc.cache_append(None, None, None, None, lens.long()),
                lambda: sbc.cache_append(q[:, :2], q[:, :2], kp, kp[:, :4], lens.long()),
                lambda: sbc.cache_append(q[:, :2], None, kp, kp, lens.long()),
                lambda: sbc.cache_append(q[:, :2], q[:, :2], kp, kp.clone(), lens)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: sbc.cache_slots(lens, table, lens, 0),
                lambda: f(q, kp, kp, table, lens, scale=-1.0),
                lambda: sbc.cache_append(q[:, :2], q[:, :2], kp, kp, lens.long()),
                lambda: sbc.cache_append(q[:, :2], None, kp[:1].expand(4, -1, -1, -1), None,
                                         lens.long())):
        with pytest.raises(L.SbcError):
            bad()
