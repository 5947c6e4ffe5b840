"""Softmax attention, norms with the rotation, and a cache in pages written plainly in
float64 (numpy), with the sums of their terms' magnitudes, from which the tests' tolerances
are derived."""
import numpy as np

from tests import sequence_ref as R


# ---------------------------------------------------------------- norms and rotation
def qk_norm(x, w, positions, freqs, sections, interleaved, eps):
    """y, and the magnitude of each output's two terms"""
    x = x.astype(np.float64)
    rstd = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    z = x * rstd * (1 if w is None else w.astype(np.float64))
    y = R.rotary(z, positions, freqs, sections, interleaved)
    return y, _pair_sums(np.abs(z), len_pairs(sections), interleaved)


def len_pairs(sections):
    return int(np.sum(sections))


def _pair_sums(a, m, interleaved):
    i = np.arange(m)
    u, v = (2 * i, 2 * i + 1) if interleaved else (i, i + m)
    out = a.copy()
    out[..., u] = out[..., v] = a[..., u] + a[..., v]
    return out


def qk_norm_grad(dy, x, w, positions, freqs, sections, interleaved, eps):
    """dx, dw, and their terms' magnitudes"""
    dy, x = dy.astype(np.float64), x.astype(np.float64)
    w = np.ones(x.shape[-1]) if w is None else w.astype(np.float64)
    rstd = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xn = x * rstd
    g = R.rotary(dy, positions, freqs, sections, interleaved, -1.0)
    dx = rstd * (g * w - xn * (g * w * xn).mean(-1, keepdims=True))
    a = _pair_sums(np.abs(dy), len_pairs(sections), interleaved)
    size = rstd * (a * np.abs(w) + np.abs(xn) * (a * np.abs(w * xn)).mean(-1, keepdims=True))
    return dx, (g * xn).sum((0, 1)), size, (a * np.abs(xn)).sum((0, 1))


# ---------------------------------------------------------------- attention
# A weight below the least normal float32 is zero, and an operand's three parts of bf16 keep
# multiples of 2^-133 of it: each weight is off by up to 2^-126 and 2^-133 besides what its size
# allows, which only shows where a whole sum is that small.
TINY = 2.0 ** -125


def visible(lq, lk, causal):
    """[lq, lk]: the last query sees the last key"""
    if not causal:
        return np.ones((lq, lk), bool)
    return np.arange(lk)[None, :] <= np.arange(lq)[:, None] + lk - lq


def _scores(q, k, scale, seen):
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    return s, np.where(seen, scale * (np.abs(q) @ np.abs(k).T), 0.0)


def attention(q, k, v, splits, k_splits, scale, causal, u=0.0):
    """(o, lse, tol_o, tol_lse).  Tolerances for float32 arithmetic: scores off by 2^-18 of
    their terms' magnitudes (products split to 2^-22, sums of up to 2^8 roundings of 2^-24 most of
    which cancel), weights by 2^-20 (1 + |s| + |lse|) more (the exponent's roundings), sums
    by 2^-18; and weights rounded to half a unit u on their way to the product with v."""
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    n, H, _ = q.shape
    group = H // k.shape[1]
    o, lse = np.zeros((n, H, v.shape[2])), np.full((n, H), -np.inf)
    tol_o, tol_lse = np.zeros(o.shape), np.zeros(lse.shape)
    for a, b, c, d in zip(splits, splits[1:], k_splits, k_splits[1:]):
        a, b, c, d = int(a), int(b), int(c), int(d)
        if a == b or c == d:
            continue
        seen = visible(b - a, d - c, causal)
        some = seen.any(1)
        for h in range(H):
            V = v[c:d, h // group]
            s, size = _scores(q[a:b, h], k[c:d, h // group], scale, seen)
            top = np.where(some, s.max(1), 0.0)
            e = np.exp(s - top[:, None])
            total = np.where(some, e.sum(1), 1.0)
            p = e / total[:, None]
            lse[a:b, h] = np.where(some, top + np.log(total), -np.inf)
            o[a:b, h] = p @ V
            l0 = np.where(some, lse[a:b, h], 0.0)
            rel = 2.0 ** -18 * size + 2.0 ** -20 * (1 + np.abs(np.where(seen, s, 0.0))
                                                    + np.abs(l0)[:, None])
            pr = p * rel
            tol_lse[a:b, h] = pr.sum(1) + 2.0 ** -20 * (1 + np.abs(l0))
            tol_o[a:b, h] = (pr @ np.abs(V) + pr.sum(1)[:, None] * np.abs(o[a:b, h])
                             + (2.0 ** -18 + u) * (p @ np.abs(V)) + TINY * (seen @ np.abs(V)))
    return o, lse, tol_o, tol_lse


def attention_grad(do, q, k, v, o, lse, splits, k_splits, scale, causal, u=0.0):
    """((dq, dk, dv), their tolerances) from the given o and lse; tolerances as above, dO v and
    dO o off by 2^-18 of their terms' magnitudes; weights rounded to u, and their gradients, in
    two parts where those are, to 2^-16."""
    do, q, k, v, o, lse = (x.astype(np.float64) for x in (do, q, k, v, o, lse))
    H = q.shape[1]
    group = H // k.shape[1]
    us = 2.0 ** -16 if u else 0.0
    out = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    tol = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    for a, b, c, d in zip(splits, splits[1:], k_splits, k_splits[1:]):
        a, b, c, d = int(a), int(b), int(c), int(d)
        if a == b or c == d:
            continue
        seen = visible(b - a, d - c, causal)
        for h in range(H):
            g = h // group
            Q, K, V, G, O = q[a:b, h], k[c:d, g], v[c:d, g], do[a:b, h], o[a:b, h]
            s, size = _scores(Q, K, scale, seen)
            ls = np.where(np.isfinite(lse[a:b, h]), lse[a:b, h], 0.0)[:, None]
            p = np.where(seen, np.exp(s - ls), 0.0)
            ds = p * (G @ V.T - (G * O).sum(1, keepdims=True))
            mag = p * (np.abs(G) @ np.abs(V).T + np.abs(G * O).sum(1, keepdims=True))
            rel = 2.0 ** -18 * size + 2.0 ** -20 * (1 + np.abs(np.where(seen, s, 0.0)) + np.abs(ls))
            full = seen * (np.abs(G) @ np.abs(V).T + np.abs(G * O).sum(1, keepdims=True) + 1)
            err = np.abs(ds) * (rel + us) + mag * (2.0 ** -18 + rel * us) + TINY * full
            out[0][a:b, h] += scale * ds @ K
            out[1][c:d, g] += scale * ds.T @ Q
            out[2][c:d, g] += p.T @ G
            err += 2.0 ** -18 * np.abs(ds)  # the sums
            tol[0][a:b, h] += scale * err @ np.abs(K)
            tol[1][c:d, g] += scale * err.T @ np.abs(Q)
            tol[2][c:d, g] += (p * (rel + u + 2.0 ** -18) + TINY * seen).T @ np.abs(G)
    return out, tol


# ---------------------------------------------------------------- a cache in pages
def cache_slots(lengths, table, free, page, splits):
    """One stream after another: (table, slots, lengths, needed)"""
    table, free = table.copy(), list(free)
    width, slots, needed = table.shape[1], [], 0
    for b, n in enumerate(lengths):
        held = min(-(-int(n) // page), width)
        upto = min(-(-(int(n) + int(splits[b + 1] - splits[b])) // page), width)
        for j in range(held, upto):
            table[b, j] = free.pop(0) if free else -1
            needed += 1
        for i in range(int(splits[b + 1] - splits[b])):
            pos = int(n) + i
            g = table[b, pos // page] if pos // page < width else -1
            slots.append(int(g) * page + pos % page if g >= 0 else -1)
    return table, np.array(slots, np.int64), lengths + np.diff(splits), needed


def gather_pages(pages, table, lengths):
    """The kept rows of all streams behind each other, and their splits"""
    page = pages.shape[1]
    rows = [pages[table[b, :-(-int(n) // page)]].reshape(-1, *pages.shape[2:])[:int(n)]
            for b, n in enumerate(lengths)]
    return np.concatenate(rows), np.concatenate([[0], np.cumsum(lengths)]).astype(int)
