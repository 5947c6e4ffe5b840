"""The sequence operators written plainly in float64 (numpy), and the sums of
their terms' magnitudes, from which the tests' tolerances are derived."""
import numpy as np


# ---------------------------------------------------------------- layer norm
def layer_norm(x, w, b, eps):
    x = x.astype(np.float64)
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1 / np.sqrt(var + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if w is not None:
        y = y * w.astype(np.float64)
    if b is not None:
        y = y + b.astype(np.float64)
    return y, mean, rstd


def layer_norm_grad(dy, x, w, mean, rstd):
    dy, x = dy.astype(np.float64), x.astype(np.float64)
    mean, rstd = mean.astype(np.float64)[:, None], rstd.astype(np.float64)[:, None]
    xn = (x - mean) * rstd
    g = dy if w is None else dy * w.astype(np.float64)
    dx = rstd * (g - g.mean(1, keepdims=True) - xn * (g * xn).mean(1, keepdims=True))
    return dx, (dy * xn).sum(0), dy.sum(0)


# ---------------------------------------------------------------- rotary positions
def rotary(x, positions, freqs, sections, interleaved, sign=1.0):
    x = x.astype(np.float64)
    axis = np.repeat(np.arange(len(sections)), sections)
    m = axis.size
    angle = sign * positions.astype(np.float64)[:, axis] * freqs.astype(np.float64)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    i = np.arange(m)
    u, v = (2 * i, 2 * i + 1) if interleaved else (i, i + m)
    y = x.copy()
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., v] * c + x[..., u] * s
    return y


# ---------------------------------------------------------------- linear attention
def _decays(rate, t):
    """exp(-rate (t_i - t_j)) for j <= i, else 0, and the gaps"""
    gap = t[:, None] - t[None, :]
    low = np.tril(np.ones(gap.shape, bool))
    return np.where(low, np.exp(-rate * np.where(low, gap, 0.0)), 0.0), np.where(low, gap, 0.0)


def _times(t, lo, hi):
    return np.arange(lo, hi, dtype=np.float64) if t is None else t[lo:hi].astype(np.float64)


def attention(q, k, v, rates, splits, t, scale, state=None, state_time=None):
    """(o, state, state_time, size): size is o with every term's magnitude"""
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    H, dk, dv = q.shape[1], q.shape[2], v.shape[2]
    B = len(splits) - 1
    o, size = np.zeros(v.shape), np.zeros(v.shape)
    S = np.zeros((B, H, dk, dv)) if state is None else state.astype(np.float64).copy()
    T = np.zeros(B) if state_time is None else state_time.astype(np.float64).copy()
    for b in range(B):
        lo, hi = int(splits[b]), int(splits[b + 1])
        if lo == hi:
            continue
        tt = _times(t, lo, hi)
        t0 = tt[0] if state is None else (lo - 1.0 if t is None else T[b])
        for h in range(H):
            r = float(rates[h])
            D, _ = _decays(r, tt)
            e = np.exp(-r * (tt - t0))[:, None]
            Q, K, V = q[lo:hi, h], k[lo:hi, h], v[lo:hi, h]
            o[lo:hi, h] = scale * ((Q @ K.T * D) @ V + e * (Q @ S[b, h]))
            size[lo:hi, h] = abs(scale) * ((abs(Q) @ abs(K).T * D) @ abs(V)
                                           + e * (abs(Q) @ abs(S[b, h])))
            w = np.exp(-r * (tt[-1] - tt))[:, None]
            S[b, h] = np.exp(-r * (tt[-1] - t0)) * S[b, h] + (K * w).T @ V
        T[b] = tt[-1]
    return o, S, T, size


def attention_grad(do, q, k, v, rates, splits, t, scale):
    """(dq, dk, dv, drates) and the same with every term's magnitude; the last of these
    also as the sum of the magnitudes without their gaps"""
    do, q, k, v = (x.astype(np.float64) for x in (do, q, k, v))
    H = q.shape[1]
    out = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(H)]
    size = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(H)]
    total = np.zeros(H)
    for b in range(len(splits) - 1):
        lo, hi = int(splits[b]), int(splits[b + 1])
        tt = _times(t, lo, hi)
        for h in range(H):
            D, gap = _decays(float(rates[h]), tt)
            for into, f in ((out, lambda x: x), (size, abs)):
                Q, K, V, G = (f(x[lo:hi, h]) for x in (q, k, v, do))
                s = f(scale)
                A, B = s * (Q @ K.T) * D, s * (G @ V.T) * D
                into[0][lo:hi, h] = B @ K
                into[1][lo:hi, h] = B.T @ Q
                into[2][lo:hi, h] = A.T @ G
                P = A * (G @ V.T)
                into[3][h] += (P * gap).sum() * (-1 if into is out else 1)
                if into is size:
                    total[h] += P.sum()
    return out, size, total
