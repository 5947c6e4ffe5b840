"""Binding of the sequence operators: layer norm, rotary positions with several
axes, linear attention with a decay for each head.

As in ops.py, argument marshalling only.  Token arrays [n, heads, d] may be
views with any strides, as long as their last axis is dense (parts of one
projection, say); everything else is contiguous.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import _lib as L
from .ops import _dtype_code, _p, _require, _stream, _Workspace

_FLOATS = (torch.float32, torch.bfloat16)


def _require_view(t, name, dtype, ndim, device=None):
    """_require() for a view whose last axis is dense."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != ndim:
        raise ValueError(f"{name} must be {ndim}-D, got shape {tuple(t.shape)}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}'s last axis must be dense")
    # everything but the layout
    _require(t.as_strided((0,) * ndim, (1,) * ndim), name, dtype, ndim, device)
    return t


def _heads(t: Optional[torch.Tensor]):
    if t is None:
        return None
    return ctypes.byref(L.SbcHeads(t.data_ptr(), t.stride(0), t.stride(1)))


# ---------------------------------------------------------------- layer norm
def _norm_common(x, weight, name="x"):
    _require_view(x, name, _FLOATS, 2)
    if weight is not None:
        _require(weight, "weight", torch.float32, 1, x.device)
        if weight.numel() != x.shape[1]:
            raise ValueError(f"weight must be [{x.shape[1]}], got {tuple(weight.shape)}")
    return x.device, x.shape[0], x.shape[1]


def _row_stride(x):
    # (a single row's stride means nothing)
    return x.stride(0) if x.shape[0] > 1 else max(x.stride(0), x.shape[1])


def layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, stats: bool = True):
    """(y, mean, rstd) of x [n, C] float32 or bf16 over its channels
    (sbc_layer_norm_forward); mean and rstd [n] float32, which the backward
    reads, are None without stats."""
    dev, n, C = _norm_common(x, weight)
    if bias is not None:
        _require(bias, "bias", torch.float32, 1, dev)
        if bias.numel() != C:
            raise ValueError(f"bias must be [{C}], got {tuple(bias.shape)}")
    y = torch.empty((n, C), dtype=x.dtype, device=dev)
    mean = torch.empty(n, dtype=torch.float32, device=dev) if stats else None
    rstd = torch.empty(n, dtype=torch.float32, device=dev) if stats else None
    L.check(L.lib().sbc_layer_norm_forward(_p(x), _row_stride(x), _p(weight), _p(bias),
                                           _dtype_code(x), n, C, float(eps), _p(y), C, _p(mean),
                                           _p(rstd), _stream(dev)))
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, need_dx: bool = True,
                        need_dweight: bool = True, need_dbias: bool = True):
    """(dx, dweight, dbias) (sbc_layer_norm_backward): dx [n, C] of x's type,
    dweight and dbias [C] float32, None where not wanted."""
    dev, n, C = _norm_common(x, weight)
    _require_view(dy, "dy", x.dtype, 2, dev)
    if dy.shape != x.shape:
        raise ValueError(f"dy must be {tuple(x.shape)}, got {tuple(dy.shape)}")
    for name, s in (("mean", mean), ("rstd", rstd)):
        _require(s, name, torch.float32, 1, dev)
        if s.numel() != n:
            raise ValueError(f"{name} must be [{n}], got {tuple(s.shape)}")
    dx = torch.empty((n, C), dtype=x.dtype, device=dev) if need_dx else None
    dw = torch.empty(C, dtype=torch.float32, device=dev) if need_dweight else None
    db = torch.empty(C, dtype=torch.float32, device=dev) if need_dbias else None
    lib = L.lib()
    ws = _Workspace(lib.sbc_layer_norm_workspace_size(n, C), dev)
    L.check(lib.sbc_layer_norm_backward(_p(dy), _row_stride(dy), _p(x), _row_stride(x),
                                        _p(weight), _p(mean), _p(rstd), _dtype_code(x), n, C,
                                        _p(dx), C, _p(dw), _p(db), ws.ptr, ws.nbytes,
                                        _stream(dev)))
    return dx, dw, db


# ---------------------------------------------------------------- rotary positions
def _rotary(q, k, positions, freqs, sections, interleaved, backward, inplace):
    one = q if q is not None else k
    if one is None:
        raise ValueError("q or k is needed")
    _require_view(one, "q" if q is not None else "k", _FLOATS, 3)
    dev, n, d = one.device, one.shape[0], one.shape[2]
    for name, x in (("q", q), ("k", k)):
        if x is not None:
            _require_view(x, name, one.dtype, 3, dev)
            if x.shape[0] != n or x.shape[2] != d:
                raise ValueError(f"{name} must be [{n}, heads, {d}], got {tuple(x.shape)}")
    sections = [int(s) for s in sections]
    if not 1 <= len(sections) <= L.SBC_MAX_AXES:
        raise ValueError(f"1 .. {L.SBC_MAX_AXES} sections expected, got {len(sections)}")
    if min(sections) < 0:
        raise ValueError(f"sections must be >= 0, got {sections}")
    _require_view(positions, "positions", (torch.float32, torch.int32), 2, dev)
    if tuple(positions.shape) != (n, len(sections)):
        raise ValueError(f"positions must be [{n}, {len(sections)}], got {tuple(positions.shape)}")
    _require(freqs, "freqs", torch.float32, 1, dev)
    if freqs.numel() != sum(sections):
        raise ValueError(f"freqs must be [{sum(sections)}], got {tuple(freqs.shape)}")
    plan = L.SbcRotaryPlan(positions.data_ptr(), _row_stride(positions),
                           int(positions.dtype == torch.float32), freqs.data_ptr(), len(sections),
                           (ctypes.c_int32 * L.SBC_MAX_AXES)(*sections), int(interleaved))
    out = [None if x is None else (x if inplace else torch.empty(x.shape, dtype=x.dtype, device=dev))
           for x in (q, k)]
    L.check(L.lib().sbc_rotary(ctypes.byref(plan), _heads(q), 0 if q is None else q.shape[1],
                               _heads(k), 0 if k is None else k.shape[1], _dtype_code(one), n, d,
                               int(backward), _heads(out[0]), _heads(out[1]), _stream(dev)))
    return tuple(out)


def rotary_forward(q, k, positions, freqs, sections: Sequence[int], interleaved: bool = False,
                   inplace: bool = False):
    """q [n, heads, d] and k [n, k_heads, d] (either may be None) turned by their
    tokens' positions (sbc_rotary); returns both.

    positions [n, axes] float32 or int32; sections: the pairs of channels of
    each axis; freqs [sum(sections)] float32, the pairs' radians per unit.
    interleaved: pairs are channels (2 p, 2 p + 1), else (p, p + pairs).
    inplace: q and k themselves are overwritten."""
    return _rotary(q, k, positions, freqs, sections, interleaved, False, inplace)


def rotary_backward(dq, dk, positions, freqs, sections: Sequence[int], interleaved: bool = False,
                    inplace: bool = False):
    """The gradients of rotary_forward's q and k from those of its outputs."""
    return _rotary(dq, dk, positions, freqs, sections, interleaved, True, inplace)


# ---------------------------------------------------------------- linear attention
def _attention(q, k, v, rates, splits, t, scale, streams=False):
    _require_view(q, "q", _FLOATS, 3)
    dev, (n, H, dk) = q.device, q.shape
    _require_view(k, "k", q.dtype, 3, dev)
    _require_view(v, "v", q.dtype, 3, dev)
    if k.shape != q.shape:
        raise ValueError(f"k must be {tuple(q.shape)}, got {tuple(k.shape)}")
    if v.shape[:2] != q.shape[:2]:
        raise ValueError(f"v must be [{n}, {H}, dv], got {tuple(v.shape)}")
    _require(rates, "rates", torch.float32, 1, dev)
    if rates.numel() != H:
        raise ValueError(f"rates must be [{H}], got {tuple(rates.shape)}")
    n_batch = n if streams else 1
    if splits is not None:
        _require(splits, "splits", torch.int32, 1, dev)
        if splits.numel() < 1:
            raise ValueError("splits must be [n_batch + 1]")
        n_batch = splits.numel() - 1
    if t is not None:
        _require(t, "t", torch.int32, 1, dev)
        if t.numel() != n:
            raise ValueError(f"t must be [{n}], got {tuple(t.shape)}")
    d = lambda x: x.data_ptr() if x is not None else None  # noqa: E731
    a = L.SbcAttention(n, n_batch, H, dk, v.shape[2], _dtype_code(q), float(scale),
                       d(rates), d(splits), d(t))
    return dev, a


def _require_state(state, state_time, a, dev, with_times):
    shape = (a.n_batch, a.heads, a.dk, a.dv)
    if state is not None:
        _require(state, "state", torch.float32, 4, dev)
        if tuple(state.shape) != shape:
            raise ValueError(f"state must be {shape}, got {tuple(state.shape)}")
    if state_time is not None:
        _require(state_time, "state_time", torch.int32, 1, dev)
        if state_time.numel() != a.n_batch:
            raise ValueError(f"state_time must be [{a.n_batch}], got {tuple(state_time.shape)}")
    if state is not None and with_times and state_time is None:
        raise ValueError("state_time is needed beside state where t is given")
    return shape


def linear_attention_forward(q, k, v, rates, splits: Optional[torch.Tensor] = None,
                             t: Optional[torch.Tensor] = None, scale: float = 1.0,
                             state: Optional[torch.Tensor] = None,
                             state_time: Optional[torch.Tensor] = None,
                             return_state: bool = False):
    """o [n, heads, dv] of q, k [n, heads, dk] and v [n, heads, dv]
    (sbc_linear_attention_forward):

        o_i = scale * sum_{j <= i} exp(-rates[h] (t_i - t_j)) (q_i . k_j) v_j

    over the tokens of a sequence; splits [n_batch + 1] int32 cuts the tokens
    into sequences (None: one), t [n] int32 are their times (None: positions).
    state [n_batch, heads, dk, dv] and, with t, state_time [n_batch] are kept
    from earlier tokens.  With return_state: (o, state, state_time), which the
    next call or linear_attention_step goes on from (state_time None without
    t)."""
    dev, a = _attention(q, k, v, rates, splits, t, scale)
    shape = _require_state(state, state_time, a, dev, t is not None)
    o = torch.empty((a.n, a.heads, a.dv), dtype=q.dtype, device=dev)
    out = torch.empty(shape, dtype=torch.float32, device=dev) if return_state else None
    out_time = (torch.empty(a.n_batch, dtype=torch.int32, device=dev)
                if return_state and t is not None else None)
    lib = L.lib()
    ws = _Workspace(lib.sbc_linear_attention_workspace_size(a.n, a.heads, a.dk, a.dv), dev)
    L.check(lib.sbc_linear_attention_forward(
        ctypes.byref(a), _heads(q), _heads(k), _heads(v), _p(state),
        _p(state_time if t is not None else None), _heads(o), _p(out), _p(out_time), ws.ptr,
        ws.nbytes, _stream(dev)))
    return (o, out, out_time) if return_state else o


def linear_attention_backward(do, q, k, v, rates, splits: Optional[torch.Tensor] = None,
                              t: Optional[torch.Tensor] = None, scale: float = 1.0,
                              need_rates: bool = True):
    """(dq, dk, dv, drates) for sequences that start from zero
    (sbc_linear_attention_backward); drates [heads] float32, None where not
    wanted."""
    dev, a = _attention(q, k, v, rates, splits, t, scale)
    _require_view(do, "do", q.dtype, 3, dev)
    if do.shape != v.shape:
        raise ValueError(f"do must be {tuple(v.shape)}, got {tuple(do.shape)}")
    dq, dk, dv = (torch.empty(x.shape, dtype=q.dtype, device=dev) for x in (q, k, v))
    dr = torch.empty(a.heads, dtype=torch.float32, device=dev) if need_rates else None
    lib = L.lib()
    ws = _Workspace(lib.sbc_linear_attention_backward_workspace_size(a.n, a.heads, a.dk, a.dv),
                    dev)
    L.check(lib.sbc_linear_attention_backward(
        ctypes.byref(a), _heads(do), _heads(q), _heads(k), _heads(v), _heads(dq), _heads(dk),
        _heads(dv), _p(dr), ws.ptr, ws.nbytes, _stream(dev)))
    return dq, dk, dv, dr


def linear_attention_step(q, k, v, rates, state, t: Optional[torch.Tensor] = None,
                          state_time: Optional[torch.Tensor] = None, scale: float = 1.0,
                          out_state: Optional[torch.Tensor] = None,
                          out_time: Optional[torch.Tensor] = None):
    """One token for each of n streams: (o [n, heads, dv], state, state_time)
    (sbc_linear_attention_step).  The new state is written to out_state, which
    may be state itself (default: a new tensor), and with t the new times to
    out_time (not state_time itself)."""
    dev, a = _attention(q, k, v, rates, None, t, scale, streams=True)
    shape = _require_state(state, state_time, a, dev, t is not None)
    if state is None:
        raise ValueError("state is needed")
    _require_state(out_state, out_time, a, dev, False)
    o = torch.empty((a.n, a.heads, a.dv), dtype=q.dtype, device=dev)
    if out_state is None:
        out_state = torch.empty(shape, dtype=torch.float32, device=dev)
    if t is None:
        out_time = None
    elif out_time is None:
        out_time = torch.empty(a.n, dtype=torch.int32, device=dev)
    L.check(L.lib().sbc_linear_attention_step(
        ctypes.byref(a), _heads(q), _heads(k), _heads(v), _p(state),
        _p(state_time if t is not None else None), _heads(o), _p(out_state), _p(out_time),
        _stream(dev)))
    return o, out_state, out_time
