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
from .ops import _dtype_code, _require, _Workspace

_FLOATS = (torch.float32, torch.bfloat16)

# The checks are those of ops._require, which words the errors.  A call on a single
# token costs little more than its checks, so a tensor that passes them is let through
# by one expression.


def _dense(t, name, dtype, ndim, index):
    """A contiguous tensor on device `index`."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == index
            and t.dim() == ndim and t.is_contiguous()):
        _require(t, name, dtype, ndim, torch.device("cuda", index))
    return t


def _view(t, name, dtype, ndim, index):
    """A view with any strides whose last axis is dense (dtype may be several)."""
    if isinstance(t, torch.Tensor) and t.dim() == ndim and t.get_device() == index \
            and (t.dtype is dtype or dtype is _FLOATS and t.dtype in _FLOATS) \
            and (t.is_contiguous() or t.stride(-1) == 1 or t.shape[-1] <= 1):
        return t
    if isinstance(t, torch.Tensor) and t.dim() == ndim and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}'s last axis must be dense")
    _require(t[:0].contiguous() if isinstance(t, torch.Tensor) and t.dim() == ndim else t, name,
             dtype, ndim, None if index is None else torch.device("cuda", index))
    return t


def _first(t, name, ndim):
    """The view that says which device and type the others have."""
    index = t.get_device() if isinstance(t, torch.Tensor) else -1
    return _view(t, name, _FLOATS, ndim, index if index >= 0 else None)


def _stream(index):
    # torch.cuda.current_stream(index).cuda_stream, without the Stream object (1.5 us)
    return torch._C._cuda_getCurrentRawStream(index)


def _ptr(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


def _heads(t: Optional[torch.Tensor]):
    if t is None:
        return None
    s = t.stride()
    return ctypes.byref(L.SbcHeads(t.data_ptr(), s[0], s[1]))


# ---------------------------------------------------------------- layer norm
def _norm_common(x, weight):
    _first(x, "x", 2)
    index, (n, C) = x.get_device(), x.shape
    if weight is not None:
        _dense(weight, "weight", torch.float32, 1, index)
        if weight.numel() != C:
            raise ValueError(f"weight must be [{C}], got {tuple(weight.shape)}")
    return index, x.device, n, C


def _row_stride(x):
    # (a single row's stride means nothing)
    return x.stride(0) if x.shape[0] > 1 else max(x.stride(0), x.shape[1])


def layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, stats: bool = True):
    """(y, mean, rstd) of x [n, C] float32 or bf16 over its channels
    (sbc_layer_norm_forward); mean and rstd [n] float32, which the backward
    reads, are None without stats."""
    index, dev, n, C = _norm_common(x, weight)
    if bias is not None:
        _dense(bias, "bias", torch.float32, 1, index)
        if bias.numel() != C:
            raise ValueError(f"bias must be [{C}], got {tuple(bias.shape)}")
    y = torch.empty((n, C), dtype=x.dtype, device=dev)
    mean = torch.empty(n, dtype=torch.float32, device=dev) if stats else None
    rstd = torch.empty(n, dtype=torch.float32, device=dev) if stats else None
    L.check(L.lib().sbc_layer_norm_forward(x.data_ptr(), _row_stride(x), _ptr(weight), _ptr(bias),
                                           _dtype_code(x), n, C, float(eps), y.data_ptr(), C,
                                           _ptr(mean), _ptr(rstd), _stream(index)))
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, need_dx: bool = True,
                        need_dweight: bool = True, need_dbias: bool = True):
    """(dx, dweight, dbias) (sbc_layer_norm_backward): dx [n, C] of x's type,
    dweight and dbias [C] float32, None where not wanted."""
    index, dev, n, C = _norm_common(x, weight)
    _view(dy, "dy", x.dtype, 2, index)
    if dy.shape != x.shape:
        raise ValueError(f"dy must be {tuple(x.shape)}, got {tuple(dy.shape)}")
    for name, s in (("mean", mean), ("rstd", rstd)):
        _dense(s, name, torch.float32, 1, index)
        if s.numel() != n:
            raise ValueError(f"{name} must be [{n}], got {tuple(s.shape)}")
    dx = torch.empty((n, C), dtype=x.dtype, device=dev) if need_dx else None
    dw = torch.empty(C, dtype=torch.float32, device=dev) if need_dweight else None
    db = torch.empty(C, dtype=torch.float32, device=dev) if need_dbias else None
    lib = L.lib()
    sums = need_dweight or need_dbias
    ws = _Workspace(lib.sbc_layer_norm_workspace_size(n, C) if sums else 0, dev)
    L.check(lib.sbc_layer_norm_backward(dy.data_ptr(), _row_stride(dy), x.data_ptr(),
                                        _row_stride(x), _ptr(weight), mean.data_ptr(),
                                        rstd.data_ptr(), _dtype_code(x), n, C, _ptr(dx), C,
                                        _ptr(dw), _ptr(db), ws.ptr, ws.nbytes, _stream(index)))
    return dx, dw, db


# ---------------------------------------------------------------- rotary positions
def _rotary(q, k, positions, freqs, sections, interleaved, backward, inplace):
    one = q if q is not None else k
    if one is None:
        raise ValueError("q or k is needed")
    _first(one, "q" if q is not None else "k", 3)
    index, dev, (n, _, d) = one.get_device(), one.device, one.shape
    for name, x in (("q", q), ("k", k)):
        if x is not None:
            _view(x, name, one.dtype, 3, index)
            if x.shape[0] != n or x.shape[2] != d:
                raise ValueError(f"{name} must be [{n}, heads, {d}], got {tuple(x.shape)}")
    sections = [int(s) for s in sections]
    if not 1 <= len(sections) <= L.SBC_MAX_AXES:
        raise ValueError(f"1 .. {L.SBC_MAX_AXES} sections expected, got {len(sections)}")
    if min(sections) < 0:
        raise ValueError(f"sections must be >= 0, got {sections}")
    is_float = isinstance(positions, torch.Tensor) and positions.dtype is torch.float32
    _view(positions, "positions", torch.float32 if is_float else torch.int32, 2, index)
    if tuple(positions.shape) != (n, len(sections)):
        raise ValueError(f"positions must be [{n}, {len(sections)}], got {tuple(positions.shape)}")
    _dense(freqs, "freqs", torch.float32, 1, index)
    if freqs.numel() != sum(sections):
        raise ValueError(f"freqs must be [{sum(sections)}], got {tuple(freqs.shape)}")
    plan = L.SbcRotaryPlan(positions.data_ptr(), _row_stride(positions),
                           int(is_float), freqs.data_ptr(), len(sections),
                           (ctypes.c_int32 * L.SBC_MAX_AXES)(*sections), int(interleaved))
    out = [None if x is None else (x if inplace else torch.empty(x.shape, dtype=x.dtype, device=dev))
           for x in (q, k)]
    L.check(L.lib().sbc_rotary(ctypes.byref(plan), _heads(q), 0 if q is None else q.shape[1],
                               _heads(k), 0 if k is None else k.shape[1], _dtype_code(one), n, d,
                               int(backward), _heads(out[0]), _heads(out[1]), _stream(index)))
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
    _first(q, "q", 3)
    index, shape = q.get_device(), q.shape
    n, H, dk = shape
    _view(k, "k", q.dtype, 3, index)
    _view(v, "v", q.dtype, 3, index)
    if k.shape != shape:
        raise ValueError(f"k must be {tuple(shape)}, got {tuple(k.shape)}")
    if v.shape[:2] != shape[:2]:
        raise ValueError(f"v must be [{n}, {H}, dv], got {tuple(v.shape)}")
    _dense(rates, "rates", torch.float32, 1, index)
    if rates.numel() != H:
        raise ValueError(f"rates must be [{H}], got {tuple(rates.shape)}")
    n_batch = n if streams else 1
    if splits is not None:
        _dense(splits, "splits", torch.int32, 1, index)
        if splits.numel() < 1:
            raise ValueError("splits must be [n_batch + 1]")
        n_batch = splits.numel() - 1
    if t is not None:
        _dense(t, "t", torch.int32, 1, index)
        if t.numel() != n:
            raise ValueError(f"t must be [{n}], got {tuple(t.shape)}")
    a = L.SbcAttention(n, n_batch, H, dk, v.shape[2], _dtype_code(q), scale, rates.data_ptr(),
                       _ptr(splits), _ptr(t))
    return index, q.device, a


def _check_state(state, state_time, a, index):
    if state is not None:
        _dense(state, "state", torch.float32, 4, index)
        if state.shape != (a.n_batch, a.heads, a.dk, a.dv):
            raise ValueError(f"state must be {(a.n_batch, a.heads, a.dk, a.dv)}, "
                             f"got {tuple(state.shape)}")
    if state_time is not None:
        _dense(state_time, "state_time", torch.int32, 1, index)
        if state_time.numel() != a.n_batch:
            raise ValueError(f"state_time must be [{a.n_batch}], got {tuple(state_time.shape)}")


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
    index, dev, a = _attention(q, k, v, rates, splits, t, scale)
    _check_state(state, state_time, a, index)
    if state is not None and t is not None and state_time is None:
        raise ValueError("state_time is needed beside state where t is given")
    o = torch.empty((a.n, a.heads, a.dv), dtype=q.dtype, device=dev)
    out = (torch.empty((a.n_batch, a.heads, a.dk, a.dv), dtype=torch.float32, device=dev)
           if return_state else None)
    out_time = (torch.empty(a.n_batch, dtype=torch.int32, device=dev)
                if return_state and t is not None else None)
    lib = L.lib()
    ws = _Workspace(lib.sbc_linear_attention_workspace_size(a.n, a.heads, a.dk, a.dv), dev)
    L.check(lib.sbc_linear_attention_forward(
        ctypes.byref(a), _heads(q), _heads(k), _heads(v), _ptr(state),
        _ptr(state_time if t is not None else None), _heads(o), _ptr(out), _ptr(out_time), ws.ptr,
        ws.nbytes, _stream(index)))
    return (o, out, out_time) if return_state else o


def linear_attention_backward(do, q, k, v, rates, splits: Optional[torch.Tensor] = None,
                              t: Optional[torch.Tensor] = None, scale: float = 1.0,
                              need_rates: bool = True):
    """(dq, dk, dv, drates) for sequences that start from zero
    (sbc_linear_attention_backward); drates [heads] float32, None where not
    wanted."""
    index, dev, a = _attention(q, k, v, rates, splits, t, scale)
    _view(do, "do", q.dtype, 3, index)
    if do.shape != v.shape:
        raise ValueError(f"do must be {tuple(v.shape)}, got {tuple(do.shape)}")
    dq, dk, dv = (torch.empty(x.shape, dtype=q.dtype, device=dev) for x in (q, k, v))
    dr = torch.empty(a.heads, dtype=torch.float32, device=dev) if need_rates else None
    lib = L.lib()
    ws = _Workspace(lib.sbc_linear_attention_backward_workspace_size(a.n, a.heads, a.dk, a.dv),
                    dev)
    L.check(lib.sbc_linear_attention_backward(
        ctypes.byref(a), _heads(do), _heads(q), _heads(k), _heads(v), _heads(dq), _heads(dk),
        _heads(dv), _ptr(dr), ws.ptr, ws.nbytes, _stream(index)))
    return dq, dk, dv, dr


def linear_attention_step(q, k, v, rates, state, t: Optional[torch.Tensor] = None,
                          state_time: Optional[torch.Tensor] = None, scale: float = 1.0,
                          out_state: Optional[torch.Tensor] = None,
                          out_time: Optional[torch.Tensor] = None):
    """One token for each of n streams: (o [n, heads, dv], state, state_time)
    (sbc_linear_attention_step).  The new state is written to out_state, which
    may be state itself (default: a new tensor), and with t the new times to
    out_time (not state_time itself)."""
    index, dev, a = _attention(q, k, v, rates, None, t, scale, streams=True)
    if state is None:
        raise ValueError("state is needed")
    _check_state(state, state_time, a, index)
    if t is not None and state_time is None:
        raise ValueError("state_time is needed beside state where t is given")
    _check_state(out_state, out_time, a, index)
    o = torch.empty((a.n, a.heads, a.dv), dtype=q.dtype, device=dev)
    if out_state is None:
        out_state = torch.empty_like(state)
    if t is None:
        state_time = out_time = None
    elif out_time is None:
        out_time = torch.empty_like(state_time)
    L.check(L.lib().sbc_linear_attention_step(
        ctypes.byref(a), _heads(q), _heads(k), _heads(v), state.data_ptr(), _ptr(state_time),
        _heads(o), out_state.data_ptr(), _ptr(out_time), _stream(index)))
    return o, out_state, out_time
