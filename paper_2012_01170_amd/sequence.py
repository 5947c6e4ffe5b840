"""Binding of the sequence operators: layer norm, rotary positions with several
axes, linear attention with a decay for each head, norms of queries and keys with
their rotation, softmax attention, and a cache in pages.

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


class _NoWorkspace:
    ptr, nbytes = None, 0


def _scratch(nbytes, device):
    """A workspace, if any is needed."""
    return _Workspace(nbytes, device) if nbytes else _NoWorkspace


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
_Sections = ctypes.c_int32 * L.SBC_MAX_AXES


def _rotary_plan(q, k, positions, freqs, sections, interleaved):
    """The checked q and k, one of them, and their plan."""
    one = q if q is not None else k
    if one is None:
        raise ValueError("q or k is needed")
    _first(one, "q" if q is not None else "k", 3)
    index, (n, _, d) = one.get_device(), one.shape
    if k is not None and k is not one:
        _view(k, "k", one.dtype, 3, index)
        if k.shape[0] != n or k.shape[2] != d:
            raise ValueError(f"k must be [{n}, heads, {d}], got {tuple(k.shape)}")
    sections = [int(s) for s in sections]
    axes = len(sections)
    if not 1 <= axes <= L.SBC_MAX_AXES:
        raise ValueError(f"1 .. {L.SBC_MAX_AXES} sections expected, got {axes}")
    if min(sections) < 0:
        raise ValueError(f"sections must be >= 0, got {sections}")
    is_float = isinstance(positions, torch.Tensor) and positions.dtype is torch.float32
    _view(positions, "positions", torch.float32 if is_float else torch.int32, 2, index)
    if positions.shape != (n, axes):
        raise ValueError(f"positions must be [{n}, {axes}], got {tuple(positions.shape)}")
    _dense(freqs, "freqs", torch.float32, 1, index)
    if freqs.shape[0] != sum(sections):
        raise ValueError(f"freqs must be [{sum(sections)}], got {tuple(freqs.shape)}")
    plan = L.SbcRotaryPlan(positions.data_ptr(), _row_stride(positions), int(is_float),
                           freqs.data_ptr(), axes, _Sections(*sections), int(interleaved))
    return one, index, plan


def _rotary(q, k, positions, freqs, sections, interleaved, backward, inplace):
    one, index, plan = _rotary_plan(q, k, positions, freqs, sections, interleaved)
    dev, (n, _, d) = one.device, one.shape
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


# ---------------------------------------------------------------- norms and rotation
def _head_weight(w, name, d, index):
    if w is not None:
        _dense(w, name, torch.float32, 1, index)
        if w.numel() != d:
            raise ValueError(f"{name} must be [{d}], got {tuple(w.shape)}")


def qk_norm_rotary_forward(q, k, q_weight, k_weight, positions, freqs, sections: Sequence[int],
                           interleaved: bool = False, eps: float = 1e-5, inplace: bool = False):
    """q [n, heads, d] and k [n, k_heads, d] (either may be None), each head
    divided by its root mean square, times its weights ([d] float32, or None), and
    turned by the tokens' positions as rotary_forward does
    (sbc_qk_norm_rotary_forward); returns both."""
    one, index, plan = _rotary_plan(q, k, positions, freqs, sections, interleaved)
    dev, (n, _, d) = one.device, one.shape
    _head_weight(q_weight, "q_weight", d, index)
    _head_weight(k_weight, "k_weight", d, index)
    out = [None if x is None else (x if inplace else torch.empty(x.shape, dtype=x.dtype, device=dev))
           for x in (q, k)]
    L.check(L.lib().sbc_qk_norm_rotary_forward(
        ctypes.byref(plan), _heads(q), 0 if q is None else q.shape[1], _heads(k),
        0 if k is None else k.shape[1], _ptr(q_weight), _ptr(k_weight), _dtype_code(one), n, d,
        float(eps), _heads(out[0]), _heads(out[1]), _stream(index)))
    return tuple(out)


def qk_norm_rotary_backward(dq, dk, q, k, q_weight, k_weight, positions, freqs,
                            sections: Sequence[int], interleaved: bool = False, eps: float = 1e-5,
                            need_weights: bool = True):
    """(dq, dk, dq_weight, dk_weight): the gradients of qk_norm_rotary_forward's q
    and k from those of its outputs, and of the weights ([d] float32; None for an
    absent q or k, and where not wanted) (sbc_qk_norm_rotary_backward)."""
    one, index, plan = _rotary_plan(q, k, positions, freqs, sections, interleaved)
    dev, (n, _, d) = one.device, one.shape
    _head_weight(q_weight, "q_weight", d, index)
    _head_weight(k_weight, "k_weight", d, index)
    for name, g, x in (("dq", dq, q), ("dk", dk, k)):
        if (g is None) != (x is None):
            raise ValueError(f"{name} and its input go together")
        if x is not None:
            _view(g, name, x.dtype, 3, index)
            if g.shape != x.shape:
                raise ValueError(f"{name} must be {tuple(x.shape)}, got {tuple(g.shape)}")
    out = [None if x is None else torch.empty(x.shape, dtype=x.dtype, device=dev) for x in (q, k)]
    dw = [torch.empty(d, dtype=torch.float32, device=dev) if need_weights and x is not None
          else None for x in (q, k)]
    lib = L.lib()
    ws = _scratch(lib.sbc_qk_norm_rotary_workspace_size(n, d) if need_weights else 0, dev)
    L.check(lib.sbc_qk_norm_rotary_backward(
        ctypes.byref(plan), _heads(dq), _heads(dk), _heads(q), 0 if q is None else q.shape[1],
        _heads(k), 0 if k is None else k.shape[1], _ptr(q_weight), _ptr(k_weight),
        _dtype_code(one), n, d, float(eps), _heads(out[0]), _heads(out[1]), _ptr(dw[0]),
        _ptr(dw[1]), ws.ptr, ws.nbytes, _stream(index)))
    return out[0], out[1], dw[0], dw[1]


# ---------------------------------------------------------------- softmax attention
def _softmax(q, k, v, splits, k_splits, scale, causal):
    _first(q, "q", 3)
    index, (n, H, dk) = q.get_device(), q.shape
    _view(k, "k", q.dtype, 3, index)
    _view(v, "v", q.dtype, 3, index)
    m, G = k.shape[:2]
    if k.shape[2] != dk:
        raise ValueError(f"k must be [m, kv_heads, {dk}], got {tuple(k.shape)}")
    if v.shape[:2] != k.shape[:2]:
        raise ValueError(f"v must be [{m}, {G}, dv], got {tuple(v.shape)}")
    n_batch = 1
    if splits is not None:
        _dense(splits, "splits", torch.int32, 1, index)
        if splits.numel() < 1:
            raise ValueError("splits must be [n_batch + 1]")
        n_batch = splits.numel() - 1
    if k_splits is not None:
        _dense(k_splits, "k_splits", torch.int32, 1, index)
        if splits is None:
            raise ValueError("k_splits needs splits")
        if k_splits.numel() != n_batch + 1:
            raise ValueError(f"k_splits must be [{n_batch + 1}], got {tuple(k_splits.shape)}")
    scale = dk ** -0.5 if scale is None else float(scale)
    return index, q.device, L.SbcSoftmaxAttention(n, m, n_batch, H, G, dk, v.shape[2],
                                                  _dtype_code(q), scale, int(causal),
                                                  _ptr(splits), _ptr(k_splits))


def softmax_attention_forward(q, k, v, splits: Optional[torch.Tensor] = None,
                              k_splits: Optional[torch.Tensor] = None,
                              scale: Optional[float] = None, causal: bool = False):
    """(o [n, heads, dv], lse [n, heads] float32) of q [n, heads, dk], k [m,
    kv_heads, dk] and v [m, kv_heads, dv] (sbc_softmax_attention_forward):

        o_i = sum_j exp(s_ij - lse_i) v_j,   s_ij = scale q_i . k_j,

    over the keys of the token's sequence, with causal those up to the token (the
    last token sees the last key).  heads is a multiple of kv_heads, head h reads
    head h // (heads // kv_heads).  splits [n_batch + 1] int32 cuts the tokens into
    sequences (None: one) and k_splits the keys (None: as splits).  scale: 1 /
    sqrt(dk) by default."""
    index, dev, a = _softmax(q, k, v, splits, k_splits, scale, causal)
    o = torch.empty((a.n, a.heads, a.dv), dtype=q.dtype, device=dev)
    lse = torch.empty((a.n, a.heads), dtype=torch.float32, device=dev)
    lib, ref = L.lib(), ctypes.byref(a)
    ws = _scratch(lib.sbc_softmax_attention_workspace_size(ref), dev)
    L.check(lib.sbc_softmax_attention_forward(ref, _heads(q), _heads(k), _heads(v), _heads(o),
                                              lse.data_ptr(), ws.ptr, ws.nbytes, _stream(index)))
    return o, lse


def softmax_attention_backward(do, q, k, v, o, lse, splits: Optional[torch.Tensor] = None,
                               k_splits: Optional[torch.Tensor] = None,
                               scale: Optional[float] = None, causal: bool = False):
    """(dq, dk, dv) from the forward pass' o and lse
    (sbc_softmax_attention_backward)."""
    index, dev, a = _softmax(q, k, v, splits, k_splits, scale, causal)
    shape = (a.n, a.heads, a.dv)
    for name, x in (("do", do), ("o", o)):
        _view(x, name, q.dtype, 3, index)
        if x.shape != shape:
            raise ValueError(f"{name} must be {shape}, got {tuple(x.shape)}")
    _dense(lse, "lse", torch.float32, 2, index)
    if lse.shape != shape[:2]:
        raise ValueError(f"lse must be {shape[:2]}, got {tuple(lse.shape)}")
    dq, dk, dv = (torch.empty(x.shape, dtype=q.dtype, device=dev) for x in (q, k, v))
    lib, ref = L.lib(), ctypes.byref(a)
    ws = _scratch(lib.sbc_softmax_attention_backward_workspace_size(ref), dev)
    L.check(lib.sbc_softmax_attention_backward(
        ref, _heads(do), _heads(q), _heads(k), _heads(v), _heads(o), lse.data_ptr(), _heads(dq),
        _heads(dk), _heads(dv), ws.ptr, ws.nbytes, _stream(index)))
    return dq, dk, dv


# ---------------------------------------------------------------- a cache in pages
def _pages(t: Optional[torch.Tensor]):
    if t is None:
        return None
    s = t.stride()
    return ctypes.byref(L.SbcPages(t.data_ptr(), s[0], s[1], s[2]))


def _streams(splits, n, n_batch, index):
    if splits is not None:
        _dense(splits, "splits", torch.int32, 1, index)
        if splits.numel() != n_batch + 1:
            raise ValueError(f"splits must be [{n_batch + 1}], got {tuple(splits.shape)}")
    elif n != n_batch:
        raise ValueError(f"without splits each of the {n_batch} streams has one new token, got {n}")


def softmax_attention_paged(q, k_pages, v_pages, table, lengths,
                            splits: Optional[torch.Tensor] = None, scale: Optional[float] = None):
    """o [n, heads, dv] of n new tokens over the streams' kept ones, themselves
    among them (sbc_softmax_attention_paged): softmax_attention_forward, causal,
    with the keys and values in pages.

    k_pages [n_pages, page, kv_heads, dk] and v_pages [n_pages, page, kv_heads, dv]
    (any strides, the last axis dense); table [n_batch, width] int32: the pages of
    each stream's tokens; lengths [n_batch] int32: its tokens, with the new ones;
    splits [n_batch + 1] int32: its new tokens (None: one)."""
    _first(q, "q", 3)
    index, dev, (n, H, dk) = q.get_device(), q.device, q.shape
    _view(k_pages, "k_pages", q.dtype, 4, index)
    _view(v_pages, "v_pages", q.dtype, 4, index)
    n_pages, page, G = k_pages.shape[:3]
    if k_pages.shape[3] != dk:
        raise ValueError(f"k_pages must be [n_pages, page, kv_heads, {dk}], "
                         f"got {tuple(k_pages.shape)}")
    if v_pages.shape[:3] != k_pages.shape[:3]:
        raise ValueError(f"v_pages must be [{n_pages}, {page}, {G}, dv], got {tuple(v_pages.shape)}")
    _dense(table, "table", torch.int32, 2, index)
    _dense(lengths, "lengths", torch.int32, 1, index)
    n_batch, width = table.shape
    if lengths.numel() != n_batch:
        raise ValueError(f"lengths must be [{n_batch}], got {tuple(lengths.shape)}")
    _streams(splits, n, n_batch, index)
    dv = v_pages.shape[3]
    a = L.SbcSoftmaxAttention(n, 0, n_batch, H, G, dk, dv, _dtype_code(q),
                              dk ** -0.5 if scale is None else float(scale), 1, _ptr(splits), None)
    o = torch.empty((n, H, dv), dtype=q.dtype, device=dev)
    lib, ref = L.lib(), ctypes.byref(a)
    ws = _scratch(lib.sbc_softmax_attention_paged_workspace_size(ref, page, width), dev)
    L.check(lib.sbc_softmax_attention_paged(
        ref, _heads(q), _pages(k_pages), _pages(v_pages), n_pages, page, table.data_ptr(), width,
        lengths.data_ptr(), _heads(o), None, ws.ptr, ws.nbytes, _stream(index)))
    return o


def cache_slots(lengths, table, free, page: int, splits: Optional[torch.Tensor] = None,
                n: Optional[int] = None, out_table: Optional[torch.Tensor] = None):
    """(table, slots, lengths, needed) for the next tokens of n_batch streams
    (sbc_cache_slots): the table [n_batch, width] int32 with the pages that they
    need, taken from free [n_free] int32 in the streams' order (-1 where free has
    no more); slots [n] int64, the new tokens' places in the pages (-1: none); the
    streams' lengths with them; and needed [1] int32, how many pages of free all
    streams need.

    splits [n_batch + 1] int32: the streams' new tokens, n in all (None: one
    each).  out_table: where the table is written, table itself if wanted (default:
    a new one)."""
    index = lengths.get_device() if isinstance(lengths, torch.Tensor) else -1
    if index < 0:
        _require(lengths, "lengths", torch.int32, 1)
    _dense(lengths, "lengths", torch.int32, 1, index)
    _dense(table, "table", torch.int32, 2, index)
    _dense(free, "free", torch.int32, 1, index)
    dev, (n_batch, width) = lengths.device, table.shape
    if lengths.numel() != n_batch:
        raise ValueError(f"lengths must be [{n_batch}], got {tuple(lengths.shape)}")
    if n is None:
        if splits is not None:
            raise ValueError("n, the number of new tokens, is needed beside splits")
        n = n_batch
    _streams(splits, n, n_batch, index)
    if out_table is None:
        out_table = torch.empty_like(table)
    else:
        _dense(out_table, "out_table", torch.int32, 2, index)
        if out_table.shape != table.shape:
            raise ValueError(f"out_table must be {tuple(table.shape)}, got {tuple(out_table.shape)}")
    slots = torch.empty(n, dtype=torch.int64, device=dev)
    after = torch.empty_like(lengths)
    needed = torch.empty(1, dtype=torch.int32, device=dev)
    lib = L.lib()
    ws = _scratch(lib.sbc_cache_slots_workspace_size(n_batch), dev)
    L.check(lib.sbc_cache_slots(lengths.data_ptr(), _ptr(splits), n, n_batch, table.data_ptr(),
                                width, int(page), free.data_ptr(), free.numel(),
                                out_table.data_ptr(), slots.data_ptr(), after.data_ptr(),
                                needed.data_ptr(), ws.ptr, ws.nbytes, _stream(index)))
    return out_table, slots, after, needed


def cache_append(k, v, k_pages, v_pages, slots):
    """The rows of k [n, kv_heads, dk] and v [n, kv_heads, dv] written to their
    slots ([n] int64, from cache_slots; outside the pages: left out, else
    distinct) of k_pages [n_pages, page, kv_heads, dk] and v_pages
    (sbc_cache_append).  k may be None with k_pages, v with v_pages."""
    one, pages = (k, k_pages) if k is not None else (v, v_pages)
    if one is None:
        raise ValueError("k or v is needed")
    _first(one, "k" if k is not None else "v", 3)
    index, (n, G) = one.get_device(), one.shape[:2]
    d = [0, 0]
    for i, (name, x, to) in enumerate((("k", k, k_pages), ("v", v, v_pages))):
        if (x is None) != (to is None):
            raise ValueError(f"{name} and {name}_pages go together")
        if x is None:
            continue
        _view(x, name, one.dtype, 3, index)
        _view(to, name + "_pages", one.dtype, 4, index)
        d[i] = x.shape[2]
        if x.shape[:2] != (n, G):
            raise ValueError(f"{name} must be [{n}, {G}, d], got {tuple(x.shape)}")
        if to.shape != (*pages.shape[:2], G, d[i]):
            raise ValueError(f"{name}_pages must be [{pages.shape[0]}, {pages.shape[1]}, {G}, {d[i]}], "
                             f"got {tuple(to.shape)}")
    _dense(slots, "slots", torch.int64, 1, index)
    if slots.numel() != n:
        raise ValueError(f"slots must be [{n}], got {tuple(slots.shape)}")
    L.check(L.lib().sbc_cache_append(_heads(k), _heads(v), n, G, d[0], d[1], _dtype_code(one),
                                     slots.data_ptr(), _pages(k_pages), _pages(v_pages),
                                     pages.shape[0], pages.shape[1], _stream(index)))
