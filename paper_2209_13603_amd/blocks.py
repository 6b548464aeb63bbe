"""What stands around a block of a network: the residual sum with its norms, gate and
dropout, and dropout alone.

The channel operators of ``libdisco.so`` (``disco_residual_norm``, ``disco_dropout``
and the gradients in ``include/disco.h``) on torch tensors [batch, tokens, channels] of any
strides whose last axis is contiguous.  Argument marshalling only; outputs and scratch
memory come from torch's allocator, on the stream that the call runs on.

    drop = blocks.Dropout(0.1, seed, offset=step)                    # no mask is stored
    h, y = blocks.residual_norm(x, f, post_norm=True, post_weight=w1, gate=g, next_weight=w2, dropout=drop)
    grads = blocks.residual_norm_backward(x, f, dh, dy, post_norm=True, post_weight=w1, gate=g, next_weight=w2,
                                          dropout=drop)
    grads.dx, grads.df, grads.dpost_weight, grads.dgate, grads.dnext_weight
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

from .attention import _Call, _dtype, _ref, _same_device
from .disco import DropoutArgs, ResidualArgs, Rows, _check, _tensor, library


class Dropout(NamedTuple):
    """How a call drops entries: with probability p (to the nearest 2^-16), by the generator's seed and offset (whole
    numbers of 64 bits; another offset for each call that is to draw anew).  counter: None, or an int64
    tensor of one entry on the GPU that is added to the offset when the call runs: raised inside a
    captured graph, it makes each replay draw anew."""
    p: float
    seed: int
    offset: int = 0
    counter: object = None


class ResidualGrads(NamedTuple):
    dx: object
    df: object
    dpost_weight: object
    dgate: object
    dnext_weight: object


def _rows(t, name) -> Rows:
    if t.dim() != 3:
        raise ValueError("%s must be [batch, tokens, channels]" % name)
    B, S, C = t.shape
    sb, st, sc = t.stride()
    if sc != 1 and C > 1:
        raise ValueError("the last axis of %s must be contiguous" % name)
    return Rows(t.data_ptr() or None, _dtype(t), 0, B, S, C, sb, st)


def _dropout(d, first):
    import torch
    if d is None:
        return None
    address = None
    if d.counter is not None:
        if d.counter.dtype != torch.int64 or d.counter.numel() != 1:
            raise ValueError("counter must be one torch.int64")
        _same_device(first, d.counter)
        address = d.counter.data_ptr()
    return DropoutArgs(d.p, d.seed & 0xFFFFFFFFFFFFFFFF, d.offset & 0xFFFFFFFFFFFFFFFF, address)


def dropout(x, how, y=None, stream=None):
    """x with each entry kept, times 1 / (1 - p), or 0, as `how` (a ``Dropout``) draws (``disco_dropout``).
    Rows run along the last axis.  Its gradient is the same call on dy.  x: fp32 or bf16 of any shape,
    contiguous, or [batch, tokens, channels] of any strides.  y: None, x itself, or a tensor to write to."""
    call = _Call(x, stream)
    if y is None:
        y = call.like(x)
    _same_device(x, y)
    if y.shape != x.shape:
        raise ValueError("x and y must have the same shape")
    args = _dropout(how, x)
    if x.dim() == 3:
        tx, ty = x, y
    else:
        if not (x.is_contiguous() and y.is_contiguous()):
            raise ValueError("x and y must be contiguous, or [batch, tokens, channels]")
        last = x.shape[-1] if x.dim() else 1
        tx, ty = (t.view(1, x.numel() // last if last else 0, last) for t in (x, y))
    if x.numel():
        _check(library().disco_dropout(_rows(tx, "x"), args, _rows(ty, "y"), call.handle))
    return y


def _residual(first, post_norm, post_weight, gate, next_weight, scale, eps, dropout):
    """(disco_residual_t, the tensors of the weights): what it points to lives as long as it does."""
    _same_device(first, post_weight, gate, next_weight)
    tensors = [_tensor(w) if w is not None else None for w in (post_weight, gate, next_weight)]
    for w in (post_weight, gate, next_weight):
        if w is not None and not w.is_contiguous():
            raise ValueError("weights must be contiguous")
    drop = _dropout(dropout, first)
    ptr = [ctypes.pointer(t) if t is not None else None for t in (*tensors, drop)]
    return ResidualArgs(scale, eps, int(post_norm), 0, *ptr), tensors


def residual_norm(x, f, post_norm=False, post_weight=None, gate=None, next_weight=None, scale=1.0, eps=1e-6, dropout=None,
                  want_h=True, want_y=True, h=None, y=None, stream=None):
    """(h, y): the residual sum of a block and its norm for the next one, in one pass (``disco_residual_norm``):

        h = scale x + gate * dropout(post_weight * f / rms(f)),  y = next_weight * h / rms(h)

    x: the residual stream [B, S, C], or None; f: the block's output, which is normed with post_norm.  The
    weights are None, [C] or [B, C] of x's type.  dropout: None or a ``Dropout``.  C up to 8192.  h, y: None, x or f itself, or
    tensors to write to; None is returned for one that is not asked for.
    """
    call = _Call(f, stream)
    if want_h and h is None:
        h = call.like(f)
    if want_y and y is None:
        y = call.like(f)
    h, y = h if want_h else None, y if want_y else None
    _same_device(f, x, h, y)
    args, keep = _residual(f, post_norm, post_weight, gate, next_weight, scale, eps, dropout)
    rows = [_rows(t, name) if t is not None else None for t, name in ((x, "x"), (f, "f"), (h, "h"), (y, "y"))]
    _check(library().disco_residual_norm(rows[0], rows[1], args, rows[2], rows[3], call.handle))
    return h, y


def residual_norm_backward(x, f, dh, dy, post_norm=False, post_weight=None, gate=None, next_weight=None, scale=1.0, eps=1e-6,
                           dropout=None, want_dx=True, want_df=True, want_weights=True, dx=None, df=None, stream=None):
    """``ResidualGrads`` of ``residual_norm`` for dh and dy (either may be None) from its inputs
    (``disco_residual_norm_backward``); None for what is not asked for or has no input.  dx, df: None,
    one of x, f, dh and dy themselves, or tensors to write to."""
    call = _Call(f, stream)
    if x is None or not want_dx:
        dx = None
    elif dx is None:
        dx = call.like(f)
    if not want_df:
        df = None
    elif df is None:
        df = call.like(f)
    _same_device(f, x, dh, dy, dx, df)
    args, keep = _residual(f, post_norm, post_weight, gate, next_weight, scale, eps, dropout)
    dw = [call.like(w) if w is not None and want_weights else None for w in (post_weight, gate, next_weight)]
    rows = [_rows(t, name) if t is not None else None
            for t, name in ((x, "x"), (f, "f"), (dh, "dh"), (dy, "dy"), (dx, "dx"), (df, "df"))]
    sums = [_tensor(t) if t is not None else None for t in dw]
    ws = (None, None, 0)
    if any(t is not None for t in dw):
        ws = call.workspace("disco_residual_norm_workspace", rows[1], args)
    _check(library().disco_residual_norm_backward(rows[0], rows[1], args, rows[2], rows[3], rows[4], rows[5], *map(_ref, sums),
                                                  ws[1], ws[2], call.handle))
    return ResidualGrads(dx, df, *dw)
