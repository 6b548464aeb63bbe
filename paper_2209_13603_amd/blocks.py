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
import struct
from typing import NamedTuple

from .attention import _Call, _dtype, _same_device
from .disco import _check, library

# disco_rows_t, disco_tensor_t, disco_dropout_t and disco_residual_t (all of whole 8-byte pieces).
_ROWS, _TENSOR = struct.Struct("=Qii5q"), struct.Struct("=Qii4q")
_DROPOUT, _RESIDUAL = struct.Struct("=d3Q"), struct.Struct("=ddii4Q")


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


class _Pack:
    """The structures of one call, in one buffer (a ctypes object for each takes several times as long).  The
    methods return the address of what they add, None for None."""
    __slots__ = ("buffer", "base", "at")

    def __init__(self):
        self.buffer = ctypes.create_string_buffer(1024)
        self.base = ctypes.addressof(self.buffer)
        self.at = 0

    def _add(self, form, *values):
        at = self.at
        form.pack_into(self.buffer, at, *values)
        self.at = at + form.size
        return self.base + at

    def rows(self, t, name):
        if t is None:
            return None
        shape = t.shape
        if len(shape) != 3:
            raise ValueError("%s must be [batch, tokens, channels]" % name)
        B, S, C = shape
        sb, st, sc = t.stride()
        if sc != 1 and C > 1:
            raise ValueError("the last axis of %s must be contiguous" % name)
        at = self.at
        _ROWS.pack_into(self.buffer, at, t.data_ptr(), _dtype(t), 0, B, S, C, sb, st)
        self.at = at + 56
        return self.base + at

    def weight(self, t, name):
        if t is None:
            return None
        shape = t.shape
        if not 1 <= len(shape) <= 2 or not t.is_contiguous():
            raise ValueError("%s must be [channels] or [batch, channels], contiguous" % name)
        at = self.at
        _TENSOR.pack_into(self.buffer, at, t.data_ptr(), _dtype(t), len(shape), shape[0], shape[-1], 0, 0)
        self.at = at + 48
        return self.base + at

    def dropout(self, d, first):
        import torch
        if d is None:
            return None
        counter = 0
        if d.counter is not None:
            if d.counter.dtype != torch.int64 or d.counter.numel() != 1:
                raise ValueError("counter must be one torch.int64")
            _same_device(first, d.counter)
            counter = d.counter.data_ptr()
        return self._add(_DROPOUT, d.p, d.seed & 0xFFFFFFFFFFFFFFFF, d.offset & 0xFFFFFFFFFFFFFFFF, counter)

    def residual(self, first, post_norm, post_weight, gate, next_weight, scale, eps, dropout):
        at = [self.weight(w, name) or 0
              for w, name in ((post_weight, "post_weight"), (gate, "gate"), (next_weight, "next_weight"))]
        return self._add(_RESIDUAL, scale, eps, 1 if post_norm else 0, 0, *at, self.dropout(dropout, first) or 0)


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
    pack = _Pack()
    args = pack.dropout(how, x)
    if x.dim() == 3:
        tx, ty = x, y
    else:
        if not (x.is_contiguous() and y.is_contiguous()):
            raise ValueError("x and y must be contiguous, or [batch, tokens, channels]")
        last = x.shape[-1] if x.dim() else 1
        tx, ty = (t.view(1, x.numel() // last if last else 0, last) for t in (x, y))
    if x.numel():
        _check(library().disco_dropout(pack.rows(tx, "x"), args, pack.rows(ty, "y"), call.handle))
    return y


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
    _same_device(f, x, h, y, post_weight, gate, next_weight)
    pack = _Pack()
    args = pack.residual(f, post_norm, post_weight, gate, next_weight, scale, eps, dropout)
    _check(library().disco_residual_norm(pack.rows(x, "x"), pack.rows(f, "f"), args, pack.rows(h, "h"), pack.rows(y, "y"),
                                         call.handle))
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
    _same_device(f, x, dh, dy, dx, df, post_weight, gate, next_weight)
    pack = _Pack()
    args = pack.residual(f, post_norm, post_weight, gate, next_weight, scale, eps, dropout)
    at_f = pack.rows(f, "f")
    dw = [call.like(w) if w is not None and want_weights else None for w in (post_weight, gate, next_weight)]
    keep, ws, n = (None, None, 0)
    if any(t is not None for t in dw):
        keep, ws, n = call.workspace("disco_residual_norm_workspace", at_f, args)
    _check(library().disco_residual_norm_backward(
        pack.rows(x, "x"), at_f, args, pack.rows(dh, "dh"), pack.rows(dy, "dy"), pack.rows(dx, "dx"), pack.rows(df, "df"),
        pack.weight(dw[0], "dpost_weight"), pack.weight(dw[1], "dgate"), pack.weight(dw[2], "dnext_weight"), ws, n, call.handle))
    return ResidualGrads(dx, df, *dw)
