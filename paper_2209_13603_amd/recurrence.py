"""Gated linear recurrence along time.

``disco_gated_recurrence`` and its gradients (``include/disco.h``) on torch tensors
[batch, tokens, channels] of any strides whose last axis is contiguous: series of the cells
of a grid with time slowest in memory and parts of a joint projection are read where they
lie.  Argument marshalling only; outputs and scratch memory come from torch's allocator, on
the stream that the call runs on.

    y, state, carries = recurrence.gated_recurrence(x, gate, return_carries=True)       # training
    grads = recurrence.gated_recurrence_backward(x, gate, carries, dy)
    y, state = recurrence.gated_recurrence(x1, gate1, state=state, state_out=state)     # one more time step
"""
from __future__ import annotations

import struct
from typing import NamedTuple

from .attention import _Call, _same_device
from .blocks import _Pack
from .disco import _check, library

_RECURRENCE = struct.Struct("=iiQ")  # disco_recurrence_t

GAINS = {"mean": 0, "power": 1, "one": 2}
RUN = 16  # tokens between two states that are kept for the gradients


class RecurrenceGrads(NamedTuple):
    dx: object
    dgate: object
    dout_gate: object
    dstate: object


def _options(pack, x, lengths, gain):
    import torch
    address = 0
    if lengths is not None:
        if lengths.dtype != torch.int32 or tuple(lengths.shape) != (x.shape[0],) or not lengths.is_contiguous():
            raise ValueError("lengths must be torch.int32 [batch], contiguous")
        _same_device(x, lengths)
        address = lengths.data_ptr()
    if gain not in GAINS:
        raise ValueError("gain must be one of %s" % ", ".join(GAINS))
    return pack._add(_RECURRENCE, GAINS[gain], 0, address)


def _floats(x, t, name, shape):
    """The address of an fp32 argument of the given shape, or None."""
    import torch
    if t is None:
        return None
    if t.dtype != torch.float32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError("%s must be torch.float32 %s, contiguous" % (name, list(shape)))
    _same_device(x, t)
    return t.data_ptr() or None


def gated_recurrence(x, gate, out_gate=None, state=None, lengths=None, gain="mean", return_carries=False, y=None,
                     state_out=None, stream=None):
    """(y, state): h_t = a_t h_(t-1) + c_t x_t along the tokens, for every channel by itself, a = sigmoid(gate); y_t = h_t,
    or h_t sigmoid(out_gate_t) (``disco_gated_recurrence``).

    x, gate, out_gate (or None): [B, T, C] of one type.  state: h before the first token, fp32 [B, C], or None (zeros).
    gain: c = 1 - a ("mean"), sqrt(1 - a^2) ("power") or 1 ("one").  lengths: None or int32 [B]; tokens beyond leave the
    state as it is and give zeros.  return_carries: (y, state, carries) for ``gated_recurrence_backward``.
    y: None, one of the inputs itself, or a tensor to write to; state_out: None, state itself, or a tensor to write to.
    """
    import torch
    call = _Call(x, stream)
    if y is None:
        y = call.like(x)
    _same_device(x, gate, out_gate, y)
    B, T, C = x.shape
    if state_out is None:
        state_out = call.empty((B, C), torch.float32)
    carries = call.empty((B, -(-T // RUN), C), torch.float32) if return_carries else None
    pack = _Pack()
    options, at_x = _options(pack, x, lengths, gain), pack.rows(x, "x")
    keep, ws, n = call.workspace("disco_gated_recurrence_workspace", at_x)
    _check(library().disco_gated_recurrence(
        at_x, pack.rows(gate, "gate"), pack.rows(out_gate, "out_gate"), options, _floats(x, state, "state", (B, C)),
        pack.rows(y, "y"), _floats(x, state_out, "state_out", (B, C)),
        carries.data_ptr() or None if carries is not None else None, ws, n, call.handle))
    return (y, state_out, carries) if return_carries else (y, state_out)


def gated_recurrence_backward(x, gate, carries, dy, out_gate=None, lengths=None, gain="mean", dstate=None, want_dx=True,
                              want_dgate=True, want_dstate=True, dx=None, dgate=None, dout_gate=None, dstate_out=None,
                              stream=None):
    """``RecurrenceGrads`` of ``gated_recurrence`` for dy and dstate (of the state it returned; None: zeros), from its
    inputs and carries (``disco_gated_recurrence_backward``): those of x, the gates and the state it was given; None for
    what is not asked for or has no input.  dx, dgate, dout_gate: None, one of the inputs themselves, or tensors
    to write to, which may be parts of one joint buffer; dstate_out: None, dstate itself, or a tensor."""
    import torch
    call = _Call(x, stream)
    B, T, C = x.shape
    dx = (call.like(x) if dx is None else dx) if want_dx else None
    dgate = (call.like(x) if dgate is None else dgate) if want_dgate else None
    if out_gate is None or not want_dgate:
        dout_gate = None
    elif dout_gate is None:
        dout_gate = call.like(x)
    if want_dstate and dstate_out is None:
        dstate_out = call.empty((B, C), torch.float32)
    _same_device(x, gate, out_gate, carries, dy, dx, dgate, dout_gate)
    pack = _Pack()
    options, at_x = _options(pack, x, lengths, gain), pack.rows(x, "x")
    keep, ws, n = call.workspace("disco_gated_recurrence_workspace", at_x)
    _check(library().disco_gated_recurrence_backward(
        at_x, pack.rows(gate, "gate"), pack.rows(out_gate, "out_gate"), options,
        _floats(x, carries, "carries", (B, -(-T // RUN), C)), pack.rows(dy, "dy"), _floats(x, dstate, "dstate", (B, C)),
        pack.rows(dx, "dx"), pack.rows(dgate, "dgate"), pack.rows(dout_gate, "dout_gate"),
        _floats(x, dstate_out, "dstate_out", (B, C)) if want_dstate else None, ws, n, call.handle))
    return RecurrenceGrads(dx, dgate, dout_gate, dstate_out if want_dstate else None)
