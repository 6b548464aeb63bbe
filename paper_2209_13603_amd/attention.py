"""Attention between grids: norm and rotation of the heads, cross attention.

The token operators of ``libdisco.so`` (``disco_norm_rotate``,
``disco_cross_attention`` and their gradients in ``include/disco.h``) on torch
tensors [batch, tokens, heads, dim] of any strides whose last axis is
contiguous: parts of a joint projection are read where they lie.  Argument
marshalling only; outputs and scratch memory come from torch's allocator, on the
stream that the call runs on.

    tables = attention.grid_rotation(64, 128, 32)                  # cosines, sines of a 64 x 128 grid
    k = attention.norm_rotate(k, k_weight, rotation=tables)        # [B, 8192, Hk, D]
    out, stats = attention.cross_attention(q, k, v, key_bias=area.log(), return_stats=True)
    dq, dk, dv = attention.cross_attention_backward(q, k, v, out, stats, dout, key_bias=area.log())
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple

from .disco import (AttentionArgs, DISCO_BFLOAT16, DISCO_FLOAT32, Heads, RotationArgs, _check, _tensor, library)

LAYOUTS = {"half": 0, "interleaved": 1}


class Stats(NamedTuple):
    """What ``cross_attention`` keeps for its gradients: rows fp32 [B, H, Sq, 2], a reference near each row's
    largest score in units of log 2 and the sum of 2^(score - reference), so that the logarithm of the
    softmax's sum is (rows[..., 0] + log2(rows[..., 1])) * log(2); low, in bf16 storage, what rounding took from out."""
    rows: object
    low: object


# Storage types (DISCO_FLOAT32, DISCO_BFLOAT16); the library refuses the others.
_DTYPES = {}


def _dtype(t):
    code = _DTYPES.get(t.dtype)
    if code is None:
        import torch
        _DTYPES.update({torch.float32: DISCO_FLOAT32, torch.bfloat16: DISCO_BFLOAT16})
        code = _DTYPES.get(t.dtype, 99)
    return code


def _heads(t, name) -> Heads:
    if t.dim() != 4:
        raise ValueError("%s must be [batch, tokens, heads, dim]" % name)
    B, S, H, D = t.shape
    sb, st, sh, sd = t.stride()
    if sd != 1 and D > 1:
        raise ValueError("the last axis of %s must be contiguous" % name)
    return Heads(t.data_ptr() or None, _dtype(t), D, H, 0, B, S, sb, st, sh)


def _small(t, name, dtype, *shapes):
    """A small argument of a given type and one of the given shapes; (address, batch stride)."""
    if t.dtype != dtype:
        raise ValueError("%s must be %s" % (name, dtype))
    shape = tuple(t.shape)
    if shape not in shapes:
        raise ValueError("%s must be one of the shapes %s" % (name, list(shapes)))
    if not t.is_contiguous() and shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("the last axis of %s must be contiguous" % name)
    return t.data_ptr() or None, t.stride(0) if len(shape) == 2 and shape[0] > 1 else 0


def _same_device(first, *others):
    at = first.get_device()
    for t in others:
        if t is not None and t.get_device() != at:
            raise ValueError("all tensors must be on %s" % first.device)


class _Call:
    """The stream of one call, and where its outputs and scratch memory come from: torch's allocator,
    on that stream."""
    __slots__ = ("first", "stream", "handle")

    def __init__(self, t, stream):
        import torch
        if not t.is_cuda:
            raise ValueError("tensors must be on a GPU")
        self.first = t
        self.stream = stream
        self.handle = torch._C._cuda_getCurrentRawStream(t.get_device()) if stream is None else stream.cuda_stream

    def like(self, t):
        """A new dense tensor of t's shape and type."""
        import torch
        if self.stream is None:
            return torch.empty_like(t, memory_format=torch.contiguous_format)
        with torch.cuda.stream(self.stream):
            return torch.empty_like(t, memory_format=torch.contiguous_format)

    def empty(self, shape, dtype):
        import torch
        if self.stream is None:
            return self.first.new_empty(shape, dtype=dtype)
        with torch.cuda.stream(self.stream):
            return self.first.new_empty(shape, dtype=dtype)

    def workspace(self, name, *args):
        """(tensor to keep until the call is enqueued, address, bytes)"""
        import torch
        need = ctypes.c_size_t()
        _check(getattr(library(), name)(*args, need))
        if need.value == 0:
            return None, None, 0
        ws = self.empty(need.value, torch.uint8)
        return ws, ws.data_ptr(), need.value


def _rotation(rotation, layout, positions, first_position, x):
    """disco_rotation_t of the tables (cosines, sines), or None."""
    import torch
    if rotation is None:
        return None
    cos, sin = rotation
    if cos.dtype != torch.float32 or sin.dtype != torch.float32:
        raise ValueError("cosines and sines must be torch.float32")
    if cos.dim() != 2 or cos.shape != sin.shape or not (cos.is_contiguous() and sin.is_contiguous()):
        raise ValueError("cosines and sines must be [rows, rotary / 2], contiguous")
    _same_device(x, cos, sin, positions)
    rows, half = cos.shape
    address, stride = None, 0
    if positions is not None:
        B, S = x.shape[:2]
        address, stride = _small(positions, "positions", torch.int32, (S,), (1, S), (B, S))
    return RotationArgs(2 * half, LAYOUTS[layout], cos.data_ptr() or None, sin.data_ptr() or None, rows, address, stride,
                        first_position)


def _ref(s):
    return ctypes.byref(s) if s is not None else None


def norm_rotate(x, weight=None, rotation=None, layout="half", positions=None, first_position=0, norm=True, eps=1e-6,
                y=None, stream=None):
    """y = rotate(weight * x / sqrt(mean(x^2) + eps)), for every head of every token of x
    [B, S, H, D] in one pass (``disco_norm_rotate``).

    weight: None, [D] or [H, D] of x's type.  rotation: None, or the tables (cosines, sines), fp32
    [rows, R / 2], R <= D; token s turns by row positions[s] (int32 [S] or [B, S]), or
    first_position + s without positions.  layout: "half" pairs entry i with i + R / 2,
    "interleaved" 2i with 2i + 1.  norm False: the rotation alone.  y: None, x itself, or a tensor
    of x's shape and type.
    """
    call = _Call(x, stream)
    if y is None:
        y = call.like(x)
    _same_device(x, weight, y)
    hx, hy = _heads(x, "x"), _heads(y, "y")
    tw = _tensor(weight) if weight is not None else None
    rot = _rotation(rotation, layout, positions, first_position, x)
    _check(library().disco_norm_rotate(hx, int(norm), _ref(tw), eps, _ref(rot), hy, call.handle))
    return y


def norm_rotate_backward(x, weight, dy, rotation=None, layout="half", positions=None, first_position=0, norm=True,
                         eps=1e-6, want_dx=True, want_dw=True, dx=None, stream=None):
    """Gradients of ``norm_rotate`` for dy: (dx, dweight), None for those not asked for or, without
    a weight, not there.  x may be None without the norm.  dx: None, dy itself, or a tensor to write to."""
    call = _Call(dy, stream)
    if want_dx and dx is None:
        dx = call.like(dy)
    dw = call.like(weight) if want_dw and weight is not None else None
    _same_device(dy, x, weight, dx)
    hx = _heads(x, "x") if x is not None else None
    hdy = _heads(dy, "dy")
    hdx = _heads(dx, "dx") if dx is not None else None
    tw = _tensor(weight) if weight is not None else None
    tdw = _tensor(dw) if dw is not None else None
    rot = _rotation(rotation, layout, positions, first_position, dy)
    keep, ws, n = call.workspace("disco_norm_rotate_workspace", hdy, _ref(tw)) if dw is not None else (None, None, 0)
    _check(library().disco_norm_rotate_backward(_ref(hx), int(norm), _ref(tw), eps, _ref(rot), hdy, _ref(hdx),
                                                _ref(tdw), ws, n, call.handle))
    return dx, dw


def _options(q, k, key_bias, key_lengths, scale):
    import torch
    B, Sk = k.shape[:2]
    bias = lengths = None
    stride = 0
    if key_bias is not None:
        bias, stride = _small(key_bias, "key_bias", torch.float32, (Sk,), (1, Sk), (B, Sk))
    if key_lengths is not None:
        lengths, _ = _small(key_lengths, "key_lengths", torch.int32, (B,))
    _same_device(q, key_bias, key_lengths)
    return AttentionArgs(0.0 if scale is None else scale, bias, stride, lengths)


def cross_attention(q, k, v, key_bias=None, key_lengths=None, scale=None, return_stats=False, out=None, stream=None):
    """out[b, i, h] = sum_j softmax_j(scale q[b, i, h] . k[b, j, h'] + key_bias[b, j]) v[b, j, h']
    (``disco_cross_attention``): q [B, Sq, H, D], k and v [B, Sk, Hk, D], h' = h // (H / Hk).

    key_bias: None or fp32 [Sk] or [B, Sk] (the logarithm of a quadrature weight; -inf takes the key
    out).  key_lengths: None or int32 [B].  scale: 1 / sqrt(D) where None.  A query that no key is left for
    gives zeros.  return_stats: (out, Stats) for ``cross_attention_backward``.
    """
    import torch
    call = _Call(q, stream)
    if out is None:
        out = call.like(q)
    if scale == 0.0:
        raise ValueError("scale must not be 0")
    _same_device(q, k, v, out)
    rows = call.empty((q.shape[0], q.shape[2], q.shape[1], 2), torch.float32) if return_stats else None
    low = call.like(q) if return_stats and q.dtype == torch.bfloat16 else None
    hlow = _heads(low, "low") if low is not None else None
    hq, hk = _heads(q, "q"), _heads(k, "k")
    opt = _options(q, k, key_bias, key_lengths, scale)
    keep, ws, n = call.workspace("disco_cross_attention_workspace", hq, hk, 0)
    _check(library().disco_cross_attention(hq, hk, _heads(v, "v"), opt, _heads(out, "out"),
                                           rows.data_ptr() or None if rows is not None else None, _ref(hlow),
                                           ws, n, call.handle))
    return (out, Stats(rows, low)) if return_stats else out


def cross_attention_backward(q, k, v, out, stats, dout, key_bias=None, key_lengths=None, scale=None, dq=None, dk=None,
                             dv=None, stream=None):
    """(dq, dk, dv) of ``cross_attention`` for dout, from its out and stats
    (``disco_cross_attention_backward``).  dq, dk, dv: None, or tensors to write to, which may be parts
    of one joint buffer."""
    import torch
    call = _Call(q, stream)
    dq = call.like(q) if dq is None else dq
    dk = call.like(k) if dk is None else dk
    dv = call.like(v) if dv is None else dv
    if scale == 0.0:
        raise ValueError("scale must not be 0")
    rows, low = stats
    _same_device(q, k, v, out, rows, low, dout, dq, dk, dv)
    _small(rows, "stats.rows", torch.float32, (q.shape[0], q.shape[2], q.shape[1], 2))
    if not rows.is_contiguous():
        raise ValueError("stats.rows must be contiguous")
    hlow = _heads(low, "stats.low") if low is not None else None
    hq, hk = _heads(q, "q"), _heads(k, "k")
    opt = _options(q, k, key_bias, key_lengths, scale)
    keep, ws, n = call.workspace("disco_cross_attention_workspace", hq, hk, 1)
    _check(library().disco_cross_attention_backward(
        hq, hk, _heads(v, "v"), opt, _heads(out, "out"), rows.data_ptr() or None,
        _ref(hlow), _heads(dout, "dout"), _heads(dq, "dq"), _heads(dk, "dk"), _heads(dv, "dv"), ws, n, call.handle))
    return dq, dk, dv


# --------------------------------------------------------------------------- #
# Rotation tables (made once, on the host in 64 bits)
# --------------------------------------------------------------------------- #
def _tables(angle, device):
    return angle.cos().float().to(device), angle.sin().float().to(device)


def line_rotation(rows, rotary_dim, base=10000.0, stretch=1.0, stretch_base=None, device="cuda"):
    """Tables of positions 0 .. rows - 1 on a line: pair i turns by (position / stretch) *
    base^(-2i / rotary_dim).  For contexts `stretch` times those trained on, positions are pressed together
    (stretch) or, with stretch_base, the base is raised by stretch^(R / (R - 2)) instead, which leaves the
    fastest pair as it was and slows the slowest by stretch."""
    import torch
    half = rotary_dim // 2
    if stretch_base:
        base, stretch = base * float(stretch) ** (rotary_dim / max(1, rotary_dim - 2)), 1.0
    i = torch.arange(half, dtype=torch.float64)
    p = torch.arange(rows, dtype=torch.float64)[:, None] / stretch
    return _tables(p * float(base) ** (-i / max(1, half)), device)


def grid_rotation(nlat, nlon, rotary_dim, device="cuda"):
    """Tables of the tokens of a cell-centred nlat x nlon grid, longitude fastest: the first half of the
    pairs turns by whole multiples of the longitude (so scores depend on longitude differences alone,
    closed around the sphere), the others by whole multiples of the colatitude."""
    import torch
    half = rotary_dim // 2
    by_lon = (half + 1) // 2
    lon = 2 * math.pi * torch.arange(nlon, dtype=torch.float64) / nlon
    colat = math.pi * (torch.arange(nlat, dtype=torch.float64) + 0.5) / nlat
    a = lon[None, :, None] * torch.arange(1, by_lon + 1, dtype=torch.float64)
    b = colat[:, None, None] * torch.arange(1, half - by_lon + 1, dtype=torch.float64)
    angle = torch.cat((a.expand(nlat, nlon, by_lon), b.expand(nlat, nlon, half - by_lon)), -1)
    return _tables(angle.reshape(nlat * nlon, half), device)
