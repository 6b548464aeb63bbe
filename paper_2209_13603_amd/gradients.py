"""Global norm of many gradients and clipping by it (``disco_gradient_clip`` in
``include/disco.h``) on torch tensors.  Argument marshalling only."""
from __future__ import annotations

import operator

import numpy as np

from .attention import _Call, _dtype
from .disco import _check, library

# disco_tensor_t
_TENSOR = np.dtype([("data", "u8"), ("dtype", "i4"), ("ndim", "i4"), ("shape", "i8", 4)])


def _array(tensors):
    """The tensors as an array of disco_tensor_t, each as one axis of its entries."""
    import torch
    a = np.zeros(len(tensors), dtype=_TENSOR)
    if not all(map(torch.Tensor.is_contiguous, tensors)):
        raise ValueError("gradients must be contiguous")
    a["data"] = list(map(torch.Tensor.data_ptr, tensors))
    a["dtype"] = list(map(_dtype, tensors))
    a["ndim"] = 1
    a["shape"][:, 0] = list(map(torch.Tensor.numel, tensors))
    return a


def clip(grads, max_norm, eps=1e-6, out=None, norm_only=False, stream=None):
    """norm = sqrt(sum of all squares); each gradient times min(1, max_norm / (norm + eps)).

    grads: fp32 and bf16 tensors on one GPU.  Written in place, or to `out` (tensors of the same
    types and shapes; each may be its gradient itself).  Returns (norm, list of the clipped
    tensors); norm is an fp32 scalar on the GPU, nothing waits for it.  norm_only: (norm, grads) with nothing written.
    """
    import torch
    grads = list(grads)
    out = grads if out is None else list(out)
    if not grads:
        raise ValueError("no gradients")
    apart = out is not grads
    shapes = operator.attrgetter("shape")
    if apart and list(map(shapes, out)) != list(map(shapes, grads)):
        raise ValueError("out must match the gradients one by one")
    if len(set(map(torch.Tensor.get_device, grads + out if apart else grads))) != 1:
        raise ValueError("all tensors must be on %s" % grads[0].device)
    call = _Call(grads[0], stream)
    norm = call.empty((), torch.float32)
    a = _array(grads)
    b = _array(out) if apart and not norm_only else a
    keep, ws, n = call.workspace("disco_gradient_clip_workspace", len(grads), a.ctypes.data)
    _check(library().disco_gradient_clip(len(grads), a.ctypes.data, None if norm_only else b.ctypes.data, max_norm, eps,
                                         norm.data_ptr(), ws, n, call.handle))
    return norm, out
