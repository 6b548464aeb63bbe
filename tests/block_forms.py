"""The block operators from their definitions in 64 bits, for the GPU tests: gradients by automatic differentiation."""
from __future__ import annotations

import numpy as np


def kept(rows, columns, seed, offset, out):
    """Which entries stay (bool [rows, columns]): the definition of the generator in numpy's unsigned words."""
    blocks = -(-columns // 8)
    m32 = np.uint64(0xFFFFFFFF)
    word = lambda v: np.uint64(v % 2 ** 32)
    a = np.tile(np.arange(blocks, dtype=np.uint64), rows)
    b = np.repeat(np.arange(rows, dtype=np.uint64), blocks)
    c, d = np.full_like(a, word(offset)), np.full_like(a, word(offset >> 32))
    k0, k1 = seed % 2 ** 32, (seed >> 32) % 2 ** 32
    for _ in range(10):
        p, q = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, d = (q >> np.uint64(32)) ^ b ^ word(k0), q & m32, (p >> np.uint64(32)) ^ d ^ word(k1), p & m32
        k0, k1 = k0 + 0x9E3779B9, k1 + 0xBB67AE85
    words = np.stack([a, b, c, d], -1).astype(np.uint32)
    halves = np.stack([words & 0xFFFF, words >> 16], -1).reshape(rows, 8 * blocks)
    return halves[:, :columns] >= out


def dropout_factor(shape, how):
    """Factors of the entries of [..., columns] for a ``blocks.Dropout``, as a 64-bit CPU tensor."""
    import torch
    out = round(how.p * 65536)
    columns = shape[-1] if len(shape) else 1
    rows = int(np.prod(shape[:-1], dtype=np.int64)) if len(shape) else 1
    seed, offset = how.seed % 2 ** 64, how.offset % 2 ** 64
    keep = torch.from_numpy(kept(rows, columns, seed, offset, out)).reshape(shape)
    return keep.double() * (65536.0 / (65536 - out) if out < 65536 else 0.0)


def residual(x, f, dh, dy, post_norm, post_weight, gate, next_weight, scale, eps, factor):
    """[h, y] and, where dh or dy is given, the gradients of x, f and the weights that are there."""
    import torch
    grads = dh is not None or dy is not None
    leaf = [t.detach().cpu().double().requires_grad_(grads) if t is not None else None
            for t in (x, f, post_weight, gate, next_weight)]
    x, f, w1, g, w2 = leaf
    wide = lambda w: w[:, None] if w.dim() == 2 else w
    u = f
    if post_norm:
        u = f / (f.pow(2).mean(-1, keepdim=True) + eps).sqrt()
        u = u * wide(w1) if w1 is not None else u
    if factor is not None:
        u = u * factor
    if g is not None:
        u = u * wide(g)
    h = u if x is None else scale * x + u
    y = h / (h.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    y = y * wide(w2) if w2 is not None else y
    out = [h.detach(), y.detach()]
    if not grads:
        return out
    total = 0.0
    for o, d in ((h, dh), (y, dy)):
        if d is not None:
            total = total + (o * d.detach().cpu().double()).sum()
    wrt = [t for t in leaf if t is not None]
    return out + list(torch.autograd.grad(total, wrt, allow_unused=True))


def recurrence(x, g, z, state, lengths, gain, dy=None, dstate=None, device="cpu"):
    """[y, state] and, for dy, the gradients of x, the gates and the state; step by step."""
    import torch
    grads = dy is not None
    B, T, C = x.shape
    x, g, z = (t.detach().to(device).double().requires_grad_(grads) if t is not None else None for t in (x, g, z))
    h0 = state.detach().to(device).double() if state is not None else torch.zeros((B, C), dtype=torch.float64, device=device)
    h0.requires_grad_(grads)
    ends = [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths.tolist()]
    inside = torch.arange(T, device=device)[None] < torch.tensor(ends, device=device)[:, None]
    a = torch.sigmoid(g)
    rest = torch.sigmoid(-g)
    c = {"mean": rest, "power": (rest * (1 + a)).sqrt(), "one": torch.ones_like(a)}[gain]
    h, ys = h0, []
    for t in range(T):
        nh = a[:, t] * h + c[:, t] * x[:, t]
        h = torch.where(inside[:, t, None], nh, h)
        y = h * torch.sigmoid(z[:, t]) if z is not None else h
        ys.append(torch.where(inside[:, t, None], y, torch.zeros_like(y)))
    y = torch.stack(ys, 1) if ys else torch.zeros((B, 0, C), dtype=torch.float64, device=device)
    out = [y.detach(), h.detach()]
    if not grads:
        return out
    total = (y * dy.detach().to(device).double()).sum()
    if dstate is not None:
        total = total + (h * dstate.detach().to(device).double()).sum()
    wrt = [t for t in (x, g, z, h0) if t is not None]
    return out + list(torch.autograd.grad(total, wrt))


def rel(got, want):
    """Relative 2-norm of the error."""
    want = want.cpu()
    d = float((got.detach().cpu().double() - want).norm())
    n = float(want.norm())
    return d / n if n else d
