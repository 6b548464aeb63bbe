"""One training step, and one station's answer, of a small model on the sphere.

A DISCO layer halves the input grid; every coarse cell's channels are a state.  A
finer decoder grid asks the states: queries and keys of each head are normed and
rotated to their places on the sphere, attention weighs each state by its cell's area
and leaves out cells without observations, and the transposed DISCO op takes the answer
back to the input grid.  The step's gradients, DISCO weights among them, are clipped by
their global norm.  ``station`` asks the same states from single places, as a served
model does.

    python examples/grid_attention.py
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2209_13603_amd import attention, disco, gradients  # noqa: E402


class GridAttention:
    def __init__(self, nlat=64, heads=4, dim=32, dtype=torch.bfloat16, seed=0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.fine, self.coarse = (nlat, 2 * nlat), (nlat // 2, nlat)
        self.heads, self.dim, C = heads, dim, heads * dim
        # fine -> coarse forward, coarse -> fine transposed, the same filter pairs
        cutoff = 3 * math.pi / (nlat // 2)
        self.plan = disco.Plan(*self.fine, *self.coarse, cutoff, backward=True)
        # A filter's basis functions integrate to about the square of their node
        # spacing: with this gain weights of order one give outputs of order one.
        self.gain = (3.0 / cutoff) ** 2

        def weight(*shape, fan):
            return (torch.randn(shape, generator=g, device=device) / math.sqrt(fan)).to(dtype)

        self.w = {"encode": weight(C, 4, 9, fan=36), "decode": weight(C, 4, 9, fan=9 * C),
                  "kv": weight(C, 2 * C, fan=C), "ask": weight(C, C, fan=C),
                  "q_norm": torch.ones(dim, device=device, dtype=dtype),
                  "k_norm": torch.ones(dim, device=device, dtype=dtype)}
        self.asks = torch.randn((self.coarse[0] * self.coarse[1], C), generator=g, device=device).to(dtype)
        self.tables = attention.grid_rotation(*self.coarse, dim, device=device)
        colat = math.pi * (torch.arange(self.coarse[0], device=device) + 0.5) / self.coarse[0]
        self.area = torch.log(torch.sin(colat)).repeat_interleave(self.coarse[1])  # [states], up to a constant

    def states(self, x):
        """Keys (normed and rotated) and values of the input x [B, 4, fine grid], with what the gradients need."""
        y = self.plan.forward(x, self.w["encode"] * self.gain)
        tokens = y.flatten(2).transpose(1, 2).contiguous()
        B, S, C = tokens.shape
        kv = (tokens.view(B * S, C) @ self.w["kv"]).view(B, S, 2, self.heads, self.dim)
        k = attention.norm_rotate(kv[:, :, 0], self.w["k_norm"], rotation=self.tables)
        return tokens, kv, k

    def bias(self, observed):
        """The states' log areas; -inf where nothing was observed (observed [B, states], bool)."""
        return self.area.expand(observed.shape).masked_fill(~observed, -math.inf).contiguous()

    def step(self, x, target, observed, rate=0.1, max_norm=1.0):
        """One step of gradient descent on the mean squared error; (loss, gradient norm) on the GPU."""
        w, B = self.w, x.shape[0]
        H, D, C = self.heads, self.dim, self.heads * self.dim
        tokens, kv, k = self.states(x)
        S, bias = tokens.shape[1], self.bias(observed)
        q0 = (self.asks @ w["ask"]).view(1, S, H, D).expand(B, S, H, D)
        q = attention.norm_rotate(q0, w["q_norm"], rotation=self.tables)
        out, stats = attention.cross_attention(q, k, kv[:, :, 1], key_bias=bias, return_stats=True)
        grid = out.view(B, S, C).transpose(1, 2).contiguous().view(B, C, *self.coarse)
        w_decode = w["decode"] * self.gain
        y = self.plan.transpose(grid, w_decode)
        diff = y.float() - target.float()
        loss = diff.square().mean()

        dy = (2.0 / diff.numel() * diff).to(y.dtype)
        dgrid, d_decode = disco.transpose_backward(self.plan, grid, w_decode, dy)
        dout = dgrid.flatten(2).transpose(1, 2).contiguous().view(B, S, H, D)
        dkv = torch.empty_like(kv)
        dq, dk, _ = attention.cross_attention_backward(q, k, kv[:, :, 1], out, stats, dout, key_bias=bias,
                                                       dv=dkv[:, :, 1])
        attention_dk, d_knorm = attention.norm_rotate_backward(kv[:, :, 0], w["k_norm"], dk, rotation=self.tables,
                                                               dx=dkv[:, :, 0])
        dq0, d_qnorm = attention.norm_rotate_backward(q0, w["q_norm"], dq, rotation=self.tables)
        dtok = (dkv.view(B * S, 2 * C) @ w["kv"].t().contiguous()).view(B, S, C)
        _, d_encode = disco.forward_backward(self.plan, x, w["encode"],
                                             dtok.transpose(1, 2).contiguous().view(B, C, *self.coarse),
                                             want_dx=False)
        grads = {"encode": d_encode * self.gain, "decode": d_decode * self.gain, "q_norm": d_qnorm, "k_norm": d_knorm,
                 "kv": tokens.view(B * S, C).t().contiguous() @ dkv.view(B * S, 2 * C),
                 "ask": self.asks.t().contiguous() @ dq0.float().sum(0).view(S, C).to(dq0.dtype)}
        norm, clipped = gradients.clip(list(grads.values()), max_norm)
        for name, g in zip(grads, clipped):
            w[name] -= rate * g
        return loss, norm

    def station(self, k, v, ask, places, observed):
        """Answers [B, n, C] of single places (cells `places`, int32 [n]) to queries ask [B, n, C]."""
        B, n, C = ask.shape
        q = (ask.reshape(B * n, C) @ self.w["ask"]).view(B, n, self.heads, self.dim)
        q = attention.norm_rotate(q, self.w["q_norm"], rotation=self.tables, positions=places)
        return attention.cross_attention(q, k, v, key_bias=self.bias(observed)).view(B, n, C)


def fields(batch, nlat, dtype, seed=1, device="cuda:0"):
    """Smooth fields [batch, 4, nlat, 2 nlat] around a mean of one."""
    g = torch.Generator(device=device).manual_seed(seed)
    colat = math.pi * (torch.arange(nlat, device=device) + 0.5)[:, None] / nlat
    lon = math.pi * torch.arange(2 * nlat, device=device)[None] / nlat
    a, b, c, s = torch.randn((4, batch, 4, 1, 1), generator=g, device=device)
    return (1.0 + 0.2 * a + b * colat.cos() + colat.sin() * (c * lon.cos() + s * lon.sin())).to(dtype)


def main():
    g = torch.Generator(device="cuda:0").manual_seed(1)
    model = GridAttention(nlat=32, dtype=torch.float32)
    x = fields(2, model.fine[0], torch.float32)
    target = torch.roll(x, 3, dims=3)
    states = model.coarse[0] * model.coarse[1]
    observed = torch.rand((2, states), generator=g, device="cuda:0") > 0.1
    for i in range(40):
        loss, norm = model.step(x, target, observed)
        print("step %2d  loss %.4f  gradient norm %.3f" % (i, float(loss), float(norm)), flush=True)
    _, kv, k = model.states(x)
    ask = torch.randn((2, 1, model.heads * model.dim), generator=g, device="cuda:0")
    answer = model.station(k, kv[:, :, 1], ask, torch.tensor([100], dtype=torch.int32, device="cuda:0"), observed)
    print("one station's answer:", tuple(answer.shape), "norm %.3f" % float(answer.float().norm()))


if __name__ == "__main__":
    main()
