"""One training step, and one more time step, of a small forecast of fields on the sphere.

A DISCO layer halves the grid of every field of a series; each coarse cell's channels are
then a series in time.  The cell's series goes through a block of a network: its norm, one
projection to values and gates, a gated recurrence along time, and the residual sum with the norm
after the block, its gate, dropout and the next norm.  The transposed DISCO op takes the
last step's channels back to the input grid as the change of the next field.  The step's gradients,
DISCO weights among them, are clipped by their global norm.  ``advance`` takes one more
field and the cells' states, as a served model does.

    python examples/grid_forecast.py
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2209_13603_amd import blocks, disco, gradients, recurrence  # noqa: E402


class GridForecast:
    def __init__(self, nlat=32, channels=64, dtype=torch.bfloat16, drop=0.1, seed=0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.fine, self.coarse = (nlat, 2 * nlat), (nlat // 2, nlat)
        self.cells, self.C, self.drop, self.seed, self.steps = self.coarse[0] * self.coarse[1], channels, drop, seed, 0
        cutoff = 3 * math.pi / (nlat // 2)
        self.plan = disco.Plan(*self.fine, *self.coarse, cutoff, backward=True)
        self.gain = (3.0 / cutoff) ** 2  # outputs of order one (see grid_attention.py)
        C = channels

        def weight(*shape, fan):
            return (torch.randn(shape, generator=g, device=device) / math.sqrt(fan)).to(dtype)

        one = lambda v=1.0: torch.full((C,), v, device=device, dtype=dtype)
        self.w = {"encode": weight(C, 4, 9, fan=36), "decode": 0.3 * weight(C, 4, 9, fan=9 * C), "in_norm": one(),
                  "mix": weight(C, 3 * C, fan=C), "post": one(), "gate": one(0.5), "next": one()}

    def series(self, fields):
        """[B, T, 4, fine grid] -> every cell's series [B cells, T, C]."""
        B, T = fields.shape[:2]
        y = self.plan.forward(fields.flatten(0, 1).contiguous(), self.w["encode"] * self.gain)
        return y.view(B, T, self.C, self.cells).permute(0, 3, 1, 2).contiguous().view(B * self.cells, T, self.C)

    def block(self, x, state=None, dropout=None):
        """(y, state, what the gradients need) of the series x [N, T, C]."""
        N, T, C = x.shape
        _, u = blocks.residual_norm(None, x, next_weight=self.w["in_norm"], want_h=False)
        joint = (u.view(N * T, C) @ self.w["mix"]).view(N, T, 3, C)
        v, forget, out = joint.unbind(2)  # read where they lie
        f, state, carries = recurrence.gated_recurrence(v, forget, out_gate=out, state=state, return_carries=True)
        _, y = blocks.residual_norm(x, f, want_h=False, **self.sums(dropout))
        return y, state, (u, joint, f, carries)

    def sums(self, dropout):
        return dict(post_norm=True, post_weight=self.w["post"], gate=self.w["gate"], next_weight=self.w["next"],
                    dropout=dropout)

    def change(self, last, B):
        """The next field's change from the last step's channels [B cells, C], and the grid it comes from."""
        grid = last.view(B, self.cells, self.C).transpose(1, 2).contiguous().view(B, self.C, *self.coarse)
        return self.plan.transpose(grid, self.w["decode"] * self.gain), grid

    def gradients(self, fields, target):
        """(loss, gradients by name) of the mean squared error of the field after `fields` [B, T, 4, fine grid]."""
        w, (B, T), C = self.w, fields.shape[:2], self.C
        drop = blocks.Dropout(self.drop, self.seed, self.steps) if self.drop else None
        x = self.series(fields)
        y, _, (u, joint, f, carries) = self.block(x, dropout=drop)
        change, grid = self.change(y[:, -1], B)
        diff = fields[:, -1].float() + change.float() - target.float()

        dchange = (2.0 / diff.numel() * diff).to(change.dtype)
        dgrid, d_decode = disco.transpose_backward(self.plan, grid, w["decode"] * self.gain, dchange)
        dy = torch.zeros_like(y)
        dy[:, -1] = dgrid.flatten(2).transpose(1, 2).reshape(B * self.cells, C)
        top = blocks.residual_norm_backward(x, f, None, dy, **self.sums(drop))
        v, forget, out = joint.unbind(2)
        djoint = torch.empty_like(joint)
        dv, dforget, dout = djoint.unbind(2)
        recurrence.gated_recurrence_backward(v, forget, carries, top.df, out_gate=out, dx=dv, dgate=dforget, dout_gate=dout,
                                             want_dstate=False)
        flat = djoint.view(-1, 3 * C)
        du = (flat @ w["mix"].t().contiguous()).view_as(u)
        low = blocks.residual_norm_backward(None, x, None, du, next_weight=w["in_norm"])
        dx = (top.dx + low.df).view(B, self.cells, T, C).permute(0, 2, 3, 1).contiguous().view(B * T, C, *self.coarse)
        _, d_encode = disco.forward_backward(self.plan, fields.flatten(0, 1).contiguous(), w["encode"], dx, want_dx=False)
        return diff.square().mean(), {
            "encode": d_encode * self.gain, "decode": d_decode * self.gain, "in_norm": low.dnext_weight,
            "mix": u.view(-1, C).t().contiguous() @ flat, "post": top.dpost_weight, "gate": top.dgate,
            "next": top.dnext_weight}

    def step(self, fields, target, rate=0.1, max_norm=1.0):
        """One step of gradient descent; (loss, gradient norm) on the GPU."""
        loss, grads = self.gradients(fields, target)
        norm, clipped = gradients.clip(list(grads.values()), max_norm)
        for name, g in zip(grads, clipped):
            self.w[name] -= rate * g
        self.steps += 1
        return loss, norm

    def advance(self, field, state=None):
        """(next field, state) from one more field [B, 4, fine grid] and the cells' states (None at the start)."""
        B = field.shape[0]
        y, state, _ = self.block(self.series(field[:, None]), state)
        return field + self.change(y[:, -1], B)[0], state


def waves(batch, steps, nlat, dtype, seed=1, device="cuda:0"):
    """Fields [batch, steps + 1, 4, nlat, 2 nlat] that turn with the longitude, each at its own speed."""
    g = torch.Generator(device=device).manual_seed(seed)
    colat = (math.pi * (torch.arange(nlat, device=device) + 0.5) / nlat)[:, None]
    lon = (math.pi * torch.arange(2 * nlat, device=device) / nlat)[None]
    t = torch.arange(steps + 1, device=device)[:, None, None, None]
    speed, phase = torch.rand((2, batch, 1, 4, 1, 1), generator=g, device=device)
    return (colat.sin() * torch.cos(lon - 0.3 * (1 + speed) * t - 6.3 * phase)).to(dtype)


def main():
    model = GridForecast(dtype=torch.float32)
    f = waves(2, 8, model.fine[0], torch.float32)
    for i in range(40):
        loss, norm = model.step(f[:, :-1], f[:, -1], rate=0.02)
        print("step %2d  loss %.4f  gradient norm %.3f" % (i, float(loss), float(norm)), flush=True)
    state = None
    for t in range(8):
        following, state = model.advance(f[:, t], state)
    print("next field:", tuple(following.shape), "error %.4f" % float((following - f[:, -1]).square().mean()))


if __name__ == "__main__":
    main()
