"""Residual sums whose workgroups take several rows one after the other: more rows than the card holds at a time, in waves
and in whole workgroups, against the definition in 64 bits; the second norm of rows whose squares leave fp32.

Tolerances: those of test_gpu_residual.py (a relative 2-norm of 2e-6 beside bf16's rounding; 5e-6 for the gradients of weights,
whose terms cancel to their root: chains of some 90 roundings of 2^-24 at random add 6e-7 to what the terms have).
"""
import pytest

from block_forms import dropout_factor, rel

pytestmark = pytest.mark.gpu

TOL = {"bf16": 2.0 ** -8 + 2e-6, "fp32": 2e-6}
# A launch has at most 1280 workgroups of four waves, or 512 of a row: these are two to six rows a wave, the last round part full.
SHAPES = [(3, 3001, 1024), (3, 2500, 520), (2, 45011, 40), (3, 501, 4100), (2, 650, 8192), (2, 701, 4093)]


def _inputs(B, S, C, dtype, per_item):
    import torch
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    g = torch.Generator(device="cuda:0").manual_seed(B + 3 * S + 7 * C)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda:0")
    x, f, dh, dy = (rnd(B, S, C).mul(m).to(dt) for m in (2.0, 0.7, 1.0, 1.0))
    w = {k: (1 + 0.3 * rnd(*((B, C) if k in per_item else (C,)))).to(dt) for k in ("post_weight", "gate", "next_weight")}
    return x, f, dh, dy, w


def _exact(x, f, dh, dy, w, post, eps, factor):
    """[h, y, gradients of x, f and the weights that are there]"""
    import torch
    leaf = {k: t.double().requires_grad_(True) for k, t in dict(x=x, f=f, **w).items()}
    wide = lambda k: leaf[k][:, None] if leaf[k].dim() == 2 else leaf[k]
    norm = lambda v: v / (v.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    u = norm(leaf["f"]) * wide("post_weight") if post else leaf["f"]
    u = u * factor if factor is not None else u
    h = leaf["x"] + (u * wide("gate") if "gate" in w else u)
    y = norm(h) * wide("next_weight")
    total = (y * dy.double()).sum() if dh is None else (h * dh.double()).sum() + (y * dy.double()).sum()
    return [h.detach(), y.detach(), *torch.autograd.grad(total, list(leaf.values()))]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["dropped", "per_item"])
@pytest.mark.parametrize("shape", SHAPES)
def test_several_rows_a_workgroup(shape, kind, dtype):
    from paper_2209_13603_amd import blocks
    x, f, dh, dy, w = _inputs(*shape, dtype, ("gate", "post_weight") if kind == "per_item" else ())
    kw = dict(post_norm=True, dropout=blocks.Dropout(0.2, 9, 4) if kind == "dropped" else None, **w)
    factor = dropout_factor(shape, kw["dropout"]).cuda() if kw["dropout"] else None
    want = _exact(x, f, dh, dy, w, True, 1e-6, factor)
    h, y = blocks.residual_norm(x, f, **kw)
    g = blocks.residual_norm_backward(x, f, dh, dy, **kw)
    for n, u, v in zip(("h", "y", "dx", "df", "dpost_weight", "dgate", "dnext_weight"), (h, y, *g), want):
        assert rel(u, v) <= (5e-6 if dtype == "fp32" and "_w" in n or n == "dgate" and dtype == "fp32" else TOL[dtype]), n
    # over the inputs, while the next row's loads are out
    a, b = x.clone(), f.clone()
    blocks.residual_norm(a, b, h=a, y=b, **kw)
    assert bool((a == h).all()) and bool((b == y).all())
    a, b = x.clone(), f.clone()
    blocks.residual_norm(a, b, h=b, y=a, **kw)
    assert bool((b == h).all()) and bool((a == y).all())
    for place in ("gradients", "inputs", "crossed"):
        t = [v.clone() for v in (x, f, dh, dy)]
        dx, df = {"gradients": (t[2], t[3]), "inputs": (t[0], t[1]), "crossed": (t[3], t[0])}[place]
        again = blocks.residual_norm_backward(*t, dx=dx, df=df, **kw)
        for u, v in zip(again, g):
            assert bool((u == v).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("channels", [24, 96, 600, 2100, 8192])
def test_second_norm_of_rows_whose_squares_leave_fp32(channels, dtype):
    """Rows of ordinary size beside rows 1e18 times as large and as small, in one wave and one workgroup; eps 0.  Gradients
    come out as much smaller and larger: compared once each row is back at order one."""
    import torch
    from paper_2209_13603_amd import blocks
    x, f, _, dy, w = _inputs(2, 13, channels, dtype, ())
    size = torch.tensor([2.0 ** 60, 1.0, 2.0 ** -60, 1.0, 1.0, 2.0 ** -60, 2.0 ** 60], device="cuda:0").repeat(4)[:26].view(2, 13, 1)
    x, f = x * size.to(x.dtype), f * size.to(x.dtype)
    w = {"next_weight": w["next_weight"]}
    kw = dict(eps=0.0, **w)
    want = _exact(x, f, None, dy, w, False, 0.0, None)
    h, y = blocks.residual_norm(x, f, **kw)
    assert rel(h / size, want[0] / size) <= TOL[dtype] and rel(y, want[1]) <= TOL[dtype]
    g = blocks.residual_norm_backward(x, f, None, dy, **kw)
    for u, v in ((g.dx, want[2]), (g.df, want[3])):
        assert rel(u.float() * size, v * size) <= TOL[dtype]
        one = (size != 1).flatten()
        assert rel((u.float() * size).view(26, -1)[one], (v * size).view(26, -1)[one]) <= TOL[dtype]
    assert rel(g.dnext_weight, want[4]) <= (5e-6 if dtype == "fp32" else TOL[dtype])
