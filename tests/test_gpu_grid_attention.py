"""The example model runs the new operators with the DISCO layers: its step's gradients agree with automatic
differentiation of a plain fp32 form, its loss falls, and its single-place answers agree with the whole grid's."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


def _model(dtype):
    import torch
    from grid_attention import GridAttention, fields
    model = GridAttention(nlat=16, heads=2, dim=16, dtype=dtype)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    x = fields(2, model.fine[0], dtype)
    observed = torch.rand((2, model.coarse[0] * model.coarse[1]), generator=g, device="cuda:0") > 0.1
    return model, x, torch.roll(x, 1, dims=3), observed


def test_the_loss_falls():
    import torch
    model, x, target, observed = _model(torch.float32)
    losses = [float(model.step(x, target, observed)[0]) for _ in range(40)]
    print("loss %.4f -> %.4f" % (losses[0], losses[-1]))
    assert all(math.isfinite(v) for v in losses) and losses[-1] < 0.95 * losses[0]


def test_gradients_against_automatic_differentiation():
    """fp32: the attention and projection gradients of one step, from the change of the weights; the step's clipping is
    switched off by a limit far above the norm."""
    import torch
    model, x, target, observed = _model(torch.float32)
    before = {k: v.clone() for k, v in model.w.items()}
    w = {k: v.double().requires_grad_(True) for k, v in before.items()}
    H, D, C = model.heads, model.dim, model.heads * model.dim
    y = model.plan.forward(x, before["encode"] * model.gain)
    tokens = y.flatten(2).transpose(1, 2).double()
    B, S, _ = tokens.shape
    cos, sin = (t.double() for t in model.tables)

    def norm_rotate(t, weight):
        t = t / (t.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * weight
        a, b = t[..., :D // 2], t[..., D // 2:]
        c, s = cos[None, :, None], sin[None, :, None]
        return torch.cat((a * c - b * s, a * s + b * c), -1)

    kv = (tokens @ w["kv"]).view(B, S, 2, H, D)
    k = norm_rotate(kv[:, :, 0], w["k_norm"])
    q = norm_rotate((model.asks.double() @ w["ask"]).view(1, S, H, D), w["q_norm"]).expand(B, S, H, D)
    scores = torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(D)
    p = torch.softmax(scores + model.bias(observed).double()[:, None, None], -1)
    out = torch.matmul(p, kv[:, :, 1].transpose(1, 2).contiguous()).transpose(1, 2).reshape(B, S, C)
    grid = out.transpose(1, 2).reshape(B, C, *model.coarse)
    # the transposed op's own gradient is taken as it is: its input gradient starts the chain
    grid32 = grid.detach().float().contiguous()
    y2 = model.plan.transpose(grid32, before["decode"] * model.gain)
    dy = 2.0 / y2.numel() * (y2 - target)
    from paper_2209_13603_amd import disco
    dgrid, _ = disco.transpose_backward(model.plan, grid32, before["decode"] * model.gain, dy)
    names = ["kv", "ask", "q_norm", "k_norm"]
    want = torch.autograd.grad(grid, [w[n] for n in names], dgrid.double())
    model.step(x, target, observed, rate=1.0, max_norm=1e9)
    for n, g in zip(names, want):
        got = (before[n] - model.w[n]).double()
        # the change of a weight of size up to 2 resolves 2^-23 of it
        err = float((got - g).norm())
        assert err <= 2e-4 * float(g.norm()) + 2.0 ** -22 * math.sqrt(g.numel()), (n, err, float(g.norm()))


def test_single_places_agree_with_the_grid():
    import torch
    from paper_2209_13603_amd import attention
    model, x, _, observed = _model(torch.bfloat16)
    _, kv, k = model.states(x)
    S = k.shape[1]
    places = torch.tensor([0, 5, S - 1], dtype=torch.int32, device="cuda:0")
    ask = model.asks[places.long()][None].expand(2, 3, -1)
    got = model.station(k, kv[:, :, 1], ask, places, observed)
    q = (model.asks @ model.w["ask"]).view(1, S, model.heads, model.dim).expand(2, S, model.heads, model.dim)
    q = attention.norm_rotate(q, model.w["q_norm"], rotation=model.tables)
    whole = attention.cross_attention(q, k, kv[:, :, 1], key_bias=model.bias(observed)).view(2, S, -1)
    want = whole[:, places.long()]
    assert float((got.float() - want.float()).norm()) <= 2.0 ** -7 * float(want.float().norm())


def test_workspace_of_the_library():
    """The C entries with no workspace given take one of the stream-ordered pool, and refuse one that is too small."""
    import ctypes
    import torch
    from paper_2209_13603_amd import attention, disco
    lib = disco.library()
    g = torch.Generator(device="cuda:0").manual_seed(5)
    q = torch.randn((1, 1, 4, 64), generator=g, device="cuda:0").bfloat16()
    kv = torch.randn((1, 5000, 2, 1, 64), generator=g, device="cuda:0").bfloat16()
    k, v = kv[:, :, 0], kv[:, :, 1]
    want = attention.cross_attention(q, k, v)
    out = torch.zeros_like(q)
    h = [attention._heads(t, "t") for t in (q, k, v, out)]
    stream = torch.cuda.current_stream().cuda_stream
    need = ctypes.c_size_t()
    assert lib.disco_cross_attention_workspace(h[0], h[1], 0, need) == disco.DISCO_OK and need.value > 0
    assert lib.disco_cross_attention(h[0], h[1], h[2], None, h[3], None, None, None, 0, stream) == disco.DISCO_OK
    torch.cuda.synchronize()
    assert bool((out == want).all())
    small = torch.empty(256, dtype=torch.uint8, device="cuda:0")
    out.fill_(7.0)
    assert lib.disco_cross_attention(h[0], h[1], h[2], None, h[3], None, None, small.data_ptr(), 256, stream) == \
        disco.DISCO_ERR_INVALID_ARGUMENT
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
