"""Cross attention where scores and biases are large beside what 32 bits hold of them: masks of -1e10 and the like,
single keys far above the others, and scores of 1e10 without a bias, forward and gradients.

What such a softmax is follows from the definition with the scores as fp32 holds them: a bias whose spacing is above
every product of q and k leaves nothing of those, so that keys of one such bias weigh alike; keys below the largest
score by more than the exponential's range weigh nothing; equal keys weigh the same.  `_weighted` takes those weights'
logarithms and computes the rest in 64 bits.  Tolerances: those of test_gpu_attention.py.  Where a single key
has all of the weight, the scores' gradient is the difference of two sums of the same D products, out
(held to 2^-17 with its remainder, fp32 2^-24) times dout and v times dout: nothing but rounding, below 1e-3 for
entries of order one.
"""
import math

import pytest

from test_gpu_attention import TOL, _close, _dt, _run

pytestmark = pytest.mark.gpu

BIG = [-1e9, -1e10, -1e12, -1e20, -1e30, 1e10, 1e20]
DIMS = [16, 36, 64, 100, 128]


def _weighted(q, k, v, dout, logits, scale):
    """(out, dq, dk, dv) with the sums of their terms' squares, for softmax weights of `logits` [B, H, Sq, Sk]."""
    import torch
    B, Sq, H, D = q.shape
    G = H // k.shape[2]
    q, k, v, dout = (t.detach().cpu().double() for t in (q, k, v, dout))
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    out, dq = torch.zeros_like(q), torch.zeros_like(q)
    sq = [torch.zeros_like(t) for t in (out, dq, dk, dv)]
    for b in range(B):
        for h in range(H):
            kk, vv, qq, g = k[b, :, h // G], v[b, :, h // G], q[b, :, h], dout[b, :, h]
            p = torch.softmax(logits[b, h].cpu().double(), 1)
            o = p @ vv
            ds = p * (g @ vv.t() - (g * o).sum(1, keepdim=True)) * scale
            out[b, :, h], dq[b, :, h] = o, ds @ kk
            dk[b, :, h // G] += ds.t() @ qq
            dv[b, :, h // G] += p.t() @ g
            sq[0][b, :, h], sq[1][b, :, h] = (p * p) @ (vv * vv), (ds * ds) @ (kk * kk)
            sq[2][b, :, h // G] += (ds * ds).t() @ (qq * qq)
            sq[3][b, :, h // G] += (p * p).t() @ (g * g)
    return list(zip((out, dq, dk, dv), sq))


def _make(B, Sq, Sk, H, Hk, D, dtype, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g)
    return [t.to("cuda:0", _dt(dtype)) for t in (1.5 * rnd(B, Sq, H, D), rnd(B, Sk, Hk, D), rnd(B, Sk, Hk, D), rnd(B, Sq, H, D))]


def _scores(q, k, scale):
    import torch
    B, Sq, H, D = q.shape
    kk = k.cpu().double().repeat_interleave(H // k.shape[2], 2).permute(0, 2, 3, 1).contiguous()
    return torch.matmul(q.cpu().double().transpose(1, 2).contiguous(), kk) * scale


# queries, keys: many rows; one row with its keys in parts (whole parts of which have the bias)
SIZES = [(150, 200), (1, 3000)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("value", BIG)
def test_every_key_with_one_large_bias(value, sizes, dim, dtype):
    import torch
    Sq, Sk = sizes
    q, k, v, dout = _make(2, Sq, Sk, 4, 2, dim, dtype, 1)
    bias = torch.full((Sk,), value, device="cuda:0")
    want = _weighted(q, k, v, dout, torch.zeros(2, 4, Sq, Sk), 1 / math.sqrt(dim))
    for name, a, b in zip(("out", "dq", "dk", "dv"), _run(q, k, v, dout, key_bias=bias), want):
        _close(name, a, b, TOL[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("value", [-2e3, -3e3, -1e4, 1e4, -1e5])
def test_every_key_with_one_bias_that_leaves_the_scores(value, sizes, dim, dtype):
    """Every product added onto such a bias rounds to its spacing: scores off by up to half of it, 2^-24 |bias|, a step
    of which there are up to eight in bf16 and three, the product with the scale and the reference among them, in fp32;
    weights, and what they sum, by as much relatively."""
    import torch
    Sq, Sk = sizes
    q, k, v, dout = _make(2, Sq, Sk, 4, 2, dim, dtype, 8)
    scale = 1 / math.sqrt(dim)
    want = _weighted(q, k, v, dout, _scores(q, k, scale), scale)
    tol = TOL[dtype] + 8 * abs(value) * 2.0 ** -24
    for name, a, b in zip(("out", "dq", "dk", "dv"), _run(q, k, v, dout, key_bias=torch.full((Sk,), value, device="cuda:0")), want):
        _close(name, a, b, tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("value", [b for b in BIG if b < 0] + ["lowest"])
@pytest.mark.parametrize("where", ["first", "last", "middle"])
def test_some_keys_masked_by_a_large_bias(where, value, sizes, dim, dtype):
    """Whole tiles and parts of the split of which no key is left; the others as if those were not there."""
    import torch
    Sq, Sk = sizes
    value = torch.finfo(torch.float32).min if value == "lowest" else value
    q, k, v, dout = _make(2, Sq, Sk, 4, 2, dim, dtype, 2)
    bias = torch.randn(Sk, generator=torch.Generator(device="cuda:0").manual_seed(3), device="cuda:0")
    lo, hi = {"first": (0, Sk // 2 + 3), "last": (Sk // 2, Sk), "middle": (Sk // 4, Sk - 7)}[where]
    bias[lo:hi] = value
    scale = 1 / math.sqrt(dim)
    want = _weighted(q, k, v, dout, _scores(q, k, scale) + bias.cpu().double(), scale)
    for name, a, b in zip(("out", "dq", "dk", "dv"), _run(q, k, v, dout, key_bias=bias), want):
        _close(name, a, b, TOL[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [36, 64, 128])
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("value", [1e9, 1e10, 1e20, "largest"])
def test_one_key_far_above_the_others(value, sizes, dim, dtype):
    import torch
    Sq, Sk = sizes
    value = torch.finfo(torch.float32).max if value == "largest" else value
    q, k, v, dout = _make(2, Sq, Sk, 4, 2, dim, dtype, 4)
    bias = torch.zeros(Sk, device="cuda:0")
    bias[Sk // 2] = value
    out, dq, dk, dv = _run(q, k, v, dout, key_bias=bias)
    want = v[:, Sk // 2].repeat_interleave(2, 1)[:, None].expand_as(out)
    assert bool((out == want).all())
    assert float(dq.float().abs().max()) <= 1e-3 and float(dk.float().abs().max()) <= 1e-3 * math.sqrt(2 * Sq)
    sums = dout.float().sum(1).view(2, 2, 2, dim).sum(2)
    assert float((dv[:, Sk // 2].float() - sums).norm()) <= 2.0 ** -8 * float(sums.norm())
    rest = torch.cat((dv[:, :Sk // 2], dv[:, Sk // 2 + 1:]), 1)
    assert not rest.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("size", [4e3, 1e5, 1e8])
@pytest.mark.parametrize("scale", [None, -0.3])
def test_large_scores_without_a_bias(scale, size, sizes, dim, dtype):
    """Every key twice, far apart: the two that score highest share the weight, to the last bit, in all three passes."""
    import torch
    Sq, Sk = sizes
    q, k, v, dout = _make(2, Sq, Sk, 4, 2, dim, dtype, 5)
    q, k = (q.float() * size).to(q.dtype), (k.float() * size).to(k.dtype)
    k[:, Sk // 2:] = k[:, :Sk // 2]
    s = _scores(q, k, 1 / math.sqrt(dim) if scale is None else scale)
    top = s.topk(3, dim=-1).values
    # the next key is below them by more than fp32 rounds and the exponential reaches
    gap = top[..., 0] - top[..., 2]
    assert float((gap / s.abs().amax(-1)).min()) > 2.0 ** -19 and float(gap.min()) > 150
    out, dq, dk, dv = _run(q, k, v, dout, scale=scale)
    want = _weighted(q, k, v, dout, s, 1 / math.sqrt(dim) if scale is None else scale)
    _close("out", out, want[0], TOL[dtype])
    _close("dv", dv, want[3], TOL[dtype])
    for name, a, b in (("dq", dq, want[1]), ("dk", dk, want[2])):
        _close(name, a, b, TOL[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_rows_beside_ordinary_ones(dtype):
    """Rows of ordinary scores are what they are without the large rows of their tile."""
    import torch
    q, k, v, dout = _make(1, 64, 300, 2, 2, 64, dtype, 6)
    big = q.clone()
    big[:, ::3] = (big[:, ::3].float() * 1e9).to(q.dtype)
    scale = 1 / 8
    want = _weighted(q, k, v, dout, _scores(q, k, scale), scale)
    out, dq, dk, dv = _run(big, k, v, dout)
    rows = [i for i in range(64) if i % 3]
    for name, a, b in (("out", out, want[0]), ("dq", dq, want[1])):
        _close(name, a[:, rows], (b[0][:, rows], b[1][:, rows]), TOL[dtype])
    assert all(bool(torch.isfinite(t.float()).all()) for t in (out, dq, dk, dv))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("queries", [1, 40])
def test_infinite_and_nan_biases(queries, dtype):
    """+inf and NaN give NaN in their batch item; the other item keeps its bits."""
    import torch
    from paper_2209_13603_amd import attention
    q, k, v, _ = _make(2, queries, 700, 2, 2, 64, dtype, 7)
    bias = torch.zeros(2, 700, device="cuda:0")
    ref = attention.cross_attention(q, k, v, key_bias=bias)
    for bad in (math.inf, math.nan):
        b = bias.clone()
        b[1, 650] = bad
        got = attention.cross_attention(q, k, v, key_bias=b)
        assert bool((got[0] == ref[0]).all()) and bool(torch.isnan(got[1].float()).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [1e-20, -1e10])
@pytest.mark.parametrize("queries", [1, 40])
def test_lowest_biases_at_scales_out_of_the_ordinary(queries, scale, dtype):
    import torch
    q, k, v, dout = _make(1, queries, 3000, 2, 1, 64, dtype, 9)
    bias = torch.full((3000,), torch.finfo(torch.float32).min, device="cuda:0")
    want = _weighted(q, k, v, dout, torch.zeros(1, 2, queries, 3000), scale)
    for name, a, b in zip(("out", "dq", "dk", "dv"), _run(q, k, v, dout, key_bias=bias, scale=scale), want):
        _close(name, a, b, TOL[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("queries", [1, 40])
@pytest.mark.parametrize("low,high", [(-1e33, -1e31), (-1e36, -1e35), (1e31, 1e33), (1e35, 1e36)])
def test_the_larger_of_two_large_biases(low, high, queries, dtype):
    """Keys of one mask below keys of another, with no other key left: the larger bias takes all."""
    import torch
    q, k, v, dout = _make(1, queries, 3000, 2, 1, 64, dtype, 10)
    bias = torch.full((3000,), low, device="cuda:0")
    bias[1500:] = high
    logits = torch.full((1, 2, queries, 3000), -math.inf)
    logits[..., 1500:] = 0.0
    want = _weighted(q, k, v, dout, logits, 1 / 8)
    for name, a, b in zip(("out", "dq", "dk", "dv"), _run(q, k, v, dout, key_bias=bias), want):
        _close(name, a, b, TOL[dtype])
