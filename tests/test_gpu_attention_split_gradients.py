"""Gradients of few keys for many queries, whose queries go to parts between workgroups: partial sums of dk and dv, and their
join, at every width of a row (16-byte pieces, 8-byte pieces, single entries), with fp32 heads whose last entries take the
vector unit, under lengths and holes.  Definition and tolerances: test_gpu_attention.py."""
import math

import pytest

from test_gpu_attention import TOL, _close, _dt, _exact, _run

pytestmark = pytest.mark.gpu

# batch, queries, keys, heads, kv heads, dim: at least 16 tiles of 32 queries for each kv head, so two parts or more
SHAPES = [
    (1, 1500, 20, 2, 2, 36), (1, 700, 5, 4, 1, 127), (2, 600, 33, 2, 2, 30), (1, 1030, 140, 3, 3, 37), (1, 513, 64, 4, 2, 100),
    (3, 800, 7, 2, 1, 68), (1, 2000, 1, 1, 1, 33), (1, 900, 50, 2, 2, 128), (2, 700, 40, 2, 1, 96),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("mask", ["none", "holes"])
def test_few_keys_for_many_queries(mask, shape, dtype):
    import torch
    B, Sq, Sk, H, Hk, D = shape
    assert -(-Sq // 32) * (H // Hk) >= 16
    g = torch.Generator(device="cuda:0").manual_seed(Sq)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda:0")
    q, dout = (1.5 * rnd(B, Sq, H, D)).to(_dt(dtype)), rnd(B, Sq, H, D).to(_dt(dtype))
    k, v = rnd(B, Sk, Hk, D).to(_dt(dtype)), rnd(B, Sk, Hk, D).to(_dt(dtype))
    bias = lengths = None
    if mask == "holes":
        lengths = torch.tensor([max(1, Sk - 3 * b) for b in range(B)], dtype=torch.int32, device="cuda:0")
        bias = rnd(B, Sk)
        gone = torch.rand((B, Sk), generator=g, device="cuda:0") < 0.3
        gone[:, 0] = False
        bias = bias.masked_fill(gone, -math.inf)
        k[gone] = float("nan")
        v[gone] = float("inf")
    want = _exact(q, k, v, dout, bias, lengths, 1 / math.sqrt(D))
    for name, a, b in zip(("out", "dq", "dk", "dv"), _run(q, k, v, dout, key_bias=bias, key_lengths=lengths), want):
        if Sk == 1 and name in ("dq", "dk"):  # one key: the scores' gradient is nothing but fp32 rounding
            assert float(a.float().abs().max()) <= 1e-3 * (math.sqrt(Sq) if name == "dk" else 1)
            continue
        _close(name, a, b, TOL[dtype])
