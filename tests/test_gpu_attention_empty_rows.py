"""Queries that no key is left for give zeros and zero gradients, whatever they and their output gradients hold, however
their keys were taken out; the other batch items keep their bits."""
import math

import pytest

from test_gpu_attention import _dt, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [36, 64, 128])
@pytest.mark.parametrize("sizes", [(1, 3000), (40, 70), (300, 20), (1, 1)])
@pytest.mark.parametrize("mask", ["bias", "lengths", "both"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, 1.0])
def test_rows_without_keys(bad, mask, sizes, dim, dtype):
    import torch
    Sq, Sk = sizes
    g = torch.Generator(device="cuda:0").manual_seed(1)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda:0").to(_dt(dtype))
    q, k, v, dout = mk(3, Sq, 4, dim), mk(3, Sk, 2, dim), mk(3, Sk, 2, dim), mk(3, Sq, 4, dim)
    bias = torch.zeros(3, Sk, device="cuda:0") if mask != "lengths" else None
    lengths = torch.full((3,), Sk, dtype=torch.int32, device="cuda:0") if mask != "bias" else None
    want = _run(q, k, v, dout, key_bias=bias, key_lengths=lengths)
    if mask == "bias":
        bias[1] = -math.inf
    elif mask == "lengths":
        lengths[1] = 0
    else:  # the first half by one, the rest by the other
        lengths[1] = (Sk + 1) // 2
        bias[1, :(Sk + 1) // 2] = -math.inf
    for t in (q, k, v, dout):
        t[1, ::2] *= bad
    got = _run(q, k, v, dout, key_bias=bias, key_lengths=lengths)
    for name, a, b in zip(("out", "dq", "dk", "dv"), got, want):
        assert not a[1].any(), name
        assert bool((a[::2] == b[::2]).all()), name
