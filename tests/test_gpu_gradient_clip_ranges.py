"""Clipping where the norm, the limit or their quotient leaves the range of fp32.

Finite gradients have a finite norm in 64 bits, up to 3.4e38 times the root of their number, and the factor is a quotient of
64-bit values: a clipped value is right to two roundings to fp32 (4e-7 as in test_gpu_gradient_clip.py, 4.1e-3 in bf16)
and two of the smallest fp32 value (1.4e-45), whatever leaves the range on the way.  The returned norm is rounded to fp32
(infinity beyond it)."""
import math

import pytest

pytestmark = pytest.mark.gpu


def _run(scale, sizes, dtype, max_norm, eps):
    import torch
    from paper_2209_13603_amd import gradients
    g = torch.Generator(device="cuda:0").manual_seed(1)
    grads = [(scale * (torch.rand(n, generator=g, device="cuda:0") - 0.5).double()).to(dtype) for n in sizes]
    norm, out = gradients.clip(grads, max_norm, eps=eps, out=[torch.empty_like(t) for t in grads])
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    c = min(1.0, max_norm / (want + eps))
    got = float(norm)
    assert math.isinf(got) if want > 3.5e38 else abs(got - want) <= 1.2e-7 * want + 1.5e-45
    tol = 4.1e-3 if dtype == torch.bfloat16 else 4e-7
    least = 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149
    for a, b in zip(grads, out):
        ref = a.double() * c
        assert bool(((b.double() - ref).abs() <= tol * ref.abs() + 2 * least).all()), float((b.double() - ref).abs().max())
    return want


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sizes", [[100, 7], [200001, 3, 70000]])
@pytest.mark.parametrize("scale,max_norm,eps", [
    (3e38, 1.0, 1e-6),       # the norm is beyond fp32
    (3e38, 1e36, 0.0),
    (3e38, 1e-6, 0.0),       # and the factor below its normal values
    (1e38, 1e39, 0.0),       # the limit too
    (1.0, 1e-40, 1e-6),      # a limit below the normal values
    (1e-30, 1e-35, 0.0), (1e-30, 1e-35, 1e-45), (1e-36, 1e30, 1e-50), (1e-20, 1e-22, 1e300),
])
def test_factors_out_of_range(scale, max_norm, eps, sizes, dtype):
    import torch
    want = _run(scale, sizes, {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype], max_norm, eps)
    print(want)


def test_no_limit():
    """An infinite limit leaves finite gradients as they are, whatever their norm."""
    import torch
    from paper_2209_13603_amd import gradients
    for n in (50, 100000):
        t = torch.full((n,), 3e38, device="cuda:0")
        norm, out = gradients.clip([t], math.inf, out=[torch.empty_like(t)])
        assert math.isinf(float(norm)) and bool((out[0] == t).all())
