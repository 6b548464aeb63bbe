"""The forecast example: runs in both types, its gradients against differences of its loss, one field at a time against
the whole series."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_training_step_runs(dtype):
    import torch
    from grid_forecast import GridForecast, waves
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    model = GridForecast(nlat=16, channels=24, dtype=dt)
    f = waves(2, 5, 16, dt)
    for _ in range(2):
        loss, norm = model.step(f[:, :-1], f[:, -1])
        assert bool(torch.isfinite(loss)) and bool(torch.isfinite(norm)) and float(norm) > 0
    assert all(bool(torch.isfinite(v).all()) for v in model.w.values())


def test_gradients_against_differences():
    """fp32 central differences: a step of 1e-2 along a direction of unit entries, truncation of its square, and the
    loss's own rounding (some 1e-7 of it) over the step."""
    import torch
    from grid_forecast import GridForecast, waves
    model = GridForecast(nlat=16, channels=16, dtype=torch.float32)
    f = waves(1, 4, 16, torch.float32)
    loss, grads = model.gradients(f[:, :-1], f[:, -1])
    g = torch.Generator(device="cuda:0").manual_seed(3)
    for name, grad in grads.items():
        d = torch.randn(grad.shape, generator=g, device="cuda:0")
        d /= d.norm()
        kept, size = model.w[name], 1e-2
        ends = []
        for s in (size, -size):
            model.w[name] = kept + s * d
            ends.append(float(model.gradients(f[:, :-1], f[:, -1])[0].double()))
        model.w[name] = kept
        diff, want = (ends[0] - ends[1]) / (2 * size), float((grad.double() * d.double()).sum())
        assert abs(diff - want) <= 1e-2 * float(grad.double().norm()) + 1e-6 * float(loss) / size, name


def test_one_field_at_a_time_is_the_series():
    """fp32, without dropout: the same arithmetic but for where runs of 16 steps begin: 1e-5."""
    import torch
    from grid_forecast import GridForecast, waves
    model = GridForecast(nlat=16, channels=20, dtype=torch.float32, drop=0.0)
    f = waves(2, 6, 16, torch.float32)[:, :-1]
    y, state, _ = model.block(model.series(f))
    whole = f[:, -1] + model.change(y[:, -1], 2)[0]
    s = None
    for t in range(f.shape[1]):
        following, s = model.advance(f[:, t], s)
    for a, b in ((following, whole), (s, state)):
        assert float((a - b).double().norm()) <= 1e-5 * float(b.double().norm())
