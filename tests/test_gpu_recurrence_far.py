"""Recurrences over items too far apart for 32-bit offsets between them: scanned as near ones are, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(2, 40, 64), (3, 600, 66), (2, 300, 35), (2, 1100, 130)])
def test_items_far_apart(shape, dtype):
    import torch
    from paper_2209_13603_amd import recurrence
    B, T, C = shape
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    apart = 1 << (31 if dtype == "bf16" else 30)  # 4 GiB
    r = torch.Generator(device="cuda:0").manual_seed(T)
    rnd = lambda *s: torch.randn(s, generator=r, device="cuda:0")
    x, g, z, dy = (rnd(B, T, C).to(dt) for _ in range(4))
    state, dstate = rnd(B, C), rnd(B, C)
    lengths = torch.tensor([T, T // 2, 3][:B], dtype=torch.int32, device="cuda:0")
    big = torch.empty((B - 1) * apart + 6 * T * C, dtype=dt, device="cuda:0")

    def far(i, t):
        place = big.as_strided((B, T, C), (apart, 6 * C, 1), i * C)
        place.copy_(t)
        return place

    for gate in (None, z):
        kw = dict(lengths=lengths, gain="power")
        y, last, carries = recurrence.gated_recurrence(x, g, out_gate=gate, state=state, return_carries=True, **kw)
        grads = recurrence.gated_recurrence_backward(x, g, carries, dy, out_gate=gate, dstate=dstate, **kw)
        big[:6 * T * C] = 7.0
        fx, fg, fz, fd = far(0, x), far(1, g), far(2, z) if gate is not None else None, far(3, dy)
        y2, last2, carries2 = recurrence.gated_recurrence(fx, fg, out_gate=fz, state=state, return_carries=True, y=far(4, x), **kw)
        assert bool((y2 == y).all()) and bool((last2 == last).all()) and bool((carries2 == carries).all())
        dz = dict(dout_gate=fz) if gate is not None else {}
        got = recurrence.gated_recurrence_backward(fx, fg, carries2, fd, out_gate=fz, dstate=dstate, dx=fd, dgate=fg, **dz, **kw)
        for u, v in zip(got, grads):
            assert v is None or bool((u == v).all())
        assert bool((fx == x).all()) and bool((big.as_strided((T, C), (6 * C, 1), 5 * C) == 7).all())
