"""Gates far below 0: what they leave of a state keeps its own size, in every type of storage.

Everything that adds up is positive, so that a relative error holds entry by entry.  A step multiplies the state by an a whose
relative error is |g| 2^-24 for the product in the exponential, |g| 2^-25 for its constant and 2^-23 each for the exponential
and the quotient, beside two roundings of the step and one of the maps' joins: (2 |g| + 8) 2^-24 is more, and a state has
that of all the steps before it.  A bf16 output has a rounding of 2^-8 more.
"""
import pytest

from block_forms import recurrence as form

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gain", ["mean", "power", "one"])
@pytest.mark.parametrize("shape", [(2, 1, 6), (3, 24, 10), (2, 300, 64), (1, 300, 7), (1, 1500, 66), (60, 33, 2200)])
def test_closed_gates_leave_a_share_of_the_state(shape, gain, dtype):
    """Every eighth step nearly empties the state, and nothing comes in for four steps from there on."""
    import torch
    from paper_2209_13603_amd import recurrence
    B, T, C = shape
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    r = torch.Generator(device="cuda:0").manual_seed(B + 3 * T + 7 * C)
    at = torch.arange(T, device="cuda:0")
    g = torch.empty((B, T, C), device="cuda:0").uniform_(-2.0, 3.0, generator=r)
    g[:, at % 8 == 0] = torch.empty((B, int((at % 8 == 0).sum()), C), device="cuda:0").uniform_(-20.0, -8.0, generator=r)
    x = torch.empty((B, T, C), device="cuda:0").uniform_(0.5, 2.0, generator=r)
    x[:, at % 8 < 4] = 0.0
    g, x = g.to(dt), x.to(dt)
    state = torch.empty((B, C), device="cuda:0").uniform_(0.5, 2.0, generator=r)
    want_y, want = form(x, g, None, state, None, gain, device="cuda:0")
    bound = torch.cumsum(2 * g.double().abs() + 8, 1) * 2.0 ** -24
    y, last, carries = recurrence.gated_recurrence(x, g, state=state, gain=gain, return_carries=True)
    assert bool(((last - want).abs() <= bound[:, -1] * want).all())
    rounding = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert bool(((y - want_y).abs() <= (rounding + 1.01 * bound) * want_y).all())
    for i in (1, 7):
        if i < carries.shape[1]:
            before = form(x[:, :16 * i], g[:, :16 * i], None, state, None, gain, device="cuda:0")[1]
            assert bool(((carries[:, i] - before).abs() <= bound[:, 16 * i - 1] * before).all())


@pytest.mark.parametrize("gain", ["mean", "power", "one"])
@pytest.mark.parametrize("T", [20, 600])
@pytest.mark.parametrize("end", [float("inf"), 200.0])
def test_gates_at_their_ends_in_bf16(end, T, gain):
    """The lower end starts anew from x, the upper one holds the state, exactly; what comes before reaches nothing behind."""
    import torch
    from paper_2209_13603_amd import recurrence
    r = torch.Generator(device="cuda:0").manual_seed(T)
    x, g, dy = (torch.randn((2, T, 6), generator=r, device="cuda:0").bfloat16() for _ in range(3))
    state = torch.randn((2, 6), generator=r, device="cuda:0")
    g[:, T // 2] = -end
    g[:, T // 2 + 1:] = end
    y, last, carries = recurrence.gated_recurrence(x, g, state=state, gain=gain, return_carries=True)
    assert bool((y[:, T // 2] == x[:, T // 2]).all())
    if gain != "one":
        assert bool((y[:, T // 2:] == x[:, T // 2, None]).all()) and bool((last == x[:, T // 2].float()).all())
    dy[:, :T // 2] = 0.0
    cut = recurrence.gated_recurrence_backward(x, g, carries, dy, gain=gain)
    assert bool(torch.isfinite(cut.dgate).all()) and not cut.dstate.any() and not cut.dx[:, :T // 2].any()


def test_a_gate_that_is_not_a_number_shows():
    import torch
    from paper_2209_13603_amd import recurrence
    for T in (20, 600):
        for dtype in (torch.bfloat16, torch.float32):
            x, g = torch.ones((1, T, 4), device="cuda:0", dtype=dtype), torch.zeros((1, T, 4), device="cuda:0", dtype=dtype)
            g[0, T // 2, 1] = float("nan")
            for gain in ("mean", "power", "one"):
                y, last = recurrence.gated_recurrence(x, g, gain=gain)
                bad = torch.isnan(y[0])
                assert bool(bad[T // 2:, 1].all()) and int(bad.sum()) == T - T // 2 and bool(torch.isnan(last[0, 1]))
