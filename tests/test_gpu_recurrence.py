"""Gated recurrence along time and its gradients against the definition in 64 bits, step by step.

Tolerances: relative 2-norm.  bf16 has one rounding (at most 2^-8) beside what fp32 has: two roundings of 2^-24 of the state
a step, which its memory of at most 1 / (1 - a) = 150 steps (gates up to 5) adds up in the worst case (1.8e-5) and by the root
in the usual one (1.5e-6), and a gate's share |q| that is off by |g| 2^-24 + 3 x 2^-24 (exponential and quotient): 1e-6.  So 3e-6; for the gradients,
products of two such, 6e-6.
"""
import pytest

from block_forms import recurrence as form
from block_forms import rel

pytestmark = pytest.mark.gpu

TOL = {"bf16": 2.0 ** -8, "fp32": 0.0}
# steps from one to several tiles of each way of working, channels odd and even, whole blocks of 64 and not
SHAPES = [(1, 1, 1), (2, 1, 64), (3, 2, 5), (2, 15, 6), (2, 16, 7), (1, 17, 130), (5, 32, 10), (2, 33, 4), (1, 127, 64), (3, 128, 66),
          (2, 129, 3), (1, 300, 65), (2, 512, 30), (1, 1500, 70), (3, 1100, 64), (1, 2600, 2)]


def _inputs(B, T, C, dtype, seed=0):
    import torch
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    r = torch.Generator(device="cuda:0").manual_seed(seed + B + 3 * T + 7 * C)
    rnd = lambda *s: torch.randn(s, generator=r, device="cuda:0")
    x, z, dy = (rnd(B, T, C).to(dt) for _ in range(3))
    g = (rnd(B, T, C) + torch.linspace(-1, 4, C, device="cuda:0")).clamp(max=5.0).to(dt)
    return x, g, z, dy, rnd(B, C), rnd(B, C)


def _all(x, g, z, dy, state, dstate, dtype, gain="mean", lengths=None, device="cpu", **places):
    from paper_2209_13603_amd import recurrence
    want = form(x, g, z, state, lengths, gain, dy, dstate, device)
    y, last, carries = recurrence.gated_recurrence(x, g, out_gate=z, state=state, lengths=lengths, gain=gain, return_carries=True)
    y2, last2 = recurrence.gated_recurrence(x, g, out_gate=z, state=state, lengths=lengths, gain=gain)
    assert bool((y == y2).all()) and bool((last == last2).all())
    assert rel(y, want[0]) <= TOL[dtype] + 3e-6 and rel(last, want[1]) <= 3e-6
    grads = recurrence.gated_recurrence_backward(x, g, carries, dy, out_gate=z, lengths=lengths, gain=gain, dstate=dstate)
    got = [grads.dx, grads.dgate] + ([grads.dout_gate] if z is not None else []) + [grads.dstate]
    assert (grads.dout_gate is None) == (z is None)
    for i, (u, v) in enumerate(zip(got, want[2:])):
        assert rel(u, v) <= (TOL[dtype] if u.dtype == x.dtype else 0.0) + 6e-6, i
    again = recurrence.gated_recurrence_backward(x, g, carries, dy, out_gate=z, lengths=lengths, gain=gain, dstate=dstate)
    for u, v in zip(grads, again):
        assert u is None or bool((u == v).all())
    return y, last, carries, grads


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["mean", "power", "one", "mean_gated"])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_definition(shape, kind, dtype):
    x, g, z, dy, state, dstate = _inputs(*shape, dtype)
    _all(x, g, z if "gated" in kind else None, dy, state, dstate, dtype, gain=kind.split("_")[0])


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", [(5, 40, 20), (4, 700, 33), (3, 1500, 64), (6, 20, 8)])
def test_lengths_and_what_lies_beyond_them(shape, gated):
    """Items that end at once, inside a run and at its border; beyond them NaN in, zeros out, the state as it was."""
    import torch
    B, T, C = shape
    x, g, z, dy, state, dstate = _inputs(*shape, "fp32")
    lengths = torch.tensor(([0, T, 17, 16, 1, T - 1] + [-3])[:B - 1] + [T + 5], dtype=torch.int32, device="cuda:0")
    z = z if gated else None
    y, last, carries, grads = _all(x, g, z, dy, state, dstate, "fp32", lengths=lengths)
    assert bool((last[0] == state[0]).all()) and bool((grads.dstate[0] == dstate[0]).all())
    beyond = torch.arange(T, device="cuda:0")[None] >= lengths.clamp(0, T)[:, None]
    bad = [torch.where(beyond[:, :, None], torch.full_like(t, float("nan")), t) if t is not None else None for t in (x, g, z, dy)]
    from paper_2209_13603_amd import recurrence
    y2, last2, carries2 = recurrence.gated_recurrence(bad[0], bad[1], out_gate=bad[2], state=state, lengths=lengths,
                                                      return_carries=True)
    g2 = recurrence.gated_recurrence_backward(bad[0], bad[1], carries2, bad[3], out_gate=bad[2], lengths=lengths, dstate=dstate)
    for u, v in zip((y2, last2, carries2, *g2), (y, last, carries, *grads)):
        assert u is None or bool((u == v).all())
    assert not y[beyond].any() and not grads.dx[beyond].any() and not grads.dgate[beyond].any()


@pytest.mark.parametrize("layout", ["joint", "time_major", "odd"])
@pytest.mark.parametrize("shape", [(3, 24, 8), (3, 24, 7), (2, 200, 64), (2, 1100, 34)])
def test_layouts_and_in_place(layout, shape):
    import torch
    from paper_2209_13603_amd import recurrence
    x, g, z, dy, state, dstate = _inputs(*shape, "bf16")
    B, T, C = shape
    y, last, carries, grads = _all(x, g, z, dy, state, dstate, "bf16")

    def lay(t):
        if layout == "joint":
            j = torch.zeros(B, T, 3, C, dtype=t.dtype, device=t.device)
            j[:, :, 1] = t
            return j[:, :, 1]
        if layout == "time_major":
            return t.transpose(0, 1).contiguous().transpose(0, 1)
        flat = torch.zeros(t.numel() + 1, dtype=t.dtype, device=t.device)
        flat[1:] = t.flatten()
        return flat[1:].view(t.shape)

    xs, gs, zs, ds = map(lay, (x, g, z, dy))
    y2, last2, carries2 = recurrence.gated_recurrence(xs, gs, out_gate=zs, state=state, return_carries=True, y=lay(y))
    g2 = recurrence.gated_recurrence_backward(xs, gs, carries2, ds, out_gate=zs, dstate=dstate, dx=lay(x), dgate=lay(x),
                                              dout_gate=lay(x))
    for u, v in zip((y2, last2, carries2, *g2), (y, last, carries, *grads)):
        assert bool((u == v).all())
    # outputs on the inputs
    for i in range(3):
        t = [v.clone() for v in (x, g, z)]
        s = state.clone()
        y3, last3 = recurrence.gated_recurrence(t[0], t[1], out_gate=t[2], state=s, y=t[i], state_out=s)
        assert y3 is t[i] and last3 is s and bool((y3 == y).all()) and bool((s == last).all())
    t = [v.clone() for v in (x, g, z, dy)]
    d = dstate.clone()
    g3 = recurrence.gated_recurrence_backward(t[0], t[1], carries, t[3], out_gate=t[2], dstate=d, dx=t[3], dgate=t[0],
                                              dout_gate=t[1], dstate_out=d)
    for u, v in zip(g3, grads):
        assert bool((u == v).all())


def test_many_series_walk_alone():
    x, g, z, dy, state, dstate = _inputs(2100, 50, 64, "bf16")
    _all(x, g, z, dy, state, dstate, "bf16", device="cuda:0")
    x, g, z, dy, state, dstate = _inputs(2000, 37, 67, "fp32")
    _all(x, g, None, dy, state, dstate, "fp32", gain="power", device="cuda:0")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_token_by_token_is_the_whole_call(dtype):
    """A series in one call, in pieces and one token at a time, from the state where the last call ended."""
    import torch
    from paper_2209_13603_amd import recurrence
    x, g, z, dy, state, _ = _inputs(3, 90, 40, dtype)
    y, last = recurrence.gated_recurrence(x, g, out_gate=z, state=state)
    for pieces in ([1] * 90, [37, 1, 52]):
        s, at, out = state.clone(), 0, []
        for n in pieces:
            part, _ = recurrence.gated_recurrence(x[:, at:at + n], g[:, at:at + n], out_gate=z[:, at:at + n], state=s, state_out=s)
            out.append(part)
            at += n
        assert rel(torch.cat(out, 1), y.double().cpu()) <= TOL[dtype] + 3e-6
        assert rel(s, last.double().cpu()) <= 3e-6


def test_gates_at_their_ends():
    """-inf starts anew from x, +inf holds the state; very large gates are as good; gradients stay finite."""
    import torch
    from paper_2209_13603_amd import recurrence
    for T in (20, 600):
        for gain in ("mean", "power", "one"):
            x, g, z, dy, state, dstate = _inputs(2, T, 6, "fp32")
            for end in (float("inf"), 200.0):
                h = g.clone()
                h[:, T // 2] = -end
                h[:, T // 2 + 1:] = end
                y, last, carries = recurrence.gated_recurrence(x, h, state=state, gain=gain, return_carries=True)
                assert bool((y[:, T // 2] == x[:, T // 2]).all())
                if gain != "one":
                    assert bool((y[:, T // 2:] == x[:, T // 2, None]).all()) and bool((last == x[:, T // 2]).all())
                grads = recurrence.gated_recurrence_backward(x, h, carries, dy, gain=gain, dstate=dstate)
                assert all(bool(torch.isfinite(t).all()) for t in grads if t is not None)
                late = dy.clone()  # nothing from the new start on reaches what came before
                late[:, :T // 2] = 0.0
                cut = recurrence.gated_recurrence_backward(x, h, carries, late, gain=gain, dstate=dstate)
                assert not cut.dstate.any() and not cut.dx[:, :T // 2].any()
                if gain != "one":
                    assert not grads.dx[:, T // 2 + 1:].any()


def test_long_memory():
    """Gates of 12 (a memory of 160000 steps): the state's sum of 40000 small steps keeps its bits.  Two roundings of 2^-25 a
    step at random: the root of 80000 of them, 1e-5."""
    import torch
    from paper_2209_13603_amd import recurrence
    r = torch.Generator(device="cuda:0").manual_seed(3)
    x = 1.0 + torch.rand((1, 40000, 4), generator=r, device="cuda:0")
    g = torch.full_like(x, 12.0)
    y, last = recurrence.gated_recurrence(x, g)
    rest = torch.sigmoid(-g.double())
    decay = torch.cumsum(torch.log1p(-rest), 1)
    want = (torch.exp(decay[:, -1:] - decay) * rest * x.double()).sum(1)
    assert rel(last, want) <= 1e-5


def test_without_tokens_and_refusals():
    import torch
    from paper_2209_13603_amd import disco, recurrence
    x, g, z, dy, state, dstate = _inputs(2, 5, 6, "fp32")
    y, last, carries = recurrence.gated_recurrence(x[:, :0], g[:, :0], state=state, return_carries=True)
    assert y.shape == (2, 0, 6) and bool((last == state).all()) and carries.shape == (2, 0, 6)
    grads = recurrence.gated_recurrence_backward(x[:, :0], g[:, :0], carries, dy[:, :0], dstate=dstate)
    assert bool((grads.dstate == dstate).all())
    y, last = recurrence.gated_recurrence(x[:, :0], g[:, :0])
    assert not last.any()
    y, last = recurrence.gated_recurrence(x[:0], g[:0])
    assert y.shape == (0, 5, 6) and last.shape == (0, 6)
    with pytest.raises(ValueError):
        recurrence.gated_recurrence(x, g, gain="sum")
    with pytest.raises(ValueError):
        recurrence.gated_recurrence(x, g, state=state.bfloat16())
    with pytest.raises(ValueError):
        recurrence.gated_recurrence(x, g, lengths=torch.zeros(2, device="cuda:0"))
    with pytest.raises(ValueError):
        recurrence.gated_recurrence(x, g, lengths=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        recurrence.gated_recurrence(x[0], g[0])
    with pytest.raises(disco.DiscoError):
        recurrence.gated_recurrence(x, g.bfloat16())
    with pytest.raises(disco.DiscoError):
        recurrence.gated_recurrence(x, g[:, :4])
    with pytest.raises(ValueError):
        recurrence.gated_recurrence_backward(x, g, torch.zeros(2, 2, 6, device="cuda:0"), dy)


def test_gradients_against_differences():
    """Central differences of the kernel's own outputs, fp32."""
    import torch
    from paper_2209_13603_amd import recurrence
    for gain in ("mean", "power", "one"):
        x, g, z, dy, state, dstate = _inputs(1, 60, 6, "fp32")
        base = dict(x=x, gate=g, out_gate=z, state=state)

        def total(p):
            y, last = recurrence.gated_recurrence(p["x"], p["gate"], out_gate=p["out_gate"], state=p["state"], gain=gain)
            return float((y.double() * dy.double()).sum() + (last.double() * dstate.double()).sum())

        _, _, carries = recurrence.gated_recurrence(x, g, out_gate=z, state=state, gain=gain, return_carries=True)
        grads = recurrence.gated_recurrence_backward(x, g, carries, dy, out_gate=z, dstate=dstate, gain=gain)
        for name, grad in (("x", grads.dx), ("gate", grads.dgate), ("out_gate", grads.dout_gate), ("state", grads.dstate)):
            d = torch.randn(base[name].shape, generator=torch.Generator(device="cuda:0").manual_seed(5), device="cuda:0")
            diff = (total({**base, name: base[name] + 1e-2 * d}) - total({**base, name: base[name] - 1e-2 * d})) / 2e-2
            want, size = float((grad.double() * d.double()).sum()), float(grad.double().norm() * d.double().norm())
            assert abs(diff - want) <= 2e-3 * size, (gain, name)


def test_lengths_on_the_host_are_refused_without_steps_too():
    """A call of no steps reads the lengths as well, to give the state: they have to be the device's."""
    import ctypes
    import torch
    from paper_2209_13603_amd import blocks, disco
    x, _, _, _, state, _ = _inputs(2, 5, 6, "fp32")
    host = (ctypes.c_int32 * 2)(1, 2)
    opt = disco.RecurrenceArgs(0, 0, ctypes.addressof(host))
    last = torch.full_like(state, 7.0)
    p = blocks._Pack()
    r = p.rows(x[:, :0], "x")
    lib, to = disco.library(), ctypes.addressof(opt)
    assert lib.disco_gated_recurrence(r, r, None, to, state.data_ptr(), r, last.data_ptr(), None, None, 0, None) == \
        disco.DISCO_ERR_DEVICE
    assert lib.disco_gated_recurrence_backward(r, r, None, to, None, r, state.data_ptr(), None, None, None, last.data_ptr(), None, 0,
                                               None) == disco.DISCO_ERR_DEVICE
    torch.cuda.synchronize()
    assert bool((last == 7).all())
