"""Recurrences whose workgroups scan several tiles of 256 steps one after the other, against the definition in 64 bits:
in one part over all time, and in several parts of several tiles each, forward and backward.

Tolerances: those of test_gpu_recurrence.py, for the same gates (memories of at most 150 steps): a relative 2-norm of 3e-6 for
states and outputs and 6e-6 for gradients, beside half a unit (2^-8) where bf16 is stored.
"""
import ctypes

import pytest

from block_forms import recurrence as form
from block_forms import rel

pytestmark = pytest.mark.gpu

TOL = {"bf16": 2.0 ** -8, "fp32": 0.0}
# 192 blocks of 64 channels and more: one part of several tiles; fewer: several parts, of two and three tiles each here
ONE_PART = [(13, 600, 1000), (16, 520, 770), (9, 530, 1431)]
PARTS = [(3, 5200, 1024), (2, 5300, 1503)]


def _inputs(B, T, C, dtype, seed=0):
    import torch
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    r = torch.Generator(device="cuda:0").manual_seed(seed + B + 3 * T + 7 * C)
    rnd = lambda *s: torch.randn(s, generator=r, device="cuda:0")
    x, z, dy = (rnd(B, T, C).to(dt) for _ in range(3))
    g = (rnd(B, T, C) + torch.linspace(-1, 4, C, device="cuda:0")).clamp(max=5.0).to(dt)
    return x, g, z, dy, rnd(B, C), rnd(B, C)


def _intended(x, T):
    """Whether the call is cut into one part of several tiles, or into parts of which one has several."""
    from paper_2209_13603_amd import disco, recurrence
    B, _, C = x.shape
    pack, need = recurrence._Pack(), ctypes.c_size_t()
    assert disco.library().disco_gated_recurrence_workspace(pack.rows(x, "x"), need) == 0
    columns, tiles = (C + 1) // 2, -(-T // 256)
    blocks = -(-B * columns // 32)
    assert B * columns < 65536 and tiles >= 2  # no thread walks alone
    if blocks >= 192:
        assert need.value == 0
    else:
        parts = (need.value // (4 * B * C) - 1) // 2
        assert 1 < parts and tiles >= 2 * parts


def _both(x, g, z, dy, state, dstate, gain, lengths, **out):
    from paper_2209_13603_amd import recurrence
    y, last, carries = recurrence.gated_recurrence(x, g, out_gate=z, state=state, lengths=lengths, gain=gain, return_carries=True)
    grads = recurrence.gated_recurrence_backward(x, g, carries, dy, out_gate=z, lengths=lengths, gain=gain, dstate=dstate)
    return y, last, carries, grads


def _check(got, want, dtype, z):
    y, last, _, grads = got
    assert rel(y, want[0]) <= TOL[dtype] + 3e-6 and rel(last, want[1]) <= 3e-6
    for u, v in zip([grads.dx, grads.dgate] + ([grads.dout_gate] if z is not None else []), want[2:]):
        assert rel(u, v) <= TOL[dtype] + 6e-6
    assert rel(grads.dstate, want[-1]) <= 6e-6


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["mean", "power", "one", "mean_gated", "power_gated"])
@pytest.mark.parametrize("shape", ONE_PART)
def test_one_part_of_several_tiles(shape, kind, dtype):
    x, g, z, dy, state, dstate = _inputs(*shape, dtype)
    _intended(x, shape[1])
    z, gain = z if "gated" in kind else None, kind.split("_")[0]
    _check(_both(x, g, z, dy, state, dstate, gain, None), form(x, g, z, state, None, gain, dy, dstate, "cuda:0"), dtype, z)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["mean", "power_gated"])
@pytest.mark.parametrize("shape", PARTS)
def test_parts_of_several_tiles(shape, kind, dtype):
    x, g, z, dy, state, dstate = _inputs(*shape, dtype)
    _intended(x, shape[1])
    z, gain = z if "gated" in kind else None, kind.split("_")[0]
    _check(_both(x, g, z, dy, state, dstate, gain, None), form(x, g, z, state, None, gain, dy, dstate, "cuda:0"), dtype, z)


def _lengths(B, T):
    import torch
    ends = [T, 300, 256, 0, 17, T - 1, 513, 255, 1, 272, T + 9, -2, 512, 100, 257, 499]
    return torch.tensor(ends[:B], dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", [(13, 600, 1000), (9, 530, 1431), (3, 5200, 1024)])
def test_lengths_and_what_lies_beyond_them(shape, gated, dtype):
    """Items that end in every tile, at its borders and inside runs; NaN beyond, zeros out, the state as it was."""
    import torch
    B, T, C = shape
    x, g, z, dy, state, dstate = _inputs(*shape, dtype)
    _intended(x, T)
    z, lengths = z if gated else None, _lengths(B, T) if B > 3 else torch.tensor([T - 700, 1300, 2050], dtype=torch.int32, device="cuda:0")
    got = _both(x, g, z, dy, state, dstate, "mean", lengths)
    _check(got, form(x, g, z, state, lengths, "mean", dy, dstate, "cuda:0"), dtype, z)
    beyond = torch.arange(T, device="cuda:0")[None] >= lengths.clamp(0, T)[:, None]
    bad = [torch.where(beyond[:, :, None], torch.full_like(t, float("nan")), t) if t is not None else None for t in (x, g, z, dy)]
    again = _both(*bad, state, dstate, "mean", lengths)
    for u, v in zip((*again[:3], *again[3]), (*got[:3], *got[3])):
        assert u is None or bool((u == v).all())
    assert not got[0][beyond].any() and not got[3].dx[beyond].any() and not got[3].dgate[beyond].any()
    none = lengths.clamp(0, T) == 0
    assert bool((got[1][none] == state[none]).all()) and bool((got[3].dstate[none] == dstate[none]).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("shape", [(13, 600, 1000), (9, 530, 1431), (3, 5200, 1024)])
def test_in_place_and_joint(shape, ragged, dtype):
    """Outputs on the inputs while the next tile's loads are out, and parts of joint buffers: the same bits."""
    import torch
    from paper_2209_13603_amd import recurrence
    B, T, C = shape
    x, g, z, dy, state, dstate = _inputs(*shape, dtype)
    lengths = torch.tensor([(T * (b + 1)) // B for b in range(B)], dtype=torch.int32, device="cuda:0") if ragged else None
    for gate in (None, z):
        y, last, carries, grads = _both(x, g, gate, dy, state, dstate, "mean", lengths)
        joint = torch.full((B, T, 4, C), 7.0, dtype=x.dtype, device="cuda:0")
        parts = joint.unbind(2)
        for p, t in zip(parts, (x, g, z)):
            p.copy_(t)
        kw = dict(out_gate=parts[2] if gate is not None else None, lengths=lengths)
        y2, last2, carries2 = recurrence.gated_recurrence(parts[0], parts[1], state=state, return_carries=True, y=parts[3], **kw)
        assert bool((y2 == y).all()) and bool((last2 == last).all()) and bool((carries2 == carries).all())
        for i in range(2 if gate is None else 3):
            t = [v.clone() if v is not None else None for v in (x, g, gate)]
            s = state.clone()
            y3, last3 = recurrence.gated_recurrence(t[0], t[1], out_gate=t[2], lengths=lengths, state=s, y=t[i], state_out=s)
            assert y3 is t[i] and bool((y3 == y).all()) and bool((s == last).all())
        # gradients: over the inputs, in another order
        t = [v.clone() if v is not None else None for v in (x, g, gate, dy)]
        d = dstate.clone()
        places = dict(dx=t[3], dgate=t[0]) if gate is None else dict(dx=t[3], dgate=t[0], dout_gate=t[1])
        got = recurrence.gated_recurrence_backward(t[0], t[1], carries, t[3], out_gate=t[2], lengths=lengths, dstate=d,
                                                   dstate_out=d, **places)
        for u, v in zip(got, grads):
            assert v is None or bool((u == v).all())
        # one of them alone
        only = recurrence.gated_recurrence_backward(x, g, carries, dy, out_gate=gate, lengths=lengths, dstate=dstate, want_dgate=False)
        assert only.dgate is None and bool((only.dx == grads.dx).all()) and bool((only.dstate == grads.dstate).all())
