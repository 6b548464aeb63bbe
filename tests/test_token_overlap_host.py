"""Which tensors of a token call count as overlapping, from their addresses and strides alone: refusals come before any
device call, and what is not refused ends, with addresses that no device knows, as a DEVICE error."""
import ctypes
import itertools
import random

import pytest

from paper_2209_13603_amd import disco

BASE = 0x100000


def heads(shape, strides, offset, dtype=disco.DISCO_FLOAT32):
    B, S, H, D = shape
    return disco.Heads(BASE + offset * (4 if dtype == disco.DISCO_FLOAT32 else 2), dtype, D, H, 0, B, S, *strides)


def places(shape, strides, offset):
    B, S, H, D = shape
    return {offset + b * strides[0] + s * strides[1] + h * strides[2] + d
            for b, s, h, d in itertools.product(range(B), range(S), range(H), range(D))}


def refused(x, y):
    status = disco.library().disco_norm_rotate(x, 0, None, 0.0, None, y, None)
    assert status in (disco.DISCO_ERR_INVALID_ARGUMENT, disco.DISCO_ERR_DEVICE)
    return status == disco.DISCO_ERR_INVALID_ARGUMENT


def nested(rng, shape):
    """Strides whose axes, in some order, step over each other, with gaps now and then."""
    strides, step = [0, 0, 0], shape[3]
    for axis in rng.sample(range(3), 3):
        strides[axis] = step + rng.choice((0, 0, 1, 3, shape[3], 2 * shape[3], step))
        step = strides[axis] * shape[axis]
    return strides


def test_parts_of_one_buffer_are_told_apart_exactly():
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(4000):
        shape = [rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 3), rng.randint(1, 4)]
        strides = nested(rng, shape)
        offset = rng.randint(-2 * max(strides), 2 * max(strides))
        x, y = heads(shape, strides, 0), heads(shape, strides, offset)
        meet = bool(places(shape, strides, 0) & places(shape, strides, offset))
        if offset == 0:
            continue  # in place
        seen[meet] += 1
        assert refused(x, y) == meet, (shape, strides, offset)
    assert min(seen) > 500


def test_no_overlap_passes():
    """Any two layouts, the input's with shared and overlapping rows too."""
    rng = random.Random(2)
    seen = 0
    for _ in range(4000):
        shape = [rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 3), rng.randint(1, 4)]
        sy = nested(rng, shape)
        sx = nested(rng, shape) if rng.random() < 0.5 else [rng.randint(0, 12) for _ in range(3)]
        offset = rng.randint(-30, 30)
        if places(shape, sx, 0) & places(shape, sy, offset):
            same = offset == 0 and all(n == 1 or a == b for n, a, b in zip(shape, sx, sy))
            seen += 1
            assert same or refused(heads(shape, sx, 0), heads(shape, sy, offset)), (shape, sx, sy, offset)
    assert seen > 1000


@pytest.mark.parametrize("layout", ["B 2 H S D", "B S H 2 D", "B S 2 H D", "2 B S H D", "H B S 2 D"])
def test_gradients_into_one_buffer(layout):
    """dk and dv as the two parts of a joint buffer in any order of its axes."""
    size = {"B": 3, "S": 7, "H": 4, "D": 8, "2": 2}
    stride, step = {}, 1
    for name in reversed(layout.split()):
        stride[name] = step
        step *= size[name]
    shape, strides = (3, 7, 4, 8), (stride["B"], stride["S"], stride["H"])
    far = lambda n, S=7: heads((3, S, 4, 8), (S * 32, 32, 8), n * 100000)
    dk, dv = heads(shape, strides, 0), heads(shape, strides, stride["2"])
    one = heads(shape, strides, stride["2"] - 1 if stride["2"] > 1 else 1)
    call = disco.library().disco_cross_attention_backward
    args = (far(1, 5), far(2), far(3), None, far(4, 5), 0x90000000, None, far(5, 5), far(6, 5))
    assert call(*args, dk, dv, None, 0, None) == disco.DISCO_ERR_DEVICE
    assert call(*args, dk, one, None, 0, None) == disco.DISCO_ERR_INVALID_ARGUMENT
    assert call(*args, dk, dk, None, 0, None) == disco.DISCO_ERR_INVALID_ARGUMENT


def test_parts_of_a_projection_with_fewer_key_heads():
    """Queries of 6 heads, keys and values of 2, side by side in a token; outputs beside inputs of one buffer."""
    B, S, D = 2, 5, 8
    sizes, at = {"q": 6, "k": 2, "v": 2, "dq": 6, "dk": 2, "dv": 2}, {}
    token = 0
    for name, n in sizes.items():
        at[name] = token
        token += n * D
    t = {name: heads((B, S, n, D), (S * token, token, D), at[name]) for name, n in sizes.items()}
    out, dout = (heads((B, S, 6, D), (S * 48, 48, D), 1000000 * i) for i in (1, 2))
    call = disco.library().disco_cross_attention_backward
    args = lambda dv: (t["q"], t["k"], t["v"], None, out, 0x90000000, None, dout, t["dq"], t["dk"], dv, None, 0, None)
    assert call(*args(t["dv"])) == disco.DISCO_ERR_DEVICE
    assert call(*args(heads((B, S, 2, D), (S * token, token, D), at["dv"] - 1))) == disco.DISCO_ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("shape", [(1, 5, 3, 8), (2, 1, 3, 8), (2, 5, 1, 8)])
def test_in_place_whatever_the_stride_of_a_single_entry(shape):
    strides = [shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3]]
    axis = shape.index(1)
    other = list(strides)
    other[axis] = 1000
    x, y = heads(shape, strides, 0), heads(shape, other, 0)
    assert not refused(x, y)
    call = disco.library().disco_norm_rotate_backward
    assert call(None, 0, None, 0.0, None, x, y, None, None, 0, None) == disco.DISCO_ERR_DEVICE
