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


# ---- outputs beside tables, masks, statistics and scratch memory ------------------------------------------------------
INVALID, DEVICE = disco.DISCO_ERR_INVALID_ARGUMENT, disco.DISCO_ERR_DEVICE
FAR = 0x80000000


def weight(address, n=8):
    return disco.Tensor(address, disco.DISCO_FLOAT32, 1, (ctypes.c_int64 * 4)(n, 0, 0, 0))


def dense(n, shape=(2, 5, 3, 8), data=None):
    B, S, H, D = shape
    h = heads(shape, (S * H * D, H * D, D), n * 100000)
    if data is not None:
        h.data = data
    return h


# y spans 960 bytes; a table of 6 rows of 2, positions [2, 5], a weight of 8
@pytest.mark.parametrize("what,size", [("weight", 32), ("cosines", 48), ("sines", 48), ("positions", 40)])
@pytest.mark.parametrize("back", [False, True])
def test_norm_rotate_refuses_outputs_over_its_small_arguments(what, size, back):
    x, y = dense(1), dense(2)
    for at, status in ((y.data, INVALID), (y.data + 956, INVALID), (y.data - size + 4, INVALID), (y.data + 960, DEVICE),
                       (y.data - size, DEVICE)):
        a = {"weight": FAR, "cosines": FAR + 4096, "sines": FAR + 8192, "positions": FAR + 16384}
        a[what] = at
        rot = disco.RotationArgs(4, 0, a["cosines"], a["sines"], 6, a["positions"], 5, 0)
        lib = disco.library()
        got = lib.disco_norm_rotate_backward(x, 1, weight(a["weight"]), 0.0, rot, dense(3), y, None, None, 0, None) if back else \
            lib.disco_norm_rotate(x, 1, weight(a["weight"]), 0.0, rot, y, None)
        assert got == status, (what, hex(at))


@pytest.mark.parametrize("what,size", [("cosines", 48), ("sines", 48), ("positions", 40)])
def test_the_weights_gradient_lies_apart_from_tables(what, size):
    a = {"cosines": FAR + 4096, "sines": FAR + 8192, "positions": FAR + 16384}
    for at, status in ((FAR + 256, INVALID), (FAR + 256 + 28, INVALID), (FAR + 256 + 32, DEVICE)):
        a[what] = at
        rot = disco.RotationArgs(4, 0, a["cosines"], a["sines"], 6, a["positions"], 5, 0)
        assert disco.library().disco_norm_rotate_backward(dense(1), 1, weight(FAR), 0.0, rot, dense(3), None, weight(FAR + 256),
                                                          None, 0, None) == status


def test_a_small_argument_between_the_rows_of_an_output():
    """Gaps that hold it are no overlap: after each token, and between batch items."""
    for shape, strides, gap, n in (((2, 5, 3, 8), (200, 40, 8), 24, 10), ((2, 5, 3, 8), (500, 24, 8), 120, 300)):
        y = heads(shape, strides, 0)
        base = disco.RotationArgs(4, 0, FAR, FAR + 4096, 6, None, 0, 0)
        for off, status in ((gap, DEVICE), (gap - 1, INVALID), (gap + 81 if n > 10 else gap + 9, INVALID)):
            rot = disco.RotationArgs(4, 0, BASE + 4 * off, FAR + 4096, n // 2, None, 0, 0)
            assert disco.library().disco_norm_rotate(dense(5), 0, None, 0.0, rot, y, None) == status, (strides, off)
        assert disco.library().disco_norm_rotate(dense(5), 0, None, 0.0, base, y, None) == DEVICE


# batch 2, 5 queries, 7 keys, 3 heads of 8, fp32: stats 2 * 3 * 5 * 2 floats, bias [2, 7], lengths [2]
@pytest.mark.parametrize("what,size", [("bias", 56), ("lengths", 8)])
@pytest.mark.parametrize("back", [False, True])
def test_attention_refuses_outputs_over_its_masks(what, size, back):
    for n, out_bytes in ((4, 960),) if not back else ((6, 960), (7, 1344), (8, 1344)):
        at0 = BASE + 400000 * n
        for at, status in ((at0, INVALID), (at0 + out_bytes - 4, INVALID), (at0 - size + 4, INVALID), (at0 + out_bytes, DEVICE)):
            a = {"bias": FAR, "lengths": FAR + 4096, what: at}
            opt = disco.AttentionArgs(0.0, a["bias"], 7, a["lengths"])
            assert attend(opt, back) == status, (what, n, hex(at))


def attend(opt=None, back=False, stats=FAR + 65536, workspace=None, nbytes=0):
    lib = disco.library()
    q, out = dense(1), dense(4)
    k, v = dense(2, (2, 7, 3, 8)), dense(3, (2, 7, 3, 8))
    if not back:
        return lib.disco_cross_attention(q, k, v, opt, out, stats, None, workspace, nbytes, None)
    return lib.disco_cross_attention_backward(q, k, v, opt, out, stats, None, dense(5), dense(6), dense(7, (2, 7, 3, 8)),
                                              dense(8, (2, 7, 3, 8)), workspace, nbytes, None)


def test_statistics_lie_apart():
    opt = disco.AttentionArgs(0.0, FAR, 7, FAR + 4096)
    for n, size in ((1, 960), (2, 1344), (3, 1344), (4, 960)):
        at = BASE + 400000 * n
        assert attend(opt, stats=at) == INVALID and attend(opt, stats=at + size - 4) == INVALID
        assert attend(opt, stats=at + size) == DEVICE
    assert attend(opt, stats=FAR) == INVALID and attend(opt, stats=FAR + 4096) == INVALID
    for n, size in ((6, 960), (7, 1344), (8, 1344)):
        at = BASE + 400000 * n
        assert attend(opt, True, stats=at) == INVALID and attend(opt, True, stats=at + size) == DEVICE


def test_the_workspace_lies_apart():
    lib, n = disco.library(), ctypes.c_size_t()
    # (the backward call's; the forward call of these sizes needs none)
    assert lib.disco_cross_attention_workspace(dense(1), dense(2, (2, 7, 3, 8)), 1, n) == 0 and n.value > 0
    opt = disco.AttentionArgs(0.0, FAR, 7, FAR + 4096)
    size = 1 << 20
    for i in range(1, 9):
        at = (BASE + 400000 * i) // 256 * 256
        assert attend(opt, True, workspace=at, nbytes=size) == INVALID, i
    for at in (FAR, FAR + 4096, FAR + 65536):
        assert attend(opt, True, workspace=at, nbytes=size) == INVALID
    assert attend(opt, True, workspace=FAR + (1 << 20), nbytes=size) == DEVICE
    # one query, keys in parts
    q, k, v, out = (dense(i, s) for i, s in ((1, (1, 1, 1, 8)), (2, (1, 4000, 1, 8)), (3, (1, 4000, 1, 8)), (4, (1, 1, 1, 8))))
    assert lib.disco_cross_attention_workspace(q, k, 0, n) == 0 and n.value > 0
    for t in (q, k, v, out):
        assert lib.disco_cross_attention(q, k, v, None, out, None, None, t.data // 256 * 256, size, None) == INVALID
    assert lib.disco_cross_attention(q, k, v, None, out, None, None, FAR, size, None) == DEVICE
    # the weight's gradient
    x, dy, dx = dense(1), dense(2), dense(3)
    assert lib.disco_norm_rotate_workspace(dy, weight(FAR), n) == 0 and n.value > 0
    run = lambda ws: lib.disco_norm_rotate_backward(x, 1, weight(FAR + 4096), 0.0, None, dy, dx, weight(FAR), ws, 1 << 30, None)
    for at in (x.data, dy.data, dx.data, FAR, FAR + 4096):
        assert run(at // 256 * 256) == INVALID
    assert run(FAR + (1 << 28)) == DEVICE


def test_clipping_keeps_its_workspace_apart():
    lib, n = disco.library(), ctypes.c_size_t()
    grads, outs = ((disco.Tensor * 1)(weight(at, 100000)) for at in (FAR, FAR + (1 << 22)))
    g, o = ctypes.addressof(grads), ctypes.addressof(outs)
    assert lib.disco_gradient_clip_workspace(1, g, n) == 0 and n.value > 0
    norm = FAR + (1 << 24)
    run = lambda ws, clipped=o: lib.disco_gradient_clip(1, g, clipped, 1.0, 0.0, norm, ws, 1 << 20, None)
    for at in (FAR, FAR + 4 * 100000 // 256 * 256, FAR + (1 << 22), norm):
        assert run(at) == INVALID
    assert run(FAR, None) == INVALID and run(FAR + (1 << 22), None) == DEVICE
    assert run(FAR + (1 << 25)) == DEVICE
