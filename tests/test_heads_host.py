"""Host-side checks of the token and gradient entries that need no GPU: refusals come before any device call, and
the rotation tables hold what they say."""
import ctypes
import math

import pytest
import torch

from paper_2209_13603_amd import attention, disco

F32, BF16 = disco.DISCO_FLOAT32, disco.DISCO_BFLOAT16


def heads(batch=2, tokens=3, n=4, dim=8, dtype=F32, data=0x10000, **kw):
    h = disco.Heads(data, dtype, dim, n, 0, batch, tokens, tokens * n * dim, n * dim, dim)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


def tensor(*shape, dtype=F32, data=0x900000):
    return disco.Tensor(data, dtype, len(shape), (ctypes.c_int64 * 4)(*(list(shape) + [0] * (4 - len(shape)))))


def rotate(x, y, norm=1, weight=None, eps=1e-6, rotation=None):
    ref = lambda t: None if t is None else ctypes.byref(t)
    return disco.library().disco_norm_rotate(ref(x), norm, ref(weight), eps, ref(rotation), ref(y), None)


def attend(q, k, v, out, opt=None, low=None):
    ref = lambda t: None if t is None else ctypes.byref(t)
    return disco.library().disco_cross_attention(ref(q), ref(k), ref(v), ref(opt), ref(out), None, ref(low), None, 0, None)


Y = dict(data=0x4000000)


@pytest.mark.parametrize("x,y,kw,status", [
    (None, heads(**Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), None, {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(dtype=7), heads(dtype=7, **Y), {}, disco.DISCO_ERR_DTYPE),
    (heads(), heads(dtype=BF16, **Y), {}, disco.DISCO_ERR_DTYPE),
    (heads(dim=0), heads(dim=0, **Y), {}, disco.DISCO_ERR_SHAPE),
    (heads(dim=129), heads(dim=129, **Y), {}, disco.DISCO_ERR_SHAPE),
    (heads(), heads(tokens=4, **Y), {}, disco.DISCO_ERR_SHAPE),
    (heads(batch=-1), heads(batch=-1, **Y), {}, disco.DISCO_ERR_SHAPE),
    (heads(tokens=1 << 31), heads(tokens=1 << 31, **Y), {}, disco.DISCO_ERR_SHAPE),
    (heads(data=None), heads(**Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(data=0x10002), heads(**Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(stride_token=-8), heads(**Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(stride_token=1 << 45), heads(**Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(reserved=1), heads(**Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(stride_head=4, **Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),       # rows of y overlap
    (heads(), heads(data=0x10020), {}, disco.DISCO_ERR_INVALID_ARGUMENT),             # y overlaps x
    (heads(), heads(**Y), dict(norm=2), disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(**Y), dict(eps=-1.0), disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(**Y), dict(eps=math.nan), disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(**Y), dict(weight=tensor(7)), disco.DISCO_ERR_SHAPE),
    (heads(), heads(**Y), dict(weight=tensor(8, dtype=BF16)), disco.DISCO_ERR_DTYPE),
    (heads(), heads(**Y), dict(weight=tensor(8), norm=0), disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(**Y), dict(rotation=disco.RotationArgs(3, 0, 0x1000, 0x1000, 9, None, 0, 0)), disco.DISCO_ERR_SHAPE),
    (heads(), heads(**Y), dict(rotation=disco.RotationArgs(10, 0, 0x1000, 0x1000, 9, None, 0, 0)), disco.DISCO_ERR_SHAPE),
    (heads(), heads(**Y), dict(rotation=disco.RotationArgs(4, 2, 0x1000, 0x1000, 9, None, 0, 0)), disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(**Y), dict(rotation=disco.RotationArgs(4, 0, None, 0x1000, 9, None, 0, 0)), disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(**Y), dict(rotation=disco.RotationArgs(4, 0, 0x1000, 0x1000, 2, None, 0, 0)), disco.DISCO_ERR_SHAPE),
    (heads(), heads(**Y), dict(rotation=disco.RotationArgs(4, 0, 0x1000, 0x1000, 9, None, 0, -1)), disco.DISCO_ERR_INVALID_ARGUMENT),
])
def test_norm_rotate_refuses(x, y, kw, status):
    assert rotate(x, y, **kw) == status
    assert disco.library().disco_last_error().decode()


@pytest.mark.parametrize("q,k,v,out,kw,status", [
    (None, heads(), heads(), heads(**Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(n=3), heads(n=3), heads(**Y), {}, disco.DISCO_ERR_SHAPE),
    (heads(), heads(), None, heads(**Y), {}, disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(), heads(tokens=5), heads(**Y), {}, disco.DISCO_ERR_SHAPE),
    (heads(), heads(batch=1), heads(batch=1), heads(**Y), {}, disco.DISCO_ERR_SHAPE),
    (heads(), heads(dtype=BF16), heads(dtype=BF16), heads(**Y), {}, disco.DISCO_ERR_DTYPE),
    (heads(), heads(), heads(), heads(), {}, disco.DISCO_ERR_INVALID_ARGUMENT),         # out is q
    (heads(), heads(), heads(), heads(**Y), dict(opt=disco.AttentionArgs(math.inf, None, 0, None)),
     disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(), heads(), heads(**Y), dict(opt=disco.AttentionArgs(1.0, 0x1000, -1, None)),
     disco.DISCO_ERR_INVALID_ARGUMENT),
    (heads(), heads(), heads(), heads(**Y), dict(low=heads(data=0x8000000)), disco.DISCO_ERR_DTYPE),
])
def test_cross_attention_refuses(q, k, v, out, kw, status):
    assert attend(q, k, v, out, **kw) == status
    assert disco.library().disco_last_error().decode()


def test_workspace_sizes_are_host_arithmetic():
    lib, n = disco.library(), ctypes.c_size_t()
    # many rows: no parts; one row against many keys: parts
    assert lib.disco_cross_attention_workspace(heads(tokens=100000, dim=64), heads(tokens=100, dim=64), 0, n) == 0
    assert n.value == 0
    assert lib.disco_cross_attention_workspace(heads(tokens=1, dim=64), heads(tokens=100000, dim=64), 0, n) == 0
    assert n.value > 0
    assert lib.disco_cross_attention_workspace(heads(), heads(), 0, None) == disco.DISCO_ERR_INVALID_ARGUMENT
    assert lib.disco_norm_rotate_workspace(heads(), None, n) == 0 and n.value == 0
    w = tensor(8)
    assert lib.disco_norm_rotate_workspace(heads(), w, n) == 0 and n.value > 0
    assert lib.disco_gradient_clip_workspace(-1, None, n) == disco.DISCO_ERR_INVALID_ARGUMENT
    assert lib.disco_gradient_clip_workspace(0, None, n) == 0


def test_gradient_clip_refuses():
    lib = disco.library()
    arr = (disco.Tensor * 1)(tensor(5, dtype=9))
    at = ctypes.addressof(arr)
    assert lib.disco_gradient_clip(1, at, None, 1.0, 0.0, 0x1000, None, 0, None) == disco.DISCO_ERR_DTYPE
    arr[0] = tensor(5, -1)
    assert lib.disco_gradient_clip(1, at, None, 1.0, 0.0, 0x1000, None, 0, None) == disco.DISCO_ERR_SHAPE
    arr[0] = tensor(5)
    assert lib.disco_gradient_clip(1, at, None, 1.0, 0.0, None, None, 0, None) == disco.DISCO_ERR_INVALID_ARGUMENT
    assert lib.disco_gradient_clip(1, at, at, -1.0, 0.0, 0x1000, None, 0, None) == disco.DISCO_ERR_INVALID_ARGUMENT
    assert lib.disco_gradient_clip(1, None, None, 1.0, 0.0, 0x1000, None, 0, None) == disco.DISCO_ERR_INVALID_ARGUMENT


def test_rotation_tables():
    cos, sin = attention.line_rotation(50, 12, base=100.0, stretch=2.0, device="cpu")
    assert cos.shape == sin.shape == (50, 6)
    angle = (7 / 2.0) * 100.0 ** (-2 * 3 / 12)
    assert abs(float(cos[7, 3]) - math.cos(angle)) < 1e-6 and abs(float(sin[7, 3]) - math.sin(angle)) < 1e-6
    # raised base: the fastest pair unchanged, the slowest slower by the stretch
    plain, _ = attention.line_rotation(50, 12, base=100.0, device="cpu")
    raised, sr = attention.line_rotation(50, 12, base=100.0, stretch=4.0, stretch_base=True, device="cpu")
    assert torch.equal(plain[:, 0], raised[:, 0])
    slow = 100.0 ** (-10 / 12) / 4.0
    assert abs(float(sr[1, 5]) - math.sin(slow)) < 1e-7
    # whole longitude frequencies close around the sphere
    cos, sin = attention.grid_rotation(3, 8, 8, device="cpu")
    z = torch.complex(cos.double(), sin.double()).view(3, 8, 4)
    turn = z[0, 1, :2] / z[0, 0, :2]
    assert float((turn ** 8 - 1).abs().max()) < 1e-6
    assert float((z[:, 0, 2:] - z[:, 5, 2:]).abs().max()) < 1e-7  # colatitude: the same along a ring
