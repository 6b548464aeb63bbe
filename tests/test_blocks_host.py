"""Host-side checks of the block entries that need no GPU: refusals come before any device call, what is not refused
ends, with addresses that no device knows, as a DEVICE error; and the generator's published test values."""
import ctypes
import math

import numpy as np
import pytest

from block_forms import kept
from paper_2209_13603_amd import disco

F32, BF16 = disco.DISCO_FLOAT32, disco.DISCO_BFLOAT16
INVALID, SHAPE, DTYPE, DEVICE = (disco.DISCO_ERR_INVALID_ARGUMENT, disco.DISCO_ERR_SHAPE, disco.DISCO_ERR_DTYPE,
                                 disco.DISCO_ERR_DEVICE)


def rows(at=1, batch=2, tokens=3, channels=8, dtype=F32, **kw):
    r = disco.Rows(at * 0x100000, dtype, 0, batch, tokens, channels, tokens * channels, channels)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def tensor(*shape, dtype=F32, at=40):
    return disco.Tensor(at * 0x100000, dtype, len(shape), (ctypes.c_int64 * 4)(*(list(shape) + [0] * (4 - len(shape)))))


def ref(t):
    return None if t is None else ctypes.byref(t)


def options(scale=1.0, eps=1e-6, post_norm=0, reserved=0, post=None, gate=None, nxt=None, drop=None):
    ptr = [ctypes.pointer(t) if t is not None else None for t in (post, gate, nxt, drop)]
    return disco.ResidualArgs(scale, eps, post_norm, reserved, *ptr)


def residual(x, f, h, y, opt=None):
    return disco.library().disco_residual_norm(ref(x), ref(f), ref(opt), ref(h), ref(y), None)


def drop(p=0.5, counter=None):
    return disco.DropoutArgs(p, 1, 2, counter)


H, Y = rows(3), rows(4)


@pytest.mark.parametrize("x,f,h,y,opt,status", [
    (rows(1), rows(2), H, Y, None, DEVICE),
    (None, rows(2), None, Y, None, DEVICE),
    (rows(1), rows(2), rows(1), rows(2), None, DEVICE),                        # h is x, y is f
    (rows(1), rows(2), rows(1), rows(1), None, INVALID),                       # h and y in one place
    (rows(1), None, H, Y, None, INVALID),
    (rows(1), rows(2), None, None, None, INVALID),
    (rows(1, dtype=9), rows(2, dtype=9), H, Y, None, DTYPE),
    (rows(1, dtype=BF16), rows(2), H, Y, None, DTYPE),
    (rows(1), rows(2), rows(3, dtype=BF16), Y, None, DTYPE),
    (rows(1, channels=8193), rows(2, channels=8193), rows(3, channels=8193), None, None, SHAPE),
    (rows(1, channels=0), rows(2, channels=0), rows(3, channels=0), None, None, SHAPE),
    (rows(1), rows(2, tokens=4), H, Y, None, SHAPE),
    (rows(1), rows(2), rows(3, batch=1), Y, None, SHAPE),
    (rows(1, batch=-1), rows(2, batch=-1), rows(3, batch=-1), None, None, SHAPE),
    (rows(1, tokens=1 << 30), rows(2, tokens=1 << 30), rows(3, tokens=1 << 30), None, None, SHAPE),
    (rows(1, reserved=1), rows(2), H, Y, None, INVALID),
    (rows(1, data=0x100002), rows(2), H, Y, None, INVALID),
    (rows(1, data=None), rows(2), H, Y, None, INVALID),
    (rows(1, stride_token=-8), rows(2), H, Y, None, INVALID),
    (rows(1, stride_batch=1 << 46), rows(2), H, Y, None, INVALID),
    (rows(1), rows(2), rows(3, stride_token=4), Y, None, INVALID),             # rows of h overlap
    (rows(1), rows(2), rows(3, stride_batch=0), Y, None, INVALID),
    (rows(1, stride_batch=0), rows(2), H, Y, None, DEVICE),                    # a broadcast input
    (rows(1), rows(2), rows(1, data=0x100020), Y, None, INVALID),              # h overlaps x
    (rows(1), rows(2), H, Y, options(scale=math.inf), INVALID),
    (rows(1), rows(2), H, Y, options(scale=1e39), INVALID),
    (rows(1), rows(2), H, Y, options(scale=math.nan), INVALID),
    (rows(1), rows(2), H, Y, options(eps=-1.0), INVALID),
    (rows(1), rows(2), H, Y, options(eps=math.nan), INVALID),
    (rows(1), rows(2), H, Y, options(post_norm=2), INVALID),
    (rows(1), rows(2), H, Y, options(reserved=1), INVALID),
    (rows(1), rows(2), H, Y, options(post=tensor(8)), INVALID),                # a weight without its norm
    (rows(1), rows(2), H, Y, options(post=tensor(8), post_norm=1), DEVICE),
    (rows(1), rows(2), H, Y, options(gate=tensor(7)), SHAPE),
    (rows(1), rows(2), H, Y, options(gate=tensor(3, 8)), SHAPE),
    (rows(1), rows(2), H, Y, options(gate=tensor(2, 8)), DEVICE),
    (rows(1), rows(2), H, Y, options(gate=tensor(8, dtype=BF16)), DTYPE),
    (rows(1), rows(2), H, Y, options(nxt=tensor(8, at=0)), INVALID),
    (rows(1), rows(2), H, Y, options(gate=tensor(8, at=3)), INVALID),          # h over a weight
    (rows(1), rows(2), H, Y, options(drop=drop(-0.1)), INVALID),
    (rows(1), rows(2), H, Y, options(drop=drop(1.1)), INVALID),
    (rows(1), rows(2), H, Y, options(drop=drop(math.nan)), INVALID),
    (rows(1), rows(2), H, Y, options(drop=drop(0.5, 0x1004)), INVALID),
    (rows(1), rows(2), H, Y, options(drop=drop(0.5, 0x300008)), INVALID),      # the counter in h
    (rows(1, tokens=0), rows(2, tokens=0), rows(3, tokens=0), None, None, 0),
])
def test_residual_norm_refuses(x, f, h, y, opt, status):
    assert residual(x, f, h, y, opt) == status
    assert bool(disco.library().disco_last_error()) == (status != 0)


def backward(opt, dh=rows(5), dy=rows(6), dx=rows(7), df=rows(8), dw=(None, None, None), x=rows(1), f=rows(2), ws=None, n=0):
    return disco.library().disco_residual_norm_backward(ref(x), ref(f), ref(opt), ref(dh), ref(dy), ref(dx), ref(df), *map(ref, dw),
                                                        ws, n, None)


def test_residual_norm_backward_refuses():
    assert backward(None) == DEVICE
    assert backward(None, dh=None) == DEVICE and backward(None, dy=None) == DEVICE
    assert backward(None, dh=None, dy=None) == INVALID
    assert backward(None, x=None) == INVALID                        # dx without x
    assert backward(None, x=None, dx=None) == DEVICE
    assert backward(None, dx=rows(5), df=rows(6)) == DEVICE         # in place
    assert backward(None, dx=rows(5), df=rows(5)) == INVALID
    assert backward(None, dx=rows(5, data=0x500020)) == INVALID
    opt = options(post=tensor(8), post_norm=1, gate=tensor(2, 8, at=41), nxt=tensor(8, at=42))
    assert backward(opt, dw=(tensor(8, at=50), tensor(2, 8, at=51), tensor(8, at=52))) == DEVICE
    assert backward(opt, dw=(tensor(7, at=50), None, None)) == SHAPE
    assert backward(opt, dw=(tensor(8, at=50, dtype=BF16), None, None)) == DTYPE
    assert backward(opt, dw=(tensor(8, at=0), None, None)) == INVALID
    assert backward(opt, dw=(tensor(8, at=2), None, None)) == INVALID      # in f
    assert backward(opt, dw=(tensor(8, at=50), None, tensor(8, at=50))) == INVALID
    assert backward(None, dw=(tensor(8, at=50), None, None)) == INVALID    # no such weight


def test_dropout_refuses():
    call = lambda x, d, y: disco.library().disco_dropout(ref(x), ref(d), ref(y), None)
    assert call(rows(1), drop(), rows(2)) == DEVICE and call(rows(1), drop(), rows(1)) == DEVICE
    assert call(rows(1), None, rows(2)) == INVALID
    assert call(rows(1), drop(2.0), rows(2)) == INVALID
    assert call(rows(1), drop(), rows(1, data=0x100020)) == INVALID
    assert call(rows(1), drop(), rows(2, channels=7)) == SHAPE
    assert call(rows(1), drop(), rows(2, dtype=BF16)) == DTYPE
    big = dict(batch=1, tokens=1 << 20, channels=1 << 14, stride_token=1 << 14, stride_batch=0)
    assert call(rows(1, **big), drop(), rows(0x100000, **big)) == SHAPE
    assert call(rows(1, tokens=0), drop(), rows(2, tokens=0)) == 0


def recur(x=rows(1), g=rows(2), z=None, opt=None, state=None, y=rows(4), last=None, carries=None, ws=None, n=0):
    return disco.library().disco_gated_recurrence(ref(x), ref(g), ref(z), ref(opt), state, ref(y), last, carries, ws, n, None)


@pytest.mark.parametrize("kw,status", [
    ({}, DEVICE),
    (dict(y=rows(1)), DEVICE), (dict(y=rows(2)), DEVICE), (dict(z=rows(3), y=rows(3)), DEVICE),  # in place
    (dict(x=None), INVALID), (dict(g=None), INVALID), (dict(y=None), INVALID),
    (dict(g=rows(2, channels=4)), SHAPE), (dict(z=rows(3, tokens=4)), SHAPE), (dict(y=rows(4, batch=3)), SHAPE),
    (dict(g=rows(2, dtype=BF16)), DTYPE),
    (dict(x=rows(1, channels=(1 << 24) + 1)), SHAPE),
    (dict(x=rows(1, batch=1 << 20, channels=1 << 12, tokens=1), g=rows(2, batch=1 << 20, channels=1 << 12, tokens=1)), SHAPE),
    (dict(y=rows(4, stride_token=4)), INVALID),
    (dict(y=rows(1, data=0x100020)), INVALID),
    (dict(opt=disco.RecurrenceArgs(3, 0, None)), INVALID),
    (dict(opt=disco.RecurrenceArgs(0, 1, None)), INVALID),
    (dict(opt=disco.RecurrenceArgs(0, 0, 0x400004)), INVALID),            # lengths in y
    (dict(state=0xA00000, last=0xA00000), DEVICE),
    (dict(state=0xA00000, last=0xA00010), INVALID),
    (dict(last=0x100010), INVALID), (dict(carries=0x200010), INVALID), (dict(carries=0xA00000, last=0xA00010), INVALID),
    (dict(state=0xA00000, carries=0xA00010), INVALID),
    (dict(x=rows(1, batch=0), g=rows(2, batch=0), y=rows(4, batch=0)), 0),
    (dict(x=rows(1, tokens=0), g=rows(2, tokens=0), y=rows(4, tokens=0)), 0),
])
def test_gated_recurrence_refuses(kw, status):
    assert recur(**kw) == status
    assert bool(disco.library().disco_last_error()) == (status != 0)


def test_gated_recurrence_backward_refuses():
    def call(x=rows(1), g=rows(2), z=rows(3), opt=None, carries=0x2000000, dy=rows(5), dlast=None, dx=rows(6), dg=rows(7),
             dz=rows(8), dstate=None):
        return disco.library().disco_gated_recurrence_backward(ref(x), ref(g), ref(z), ref(opt), carries, ref(dy), dlast, ref(dx),
                                                               ref(dg), ref(dz), dstate, None, 0, None)
    assert call() == DEVICE
    assert call(dx=rows(1), dg=rows(2), dz=rows(3)) == DEVICE
    assert call(dx=rows(5)) == DEVICE
    assert call(dx=rows(6), dg=rows(6)) == INVALID
    assert call(carries=None) == INVALID
    assert call(z=None) == INVALID
    assert call(z=None, dz=None) == DEVICE
    assert call(dy=None) == INVALID
    assert call(dlast=0xA00000, dstate=0xA00000) == DEVICE
    assert call(dlast=0xA00000, dstate=0xA00010) == INVALID
    assert call(dx=rows(0x20)) == INVALID                                # over the carries
    assert call(dx=None, dg=None, dz=None) == 0


def test_workspace_sizes_are_host_arithmetic():
    lib, n = disco.library(), ctypes.c_size_t()
    assert lib.disco_gated_recurrence_workspace(ref(rows(1)), n) == 0 and n.value == 0
    assert lib.disco_gated_recurrence_workspace(ref(rows(1, tokens=100000)), n) == 0 and n.value > 0  # one long series: splits
    assert lib.disco_gated_recurrence_workspace(ref(rows(1, tokens=24, batch=100000)), n) == 0 and n.value == 0
    assert lib.disco_gated_recurrence_workspace(ref(rows(1)), None) == INVALID
    assert lib.disco_residual_norm_workspace(ref(rows(1)), None, n) == 0 and n.value == 0
    opt = options(gate=tensor(8))
    assert lib.disco_residual_norm_workspace(ref(rows(1)), ref(opt), n) == 0 and n.value > 0
    shared = n.value
    opt = options(gate=tensor(2, 8))
    assert lib.disco_residual_norm_workspace(ref(rows(1)), ref(opt), n) == 0 and n.value > shared


def test_generator_gives_its_published_values():
    """Known answers of Philox4x32-10 (its authors' test vectors), through the reference of the GPU tests."""
    def words(counter, key):
        # row and block of the counter's first two words: one entry of a mask tells whether its half is at least a bound
        got = []
        for half in range(8):
            lo, hi = 0, 65536
            while hi - lo > 1:
                mid = (lo + hi) // 2
                seed, offset = key[0] | key[1] << 32, counter[2] | counter[3] << 32
                stays = kept(counter[1] + 1, 8 * (counter[0] + 1), seed, offset, mid)[counter[1], 8 * counter[0] + half]
                lo, hi = (mid, hi) if stays else (lo, mid)
            got.append(lo)
        return [got[2 * i] | got[2 * i + 1] << 16 for i in range(4)]
    assert words((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    # a share of entries as asked for
    share = kept(500, 1000, 7, 1, round(0.3 * 65536)).mean()
    assert abs(share - 0.7) < 5 * math.sqrt(0.21 / 500000)
    assert np.array_equal(kept(5, 21, 3, 4, 30000), kept(9, 24, 3, 4, 30000)[:5, :21])
