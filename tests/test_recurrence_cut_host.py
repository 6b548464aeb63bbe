"""How a recurrence call is cut, as its scratch memory shows it (host arithmetic: no memory stands behind the tensors).

Few long series are scanned along time in several parts, which takes scratch memory; threads that walk alone take none.
"""
import ctypes

import pytest

from paper_2209_13603_amd import disco

F32, BF16 = disco.DISCO_FLOAT32, disco.DISCO_BFLOAT16


def workspace(batch, tokens, channels, dtype, stride_token=None, stride_batch=None):
    st = stride_token or channels
    sb = stride_batch if stride_batch is not None else tokens * st
    rows, n = disco.Rows(0x1000000, dtype, 0, batch, tokens, channels, sb, st), ctypes.c_size_t()
    assert disco.library().disco_gated_recurrence_workspace(ctypes.byref(rows), n) == 0
    return n.value


@pytest.mark.parametrize("batch,tokens,channels,dtype,parts", [
    (2, 200000, 2048, BF16, 3), (2, 131072, 1536, F32, 3),        # parts of a joint projection: items 1.2e9 and 6e8 apart
    (2, 200000, 2050, BF16, 3), (3, 131072, 1501, F32, 3),        # channels that do not fill whole workgroups
    (2, 1000000, 1100, BF16, 1), (7, 1000000, 130, F32, 5),
])
def test_items_far_apart_are_scanned_as_one_is(batch, tokens, channels, dtype, parts):
    st = parts * channels
    far = workspace(batch, tokens, channels, dtype, st)
    assert workspace(1, tokens, channels, dtype, st) > 0
    near = workspace(batch, tokens, channels, dtype, st, stride_batch=0)  # (one series for all items)
    assert 0 < far <= near
    if channels % 64 == 0:
        assert far == near


@pytest.mark.parametrize("dtype,apart", [(BF16, 1 << 23), (F32, 1 << 22)])
def test_steps_too_far_apart_walk_alone(dtype, apart):
    """256 steps of a workgroup within 2^31 bytes, or no scan."""
    assert workspace(1, 4096, 64, dtype, apart) == 0
    assert workspace(1, 4096, 64, dtype, apart // 4) > 0
