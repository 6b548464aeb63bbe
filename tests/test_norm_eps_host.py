"""An eps that fp32 does not hold is refused by the calls that norm rows: taken as infinity it made every row zero."""
import ctypes

import pytest

from paper_2209_13603_amd import disco

EPS = [(1e39, disco.DISCO_ERR_INVALID_ARGUMENT), (1e300, disco.DISCO_ERR_INVALID_ARGUMENT),
       (float("inf"), disco.DISCO_ERR_INVALID_ARGUMENT), (3.4e38, disco.DISCO_ERR_DEVICE), (0.0, disco.DISCO_ERR_DEVICE),
       (1e-300, disco.DISCO_ERR_DEVICE)]


def rows(at):
    return disco.Rows(at * 0x100000, disco.DISCO_FLOAT32, 0, 2, 3, 8, 24, 8)


@pytest.mark.parametrize("eps,status", EPS)
def test_residual_norm(eps, status):
    opt = disco.ResidualArgs(1.0, eps, 1, 0, None, None, None, None)
    r = [ctypes.byref(rows(i)) for i in range(1, 7)]
    lib, o = disco.library(), ctypes.byref(opt)
    assert lib.disco_residual_norm(r[0], r[1], o, r[2], r[3], None) == status
    assert lib.disco_residual_norm_backward(r[0], r[1], o, r[2], r[3], r[4], r[5], None, None, None, None, 0, None) == status


@pytest.mark.parametrize("eps,status", EPS)
def test_norm_rotate(eps, status):
    h = [ctypes.byref(disco.Heads(at * 0x100000, disco.DISCO_FLOAT32, 8, 2, 0, 1, 3, 48, 16, 8)) for at in range(1, 4)]
    lib = disco.library()
    assert lib.disco_norm_rotate(h[0], 1, None, eps, None, h[1], None) == status
    assert lib.disco_norm_rotate(h[0], 0, None, 1e39, None, h[1], None) == disco.DISCO_ERR_DEVICE  # no norm, no eps
