"""Numbers of token calls that fp32, in which the kernels take them, does not hold: refused before any device call."""
import math

import pytest

from paper_2209_13603_amd import disco
from test_heads_host import attend, heads

FAR = {n: heads(data=0x4000000 * n) for n in (1, 2, 3, 4)}


@pytest.mark.parametrize("scale,status", [
    (1e300, disco.DISCO_ERR_INVALID_ARGUMENT), (-1e39, disco.DISCO_ERR_INVALID_ARGUMENT), (3e38, disco.DISCO_ERR_INVALID_ARGUMENT),
    (1e-300, disco.DISCO_ERR_INVALID_ARGUMENT), (-1e-46, disco.DISCO_ERR_INVALID_ARGUMENT), (1e-39, disco.DISCO_ERR_INVALID_ARGUMENT),
    (math.nan, disco.DISCO_ERR_INVALID_ARGUMENT), (-math.inf, disco.DISCO_ERR_INVALID_ARGUMENT),
    # what it holds goes on, to the device that knows no such addresses
    (2e38, disco.DISCO_ERR_DEVICE), (-1e-37, disco.DISCO_ERR_DEVICE), (0.0, disco.DISCO_ERR_DEVICE),
])
def test_attention_scales(scale, status):
    opt = disco.AttentionArgs(scale, None, 0, None)
    assert attend(FAR[1], FAR[2], FAR[3], FAR[4], opt) == status
