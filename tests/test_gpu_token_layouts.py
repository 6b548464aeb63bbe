"""Token tensors as parts of joint buffers in other orders of their axes: the same bits as in buffers of their own."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("order", ["b2hsd", "bsh2d", "2bshd", "b2shd"])
def test_gradients_into_one_buffer(order, dtype):
    import torch
    from paper_2209_13603_amd import attention
    g = torch.Generator(device="cuda:0").manual_seed(1)
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    size = {"b": 3, "2": 2, "h": 2, "s": 70, "d": 64}
    mk = lambda *s: torch.randn(s, generator=g, device="cuda:0").to(dt)
    q, k, v, dout = mk(3, 50, 4, 64), mk(3, 70, 2, 64), mk(3, 70, 2, 64), mk(3, 50, 4, 64)
    out, stats = attention.cross_attention(q, k, v, return_stats=True)
    want = attention.cross_attention_backward(q, k, v, out, stats, dout)
    joint = torch.full([size[c] for c in order], float("nan"), device="cuda:0").to(dt)
    parts = joint.permute([order.index(c) for c in "2bshd"])
    got = attention.cross_attention_backward(q, k, v, out, stats, dout, dk=parts[0], dv=parts[1])
    assert all(bool((a == b).all()) for a, b in zip(got, want))
    assert bool((parts[0] == want[1]).all()) and bool((parts[1] == want[2]).all())
