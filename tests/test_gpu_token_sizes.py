"""Cross attention of more rows than 32-bit counts of their parts hold."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _free():
    yield
    import torch
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def test_gradients_of_2_to_29_queries():
    """One query over and over: dk and dv are its gradients as often.  The sums of some 2^17 equal tiles in fp32 round the
    same way each time: 2^17 times 2^-24 of the sum, tested at 2^-5."""
    import torch
    from paper_2209_13603_amd import attention
    tokens = (1 << 29) + 64
    q, dout = (torch.full((1, 1, 1, 1), c, device="cuda:0").bfloat16() for c in (1.5, 0.75))
    k = torch.tensor([1.0, -0.5, 0.25], device="cuda:0").view(1, 3, 1, 1).bfloat16()
    v = torch.tensor([2.0, -1.0, 4.0], device="cuda:0").view(1, 3, 1, 1).bfloat16()
    out, stats = attention.cross_attention(q.expand(1, tokens, 1, 1), k, v, return_stats=True)
    dq, dk, dv = attention.cross_attention_backward(q.expand(1, tokens, 1, 1), k, v, out, stats, dout.expand(1, tokens, 1, 1))
    p = torch.softmax(1.5 * k.double().cpu().view(3), 0)
    o = float((p * v.double().cpu().view(3)).sum())
    ds = p * 0.75 * (v.double().cpu().view(3) - o)
    for got, want in ((dk, ds * 1.5 * tokens), (dv, p * 0.75 * tokens)):
        got = got.double().cpu().view(3)
        assert float((got - want).norm()) <= 2.0 ** -5 * float(want.norm()), (got, want)
    assert abs(float(out[0, -1]) - o) <= 2.0 ** -7 * abs(o)
    assert abs(float(dq[0, -1]) - float((ds * k.double().cpu().view(3)).sum())) <= 2.0 ** -7 * float(ds.norm())
