"""Calls of more rows than 32-bit counts of their parts hold, and than one axis of a launch takes (2^32 threads)."""
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


def test_norm_rotate_of_more_than_2_to_26_wide_rows():
    """Heads of 65 take 64 lanes a row, in place, forward and back."""
    import torch
    from paper_2209_13603_amd import attention
    n, D = (1 << 14) + 1, 65
    g = torch.Generator(device="cuda:0").manual_seed(1)
    base = torch.randn(1, 4096, 1, D, generator=g, device="cuda:0").bfloat16()
    grad = torch.randn(1, 4096, 1, D, generator=g, device="cuda:0").bfloat16()
    x = base.expand(n, 4096, 1, D).reshape(1, n * 4096, 1, D)
    dy = grad.expand(n, 4096, 1, D).reshape(1, n * 4096, 1, D)
    assert x.shape[1] > 1 << 26
    attention.norm_rotate_backward(x, None, dy, dx=dy)
    want, _ = attention.norm_rotate_backward(base, None, grad)
    assert bool((dy.view(n, 4096, D) == want.view(4096, D)).all())
    del dy
    attention.norm_rotate(x, y=x)
    want = attention.norm_rotate(base)
    assert bool((x.view(n, 4096, D) == want.view(4096, D)).all())


def test_attention_of_more_than_2_to_31_rows():
    import torch
    from paper_2209_13603_amd import attention
    tokens = (1 << 29) + 64
    g = torch.Generator(device="cuda:0").manual_seed(2)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda:0").bfloat16()
    q, dout, k, v = mk(2, 1, 2, 1), mk(2, 1, 2, 1), mk(2, 3, 2, 1), mk(2, 3, 2, 1)
    small = [t.expand(2, 64, 2, 1) for t in (q, dout)]
    large = [t.expand(2, tokens, 2, 1) for t in (q, dout)]
    assert 2 * tokens * 2 > 1 << 31
    out, stats = attention.cross_attention(small[0], k, v, return_stats=True)
    want, (dq, _, _) = out, attention.cross_attention_backward(small[0], k, v, out, stats, small[1])
    out = torch.full((2, tokens, 2, 1), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    _, stats = attention.cross_attention(large[0], k, v, return_stats=True, out=out)
    assert bool((out == want[:, :1]).all())
    got, _, _ = attention.cross_attention_backward(large[0], k, v, out, stats, large[1])
    assert bool((got == dq[:, :1]).all())
