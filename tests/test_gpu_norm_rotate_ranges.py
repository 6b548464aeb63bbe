"""Head norm with rotation for rows whose squares leave the range of fp32, beside ordinary rows, against the definition in 64
bits, row by row.  Rows are of entries between 1e-40 and 3e37; the norm makes them of order one again.  Tolerances: those of
test_gpu_norm_rotate.py, and two of the smallest values that the type holds."""
import pytest

from test_gpu_norm_rotate import TOL, _exact

pytestmark = pytest.mark.gpu

LEAST = {"bf16": 2.0 ** -133, "fp32": 2.0 ** -149}


def _rows(got, want, tol, least):
    import torch
    got, want = got.detach().cpu().double(), want.double()
    assert torch.isfinite(got).all()
    err, size = (got - want).norm(dim=-1), want.norm(dim=-1)
    bound = tol * size + 2 * least * want.shape[-1] ** 0.5
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(2, 30, 3, 64, 64), (1, 41, 5, 36, 20), (2, 9, 2, 127, 0), (1, 50, 1, 128, 64)])
@pytest.mark.parametrize("weight", ["none", "shared"])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-50])
def test_rows_of_any_size(eps, weight, shape, dtype):
    import torch
    from paper_2209_13603_amd import attention
    B, S, H, D, R = shape
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(D)
    size = 10.0 ** torch.tensor([0.0, 18.0, 20.0, 30.0, 37.0, -12.0, -18.0, -22.0, -30.0, -36.0], dtype=torch.float64)
    size = size[torch.randint(0, 10, (B, S, H, 1), generator=g)]
    x = (size * torch.randn(B, S, H, D, generator=g).double()).to("cuda:0", dt)
    dy = torch.randn(B, S, H, D, generator=g).to("cuda:0", dt)
    w = (1 + 0.2 * torch.randn(D, generator=g)).to("cuda:0", dt) if weight == "shared" else None
    angle = 20 * torch.randn(S, R // 2, generator=g).cuda()
    pos = torch.arange(S, dtype=torch.int32)[None].expand(B, S)
    kw = dict(rotation=(angle.cos(), angle.sin()), eps=eps)
    want = _exact(x, w, dy, angle.cos(), angle.sin(), pos, "half", True, eps)
    _rows(attention.norm_rotate(x, w, **kw), want[0], TOL[dtype], LEAST[dtype])
    # gradients of rows below 1e-37 pass the largest value that the types hold
    small = size < 1e-35
    dy = torch.where(small.cuda(), dy * 1e-3, dy)
    want = _exact(x, w, dy, angle.cos(), angle.sin(), pos, "half", True, eps)
    dx, dw = attention.norm_rotate_backward(x, w, dy, **kw)
    _rows(dx, want[1], TOL[dtype], LEAST[dtype])
    if w is not None:
        _rows(dw, want[2], TOL[dtype] if dtype == "bf16" else 5e-6, LEAST[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_zero_rows(dtype):
    """Zeros where eps is above zero, however little; 0 / 0 where it is not."""
    import torch
    from paper_2209_13603_amd import attention
    x = torch.ones(1, 4, 2, 64, device="cuda:0").to({"bf16": torch.bfloat16, "fp32": torch.float32}[dtype])
    x[0, 1] = 0
    for eps in (1e-6, 1e-40, 1e-50):
        assert not attention.norm_rotate(x, eps=eps)[0, 1].any()
    assert bool(torch.isnan(attention.norm_rotate(x, eps=0.0)[0, 1].float()).all())
