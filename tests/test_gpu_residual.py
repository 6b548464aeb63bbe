"""Residual sum with its norms, gate and dropout, and its gradients, against the definition in 64 bits.

Tolerances: relative 2-norm.  Both types hold everything in fp32 between one load and one rounding, so bf16 has its
rounding alone (at most 2^-8).  fp32: some ten roundings of 2^-24 an entry, and half the error of the two sums of squares,
each of at most 32 terms in a row a thread and 10 levels above (21 x 2^-24): 2e-6.  Gradients of weights add up to a few
thousand rows whose terms cancel to their root: 5e-6.
"""
import pytest

from block_forms import dropout_factor, rel, residual

pytestmark = pytest.mark.gpu

TOL = {"bf16": 2.0 ** -8 + 2e-6, "fp32": 2e-6}


def _inputs(B, S, C, dtype, seed=0, per_item=()):
    import torch
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    g = torch.Generator(device="cuda:0").manual_seed(seed + B + 3 * S + 7 * C)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda:0")
    x, f, dh, dy = (rnd(B, S, C).mul(m).to(dt) for m in (2.0, 0.7, 1.0, 1.0))
    w = {k: (1 + 0.3 * rnd(*((B, C) if k in per_item else (C,)))).to(dt) for k in ("post_weight", "gate", "next_weight")}
    return x, f, dh, dy, w


def _all(x, f, dh, dy, kw, dtype):
    from paper_2209_13603_amd import blocks
    factor = dropout_factor(tuple(f.shape), kw["dropout"]) if kw.get("dropout") else None
    form = lambda a, b: residual(x, f, a, b, kw.get("post_norm", False), kw.get("post_weight"), kw.get("gate"),
                                 kw.get("next_weight"), kw.get("scale", 1.0), kw.get("eps", 1e-6), factor)
    want = form(dh, dy)
    h, y = blocks.residual_norm(x, f, **kw)
    assert rel(h, want[0]) <= TOL[dtype] and rel(y, want[1]) <= TOL[dtype]
    g = blocks.residual_norm_backward(x, f, dh, dy, **kw)
    names = [n for n, t in (("dx", x), ("df", f), ("dpost_weight", kw.get("post_weight")), ("dgate", kw.get("gate")),
                            ("dnext_weight", kw.get("next_weight"))) if t is not None]
    for n, v in zip(names, want[2:]):
        got = getattr(g, n)
        if v is None:  # the output that it works through is not there
            assert not got.any(), n
            continue
        if f.shape[-1] == 1 and n in ("dx", "df"):
            continue  # a norm of one entry is its sign: two terms that cancel wholly
        assert got.shape == v.shape
        assert rel(got, v) <= (5e-6 if dtype == "fp32" and n[-1] in "et" and n not in ("dx", "df") else TOL[dtype]), n
    for n in ("dx", "df", "dpost_weight", "dgate", "dnext_weight"):
        assert (getattr(g, n) is None) == (n not in names)
    again = blocks.residual_norm_backward(x, f, dh, dy, **kw)
    for a, b in zip(g, again):
        assert a is None or bool((a == b).all())
    return h, y, g


SHAPES = [(1, 1, 8), (1, 1, 1024), (2, 1, 64), (3, 7, 16), (1, 5, 1), (2, 3, 7), (1, 33, 180), (2, 40, 150), (2, 65, 512),
          (1, 19, 520), (2, 9, 1000), (1, 6, 2048), (2, 5, 2056), (1, 4, 4100), (2, 3, 8192), (1, 3, 8190), (1, 2, 8185),
          (3, 700, 24), (1, 5000, 40)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["all", "plain", "per_item", "norm_alone"])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_definition(shape, kind, dtype):
    from paper_2209_13603_amd import blocks
    x, f, dh, dy, w = _inputs(*shape, dtype, per_item=("post_weight", "gate", "next_weight") if kind == "per_item" else ())
    kw = {"all": dict(post_norm=True, dropout=blocks.Dropout(0.2, 9, 4), scale=0.8, **w),
          "per_item": dict(post_norm=True, dropout=blocks.Dropout(0.2, 9, 4), **w),
          "plain": {}, "norm_alone": dict(next_weight=w["next_weight"], eps=1e-5)}[kind]
    _all(None if kind == "norm_alone" else x, f, dh, dy, kw, dtype)


@pytest.mark.parametrize("mixed", [("post_weight",), ("gate",), ("next_weight",), ("post_weight", "next_weight")])
@pytest.mark.parametrize("shape", [(5, 37, 72), (40, 3, 24), (3, 1, 600), (2, 900, 16)])
def test_weights_by_item_beside_shared_ones(shape, mixed):
    """Runs of rows that begin and end inside items."""
    x, f, dh, dy, w = _inputs(*shape, "fp32", per_item=mixed)
    _all(x, f, dh, dy, dict(post_norm=True, **w), "fp32")


@pytest.mark.parametrize("missing", ["dh", "dy"])
def test_one_gradient_alone(missing):
    x, f, dh, dy, w = _inputs(2, 21, 56, "fp32")
    kw = dict(post_norm=True, **w)
    _all(x, f, None if missing == "dh" else dh, None if missing == "dy" else dy, kw, "fp32")


def test_outputs_alone_and_in_place():
    import torch
    from paper_2209_13603_amd import blocks
    x, f, dh, dy, w = _inputs(2, 30, 320, "bf16")
    kw = dict(post_norm=True, dropout=blocks.Dropout(0.1, 3), **w)
    h, y = blocks.residual_norm(x, f, **kw)
    h1, none = blocks.residual_norm(x, f, want_y=False, **kw)
    none2, y1 = blocks.residual_norm(x, f, want_h=False, **kw)
    assert none is None and none2 is None and bool((h1 == h).all()) and bool((y1 == y).all())
    a, b = x.clone(), f.clone()
    blocks.residual_norm(a, b, h=a, y=b, **kw)
    assert bool((a == h).all()) and bool((b == y).all())
    want = blocks.residual_norm_backward(x, f, dh, dy, **kw)
    for place in ("gradients", "inputs", "crossed"):
        t = [v.clone() for v in (x, f, dh, dy)]
        dx, df = {"gradients": (t[2], t[3]), "inputs": (t[0], t[1]), "crossed": (t[3], t[0])}[place]
        g = blocks.residual_norm_backward(*t, dx=dx, df=df, **kw)
        assert g.dx is dx and g.df is df
        for u, v in zip(g, want):
            assert bool((u == v).all())
    g = blocks.residual_norm_backward(x, f, dh, dy, want_dx=False, want_weights=False, **kw)
    assert g.dx is None and g.dgate is None and bool((g.df == want.df).all())
    g = blocks.residual_norm_backward(x, f, dh, dy, want_dx=False, want_df=False, **kw)
    assert g.dx is None and g.df is None and bool((g.dgate == want.dgate).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("channels", [5, 12, 14, 64])
def test_strides(channels, dtype):
    """Parts of joint buffers, other orders of the axes, broadcast inputs and addresses off the wide pieces."""
    import torch
    from paper_2209_13603_amd import blocks
    x, f, dh, dy, w = _inputs(3, 10, channels, dtype)
    kw = dict(post_norm=True, dropout=blocks.Dropout(0.3, 8, 1), **w)
    h, y = blocks.residual_norm(x, f, **kw)
    g = blocks.residual_norm_backward(x, f, dh, dy, **kw)

    def joint(t):
        j = torch.zeros(3, 10, 2, channels, dtype=t.dtype, device=t.device)
        j[:, :, 1] = t
        return j[:, :, 1]

    def major(t):
        return t.transpose(0, 1).contiguous().transpose(0, 1)

    def odd(t):
        flat = torch.zeros(t.numel() + 1, dtype=t.dtype, device=t.device)
        flat[1:] = t.flatten()
        return flat[1:].view(t.shape)

    for lay in (joint, major, odd):
        h2, y2 = blocks.residual_norm(lay(x), lay(f), h=lay(h), y=lay(y), **kw)
        g2 = blocks.residual_norm_backward(lay(x), lay(f), lay(dh), lay(dy), dx=lay(dh), df=lay(dy), **kw)
        for u, v in zip((h2, y2, *g2), (h, y, *g)):
            assert rel(u, v.double().cpu()) <= TOL[dtype]
    shared = x[:1].expand(3, 10, channels)
    h3, y3 = blocks.residual_norm(shared, f, **kw)
    h4, y4 = blocks.residual_norm(shared.contiguous(), f, **kw)
    assert bool((h3 == h4).all()) and bool((y3 == y4).all())


@pytest.mark.parametrize("factor", [1e-30, 1e-18, 1e18, 3e36])
def test_rows_whose_squares_leave_fp32(factor):
    """Norms of entries of any size.  eps is too small to count beside them."""
    import torch
    from paper_2209_13603_amd import blocks
    x, f, dh, dy, w = _inputs(2, 12, 96, "fp32")
    x, f = x * factor, f * factor
    kw = dict(post_norm=True, eps=0.0, post_weight=w["post_weight"], next_weight=w["next_weight"])
    # (f is normed to order one: as the residual it counts where x is small, and not beside a large x)
    want = residual(None, f, dh, dy, True, w["post_weight"], None, w["next_weight"], 1.0, 0.0, None)
    h, y = blocks.residual_norm(None, f, **kw)
    assert rel(h, want[0]) <= 2e-6 and rel(y, want[1]) <= 2e-6
    g = blocks.residual_norm_backward(None, f, dh, dy, **kw)
    if factor < 1e30:  # (df of order 1 / factor stays in the normal range)
        assert rel(g.df * factor, want[2] * factor) <= 2e-6 if factor > 1e-20 else bool(torch.isfinite(g.df).all())
    kw = dict(eps=0.0, next_weight=w["next_weight"])
    want = residual(x, f, None, dy, False, None, None, w["next_weight"], 1.0, 0.0, None)
    _, y = blocks.residual_norm(x, f, want_h=False, **kw)
    assert rel(y, want[1]) <= 2e-6


def test_weights_without_an_eps():
    """Slots of a workgroup that have no row bring nothing to the sums."""
    for shape in ((1, 1, 40), (1, 7, 96), (3, 5, 24)):
        x, f, dh, dy, w = _inputs(*shape, "fp32")
        _all(x, f, dh, dy, dict(post_norm=True, eps=0.0, **w), "fp32")


def test_what_is_not_finite_stays_in_its_row():
    import torch
    from paper_2209_13603_amd import blocks
    for channels in (40, 600, 2100):
        x, f, dh, dy, w = _inputs(2, 11, channels, "fp32")
        kw = dict(post_norm=True, post_weight=w["post_weight"], gate=w["gate"], next_weight=w["next_weight"])
        want = blocks.residual_norm(x, f, **kw)
        gw = blocks.residual_norm_backward(x, f, dh, dy, **kw)
        x[0, 3, 5], f[1, 7, 2] = float("nan"), float("inf")
        got = blocks.residual_norm(x, f, **kw)
        g = blocks.residual_norm_backward(x, f, dh, dy, **kw)
        ok = torch.ones(2, 11, dtype=torch.bool, device="cuda:0")
        ok[0, 3] = ok[1, 7] = False
        for u, v in zip((*got, g.dx, g.df), (*want, gw.dx, gw.df)):
            assert bool((u[ok] == v[ok]).all())
            assert not bool(torch.isfinite(u[~ok]).all())


def test_zero_rows_and_no_rows():
    import torch
    from paper_2209_13603_amd import blocks
    x, f, dh, dy, w = _inputs(2, 5, 48, "fp32", per_item=("gate",))
    kw = dict(post_norm=True, **w)
    z = torch.zeros_like(x)
    h, y = blocks.residual_norm(z, z, **kw)
    assert not h.any() and not y.any()
    g = blocks.residual_norm_backward(z, z, dh, dy, **kw)
    assert all(bool(torch.isfinite(t).all()) for t in g)
    none = x[:, :0]
    h, y = blocks.residual_norm(none, none, **kw)
    assert h.shape == y.shape == (2, 0, 48)
    g = blocks.residual_norm_backward(none, none, none, none, **kw)
    assert g.dx.shape == (2, 0, 48)
    assert not any(t.any() for t in (g.dpost_weight, g.dgate, g.dnext_weight)) and g.dgate.shape == (2, 48)
    kw["gate"] = kw["gate"][:0]
    g = blocks.residual_norm_backward(x[:0], f[:0], dh[:0], dy[:0], **kw)
    assert g.dgate.shape == (0, 48) and not g.dpost_weight.any()


def test_gradients_against_differences():
    """Central differences of the kernel's own outputs, fp32: truncation 1e-4 of the step's square, rounding 2^-23 of
    sums of some hundred terms over steps of 1e-2."""
    import torch
    from paper_2209_13603_amd import blocks
    x, f, dh, dy, w = _inputs(1, 3, 24, "fp32")
    base = dict(x=x, f=f, **w)
    drop = blocks.Dropout(0.25, 6)

    def total(p):
        h, y = blocks.residual_norm(p["x"], p["f"], post_norm=True, post_weight=p["post_weight"], gate=p["gate"],
                                    next_weight=p["next_weight"], dropout=drop, scale=0.9)
        return float((h.double() * dh.double()).sum() + (y.double() * dy.double()).sum())

    g = blocks.residual_norm_backward(x, f, dh, dy, post_norm=True, dropout=drop, scale=0.9, **w)
    for name, grad in (("x", g.dx), ("f", g.df), ("post_weight", g.dpost_weight), ("gate", g.dgate), ("next_weight", g.dnext_weight)):
        d = torch.randn(base[name].shape, generator=torch.Generator(device="cuda:0").manual_seed(5), device="cuda:0")
        eps = 1e-2
        diff = (total({**base, name: base[name] + eps * d}) - total({**base, name: base[name] - eps * d})) / (2 * eps)
        want = float((grad.double() * d.double()).sum())
        size = float(grad.double().norm() * d.double().norm())
        assert abs(diff - want) <= 2e-3 * size, name


def test_refusals():
    import torch
    from paper_2209_13603_amd import blocks, disco
    x, f, dh, dy, w = _inputs(2, 5, 48, "fp32")
    with pytest.raises(ValueError):
        blocks.residual_norm(x.transpose(1, 2), f)
    with pytest.raises(ValueError):
        blocks.residual_norm(x, f[0])
    with pytest.raises(ValueError):
        blocks.residual_norm(x.cpu(), f)
    with pytest.raises(ValueError):
        blocks.residual_norm(x, f, gate=torch.ones(48, 2, device="cuda:0").t()[0])
    with pytest.raises(disco.DiscoError):
        blocks.residual_norm(x, f.bfloat16())
    with pytest.raises(disco.DiscoError):
        blocks.residual_norm(x, f, post_weight=w["post_weight"])
    with pytest.raises(disco.DiscoError):
        blocks.residual_norm(x, f, gate=torch.ones(3, 48, device="cuda:0"))
    with pytest.raises(disco.DiscoError):
        blocks.residual_norm(x, f, want_h=False, want_y=False)
    with pytest.raises(disco.DiscoError):
        blocks.residual_norm(x, f, h=x, y=x)
    with pytest.raises(disco.DiscoError):
        blocks.residual_norm_backward(x, f, None, None)
    with pytest.raises(disco.DiscoError):
        blocks.residual_norm(torch.ones(1, 1, 8200, device="cuda:0"), torch.ones(1, 1, 8200, device="cuda:0"))
