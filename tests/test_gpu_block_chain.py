"""The block operators together, as a layer runs them, captured into graphs, on other streams and in large buffers."""
import pytest

from block_forms import dropout_factor, recurrence as recur_form, rel

pytestmark = pytest.mark.gpu


def _layer_inputs(B, T, C, dtype, seed=0):
    import torch
    r = torch.Generator(device="cuda:0").manual_seed(seed + B + 3 * T + 7 * C)
    rnd = lambda *s: torch.randn(s, generator=r, device="cuda:0").to(dtype)
    w = {k: (1 + 0.2 * rnd(C).float()).to(dtype) for k in ("in_norm", "post", "gate", "next")}
    return rnd(B, T, C), rnd(B, T, C), rnd(B, T, C), rnd(B, T, C), w


def _layer(x, g, dh, dy, w, drop, state=None):
    """Norm, recurrence, residual sum with dropout and the next norm, and all gradients."""
    from paper_2209_13603_amd import blocks, recurrence
    _, u = blocks.residual_norm(None, x, next_weight=w["in_norm"], want_h=False)
    f, last, carries = recurrence.gated_recurrence(u, g, state=state, return_carries=True)
    how = dict(post_norm=True, post_weight=w["post"], gate=w["gate"], next_weight=w["next"], dropout=drop)
    h, y = blocks.residual_norm(x, f, **how)
    top = blocks.residual_norm_backward(x, f, dh, dy, **how)
    mid = recurrence.gated_recurrence_backward(u, g, carries, top.df)
    low = blocks.residual_norm_backward(None, x, None, mid.dx, next_weight=w["in_norm"])
    return [h, y, last, top.dx + low.df, mid.dgate, low.dnext_weight, top.dpost_weight, top.dgate, top.dnext_weight]


@pytest.mark.parametrize("shape", [(2, 30, 24), (1, 700, 66), (3, 17, 7)])
def test_a_layer_against_the_definition(shape):
    """fp32.  A dozen roundings of 2^-24 an entry through three operators, sums of some thousand rows: 1e-5."""
    import torch
    from paper_2209_13603_amd import blocks
    x, g, dh, dy, w = _layer_inputs(*shape, torch.float32)
    drop = blocks.Dropout(0.2, 5, 3)
    got = _layer(x, g, dh, dy, w, drop)
    leaf = {k: v.cpu().double().requires_grad_(True) for k, v in dict(x=x, g=g, **w).items()}
    rms = lambda v: v / (v.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
    u = rms(leaf["x"]) * leaf["in_norm"]
    a = torch.sigmoid(leaf["g"])
    s, steps = torch.zeros_like(u[:, 0]), []
    for t in range(shape[1]):
        s = a[:, t] * s + (1 - a[:, t]) * u[:, t]
        steps.append(s)
    f = torch.stack(steps, 1)
    h = leaf["x"] + leaf["gate"] * (rms(f) * leaf["post"] * dropout_factor(shape, drop))
    y = rms(h) * leaf["next"]
    total = (h * dh.cpu().double()).sum() + (y * dy.cpu().double()).sum()
    grads = torch.autograd.grad(total, [leaf[k] for k in ("x", "g", "in_norm", "post", "gate", "next")])
    for i, (u, v) in enumerate(zip(got, [h.detach(), y.detach(), s.detach(), *grads])):
        assert rel(u, v) <= 1e-5, i


@pytest.mark.parametrize("shape", [(2, 30, 24), (2, 1500, 64)])
def test_a_layer_replayed_from_a_graph(shape):
    """Every replay against the eager call, with new inputs, another dropout offset and eager work in between."""
    import torch
    from paper_2209_13603_amd import blocks
    x, g, dh, dy, w = _layer_inputs(*shape, torch.bfloat16)
    counter = torch.zeros(1, dtype=torch.int64, device="cuda:0")
    drop = blocks.Dropout(0.2, 5, 7, counter)
    _layer(x, g, dh, dy, w, drop)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _layer(x, g, dh, dy, w, drop)
        counter.add_(1)
    counter.zero_()
    for i in range(4):
        x.copy_(torch.roll(x, 1, 1))
        g.add_(0.125)
        graph.replay()
        torch.cuda.synchronize()
        want = _layer(x, g, dh, dy, w, blocks.Dropout(0.2, 5, 7 + i))
        for u, v in zip(out, want):
            assert bool((u == v).all())


def test_two_graphs_of_one_memory_pool():
    """Scratch memory that both graphs take from the same pool is free again before the next call uses it."""
    import torch
    from paper_2209_13603_amd import blocks
    a = _layer_inputs(1, 1500, 64, torch.bfloat16, seed=1)
    b = _layer_inputs(1, 1500, 64, torch.bfloat16, seed=2)
    drop = blocks.Dropout(0.1, 3)
    want = [[t.clone() for t in _layer(*i, drop)] for i in (a, b)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0].pool() if graphs else None):
            outs.append(_layer(*i, drop))
        graphs.append(graph)
    for _ in range(3):
        for k in (0, 1):
            graphs[k].replay()
            torch.cuda.synchronize()
            for u, v in zip(outs[k], want[k]):
                assert bool((u == v).all())


def test_other_streams():
    """stream= runs there, and two streams at once give what one does."""
    import torch
    from paper_2209_13603_amd import blocks, recurrence
    x, g, dh, dy, w = _layer_inputs(2, 1300, 64, torch.bfloat16)
    how = dict(post_norm=True, post_weight=w["post"], gate=w["gate"], next_weight=w["next"], dropout=blocks.Dropout(0.3, 1))
    want = blocks.residual_norm(x, g, **how), recurrence.gated_recurrence(x, g), blocks.dropout(x, blocks.Dropout(0.3, 2)), \
        blocks.residual_norm_backward(x, g, dh, dy, **how)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s in streams:
            got.append((blocks.residual_norm(x, g, stream=s, **how), recurrence.gated_recurrence(x, g, stream=s),
                        blocks.dropout(x, blocks.Dropout(0.3, 2), stream=s),
                        blocks.residual_norm_backward(x, g, dh, dy, stream=s, **how)))
        torch.cuda.synchronize()
        for one in got:
            for u, v in zip(one, want):
                for p, q in zip(u if isinstance(u, tuple) else (u,), v if isinstance(v, tuple) else (v,)):
                    assert bool((p == q).all())
    with torch.cuda.stream(streams[0]):
        again = _layer(x, g, dh, dy, w, None)
    torch.cuda.synchronize()
    for u, v in zip(again, _layer(x, g, dh, dy, w, None)):
        assert bool((u == v).all())


@pytest.mark.parametrize("strides", [(1 << 31, 64), (1 << 31, 1 << 25), (64, 1 << 26)])
def test_offsets_beyond_32_bits(strides):
    """Parts of buffers of more than 2^31 elements, and steps too far apart for offsets within a tile."""
    import torch
    from paper_2209_13603_amd import blocks, recurrence
    B, T, C = 2, 40, 64
    n = (B - 1) * strides[0] + (T - 1) * strides[1] + C
    if strides[1] > strides[0]:
        n = max(n, strides[1] * (T - 1) + B * C)
    big = torch.empty(n, dtype=torch.bfloat16, device="cuda:0")
    place = big.as_strided((B, T, C), (*strides, 1))
    x, g, dh, dy, w = _layer_inputs(B, T, C, torch.bfloat16)
    how = dict(post_norm=True, post_weight=w["post"], gate=w["gate"], next_weight=w["next"])
    want = blocks.residual_norm(x, g, **how)
    place.copy_(x)
    got = blocks.residual_norm(place, g, **how)
    assert all(bool((u == v).all()) for u, v in zip(got, want))
    blocks.residual_norm(x, g, h=place, **how)
    assert bool((place == want[0]).all())
    place.copy_(x)
    assert bool((blocks.dropout(place, blocks.Dropout(0.5, 1)) == blocks.dropout(x, blocks.Dropout(0.5, 1))).all())
    # (steps too far apart walk alone, whose sums of a run differ by their roundings)
    y, last, carries = recurrence.gated_recurrence(x, g, return_carries=True)
    y2, last2, carries2 = recurrence.gated_recurrence(place, g, return_carries=True)
    assert rel(y2, y.double().cpu()) <= 2.0 ** -8 + 3e-6 and rel(last2, last.double().cpu()) <= 3e-6
    grads = recurrence.gated_recurrence_backward(x, g, carries, dy)
    place.copy_(x)
    grads2 = recurrence.gated_recurrence_backward(place, g, carries2, dy, dx=place)
    assert rel(grads2.dx, grads.dx.double().cpu()) <= 2.0 ** -8 + 6e-6
    assert rel(grads2.dgate, grads.dgate.double().cpu()) <= 2.0 ** -8 + 6e-6


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("channels", [5, 8, 34, 64])
def test_what_lies_between_the_rows_is_left_as_it_was(channels, dtype):
    """Outputs into parts of joint buffers: the other parts keep what they hold."""
    import torch
    from paper_2209_13603_amd import blocks, recurrence
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    for T in (3, 50):
        x, g, dh, dy, w = _layer_inputs(3, T, channels, dt)

        def hole():
            j = torch.full((3, T + 1, 3, channels), 7.0, dtype=dt, device="cuda:0")
            return j, j[:, :T, 1]

        def kept(j):
            return bool((j[:, T] == 7).all()) and bool((j[:, :, 0] == 7).all()) and bool((j[:, :, 2] == 7).all())

        (jh, h), (jy, y), (jx, dx), (jf, df), (jr, r), (jg, dg) = (hole() for _ in range(6))
        how = dict(post_norm=True, post_weight=w["post"], gate=w["gate"], next_weight=w["next"])
        blocks.residual_norm(x, g, h=h, y=y, **how)
        blocks.residual_norm_backward(x, g, dh, dy, dx=dx, df=df, **how)
        _, _, carries = recurrence.gated_recurrence(x, g, y=r, return_carries=True)
        for j in (jh, jy, jx, jf, jr):
            assert kept(j)
        recurrence.gated_recurrence_backward(x, g, carries, dy, dx=r, dgate=dg)
        blocks.dropout(x, blocks.Dropout(0.5, 1), y=h)
        assert kept(jr) and kept(jg) and kept(jh)


def test_workspaces_of_the_library():
    """The C entries with no workspace given take one of the stream-ordered pool, and refuse one that is too small or not
    aligned before anything is written."""
    import ctypes
    import torch
    from paper_2209_13603_amd import blocks, disco, recurrence
    lib = disco.library()
    x, g, dh, dy, w = _layer_inputs(1, 900, 64, torch.float32)
    stream = torch.cuda.current_stream().cuda_stream
    want_y, _ = recurrence.gated_recurrence(x, g)
    want = blocks.residual_norm_backward(x, g, dh, dy, gate=w["gate"])
    y, dx, df, dw = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(w["gate"])
    p = blocks._Pack()
    rx, rg, ry = p.rows(x, "x"), p.rows(g, "g"), p.rows(y, "y")
    opt = p.residual(x, False, None, w["gate"], None, 1.0, 1e-6, None)
    grads = [p.rows(t, "t") for t in (dh, dy, dx, df)] + [None, p.weight(dw, "dw"), None]
    need = ctypes.c_size_t()
    assert lib.disco_gated_recurrence_workspace(rx, need) == 0 and need.value > 256
    assert lib.disco_gated_recurrence(rx, rg, None, None, None, ry, None, None, None, 0, stream) == 0
    assert lib.disco_residual_norm_backward(rx, rg, opt, *grads, None, 0, stream) == 0
    torch.cuda.synchronize()
    assert bool((y == want_y).all()) and bool((dx == want.dx).all()) and bool((dw == want.dgate).all())
    small = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0")
    for t in (y, dx, dw):
        t.fill_(7.0)
    for at, n in ((small.data_ptr(), 256), (small.data_ptr() + 8, 1 << 19)):
        assert lib.disco_gated_recurrence(rx, rg, None, None, None, ry, None, None, at, n, stream) == \
            disco.DISCO_ERR_INVALID_ARGUMENT
        assert lib.disco_residual_norm_backward(rx, rg, opt, *grads, at, n, stream) == disco.DISCO_ERR_INVALID_ARGUMENT
    torch.cuda.synchronize()
    assert bool((y == 7).all()) and bool((dx == 7).all()) and bool((dw == 7).all())
