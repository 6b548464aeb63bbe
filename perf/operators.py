"""The attention between grids, and the clipping of gradients, that users of the
sphere layers run beside them, case by case.

An encoder of DISCO layers leaves states on a coarse grid (32 x 64 = 2048 tokens, 64 x 128
= 8192, 128 x 256 = 32768); a decoder grid, a set of latent tokens or one station reads them
by cross attention, after the queries and keys of each head were normed and rotated to
their positions, and a training step clips all gradients by their global norm.  A case
names one of these calls ("op"), its direction ("pass": "forward", or "step" for the
forward and its gradients), sizes, head layout and type; ``listed`` gives the working
sizes from single tokens to whole grids, ``draw`` more of the same ranges.

``run`` with ``own`` false is the plain form, in 32 bits; ``exact`` the definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


# --------------------------------------------------------------------------- #
# Cases
# --------------------------------------------------------------------------- #
def _rotate_case(name, direction, batch, tokens, heads, dim, rotary, layout="half", dtype="bf16", norm=True,
                 weight="shared", table="line", fused=1):
    """fused: x is one of this many equal parts of a joint projection (its rows lie apart)."""
    return {"name": name, "op": "rotate", "pass": direction, "batch": batch, "tokens": tokens, "heads": heads,
            "dim": dim, "rotary": rotary, "layout": layout, "dtype": dtype, "norm": norm, "weight": weight,
            "table": table, "fused": fused}


def _attend_case(name, direction, batch, queries, keys, heads, kv_heads, dim, dtype="bf16", bias="none",
                 lengths="full", empty=False):
    """bias: "area" for log quadrature weights, "holes" for the same with a tenth of the states missing;
    lengths: "ragged" for a batch of unequal numbers of states; empty: one item of the batch has none."""
    return {"name": name, "op": "attend", "pass": direction, "batch": batch, "queries": queries, "keys": keys,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "bias": bias, "lengths": lengths,
            "empty": empty}


def _clip_case(name, tensors, smallest, largest, mixed, clipped, sizes_seed):
    """`tensors` gradients of `smallest` to `largest` elements; mixed: every third in bf16;
    clipped: whether the norm is over the limit."""
    return {"name": name, "op": "clip", "tensors": tensors, "smallest": smallest, "largest": largest,
            "mixed": mixed, "clipped": clipped, "sizes_seed": sizes_seed}


def listed():
    return [
        # The queries of one new station for each of eight fields: launches and latency are all there is.
        _rotate_case("rotate_one_token", "forward", 8, 1, 16, 64, 64),
        # Keys of a 64 x 128 encoder grid out of a joint key-value projection, half of each head rotated.
        _rotate_case("rotate_keys_64x128", "forward", 4, 8192, 8, 64, 32, layout="interleaved", table="grid", fused=2),
        # Queries of a 128 x 256 decoder grid in a training step.
        _rotate_case("rotate_step_128x256", "step", 4, 32768, 8, 64, 64, table="grid"),
        # A two-degree grid in fp32: odd heads, a head size that is no power of two, a weight for each head.
        _rotate_case("rotate_step_90x180_fp32", "step", 3, 16200, 5, 36, 20, layout="interleaved", dtype="fp32",
                     weight="per_head", table="grid"),
        # One station's query against the states of a 32 x 64 encoder, grouped heads, unequal lengths.
        _attend_case("attend_one_token", "forward", 8, 1, 2048, 16, 4, 64, lengths="ragged"),
        # The same against a fine grid's states: 256 x 512 states, read once.
        _attend_case("attend_one_token_256x512", "forward", 4, 1, 131072, 16, 4, 128, bias="area"),
        # A decoder grid reading a coarser encoder grid, weighted by cell areas, inference.
        _attend_case("attend_128x256_to_64x128", "forward", 1, 32768, 8192, 8, 8, 64, bias="area"),
        # A wide level's training step: grouped heads of 128.
        _attend_case("attend_step_64x128_to_32x64", "step", 2, 8192, 2048, 16, 4, 128),
        # Training step of a whole grid reading a few latent states, lengths unequal.
        _attend_case("attend_step_few_states", "step", 2, 32768, 77, 8, 8, 64, lengths="ragged"),
        # fp32, ragged in everything: a four-degree grid, missing states, an item with no states at all.
        _attend_case("attend_step_45x90_fp32", "step", 3, 4050, 1013, 5, 5, 36, dtype="fp32", bias="holes",
                     lengths="ragged", empty=True),
        # The weights of a small network of DISCO layers, [Cout, Cin, 9] each.
        _clip_case("clip_small_network", 24, 4 * 4 * 9, 64 * 64 * 9, False, True, 1),
        # A large network's gradients, fp32 and bf16 beside each other.
        _clip_case("clip_large_network", 60, 1000, 40000000, True, True, 2),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# What the largest listed attention computes; a drawn one stays below.
MOST_SCORES = 8 * 32768 * 8192


def draw(rng):
    """Another case of the listed kinds, its sizes spread over their ranges."""
    kind = rng.choice(("rotate", "rotate", "token", "attend", "attend", "clip"))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    if kind == "rotate":
        dim = rng.choice((16, 32, 36, 64, 72, 96, 128))
        case = _rotate_case(None, rng.choice(("forward", "step")), rng.randint(1, 8), _log_uniform(rng, 1, 32768),
                            rng.randint(1, 16), dim, 2 * rng.randint(0, dim // 2),
                            layout=rng.choice(("half", "interleaved")), dtype=dtype, norm=rng.random() < 0.8,
                            weight=rng.choice(("shared", "per_head")), table=rng.choice(("line", "grid")),
                            fused=rng.randint(1, 3))
        while case["batch"] * case["tokens"] * case["heads"] * case["dim"] * case["fused"] > 4 * 32768 * 8 * 64:
            case["tokens"] = max(1, case["tokens"] // 2)
    elif kind == "token":
        kv = rng.choice((1, 2, 4, 8))
        case = _attend_case(None, "forward", rng.randint(1, 8), rng.choice((1, 1, 1, 2, 3, 5)),
                            _log_uniform(rng, 1, 131072), kv * rng.choice((1, 2, 4, 8)), kv,
                            rng.choice((32, 36, 64, 96, 128)), dtype=dtype, bias=rng.choice(("none", "area", "holes")),
                            lengths=rng.choice(("full", "ragged")))
        while case["batch"] * case["keys"] * kv * case["dim"] * (2 if dtype == "fp32" else 1) > 4 * 131072 * 4 * 128:
            case["keys"] //= 2
    elif kind == "attend":
        kv = rng.choice((1, 2, 3, 4, 8))
        case = _attend_case(None, rng.choice(("forward", "step")), rng.randint(1, 4), _log_uniform(rng, 16, 32768),
                            _log_uniform(rng, 1, 8192), kv * rng.choice((1, 2, 4)), kv,
                            rng.choice((16, 32, 36, 64, 80, 128)), dtype=dtype,
                            bias=rng.choice(("none", "area", "holes")), lengths=rng.choice(("full", "ragged")),
                            empty=rng.random() < 0.2)
        # A step is 3.5 forward passes, a product in fp32 some eight in bf16.
        weight = (4 if case["pass"] == "step" else 1) * (8 if dtype == "fp32" else 1) * max(1.0, case["dim"] / 64.0)
        while weight * case["batch"] * case["heads"] * case["queries"] * case["keys"] > MOST_SCORES:
            big = "queries" if case["queries"] > case["keys"] else "keys"
            case[big] = max(1, case[big] // 2)
    else:
        largest = _log_uniform(rng, 1000, 40000000)
        case = _clip_case(None, _log_uniform(rng, 1, 60), max(1, largest // rng.choice((1, 10, 1000))), largest,
                          rng.random() < 0.5, rng.random() < 0.8, rng.randint(0, 1 << 20))
        while sum(_clip_sizes(case)) > 300000000:
            case["tensors"] //= 2
    del case["name"]
    return case


def _lengths(case):
    """States of each batch item: unequal ones fall to half along the batch."""
    B, n = case["batch"], case["keys"]
    out = [n - (b * n) // (2 * B) for b in range(B)] if case["lengths"] == "ragged" else [n] * B
    if case["empty"]:
        out[-1] = 0
    return out


def _clip_sizes(case):
    rng = random.Random(case["sizes_seed"])
    return [_log_uniform(rng, case["smallest"], case["largest"]) for _ in range(case["tensors"])]


def _clip_types(case):
    return ["bf16" if case["mixed"] and i % 3 == 2 else "fp32" for i in range(case["tensors"])]


def work(case):
    size = {"bf16": 2, "fp32": 4}
    if case["op"] == "rotate":
        n = case["batch"] * case["tokens"] * case["heads"] * case["dim"]
        table = 4 * case["rotary"] * min(case["tokens"] * case["batch"], _table_rows(case))
        step = case["pass"] == "step"  # forward: x in, y out; gradients: x once for both, dy in, dx out
        return {"bytes": n * size[case["dtype"]] * (4 if step else 2) + table, "flops": n * (22 if step else 7)}
    if case["op"] == "attend":
        lengths, B, D, e = _lengths(case), case["batch"], case["dim"], size[case["dtype"]]
        q = B * case["queries"] * case["heads"] * D
        kv = 2 * sum(lengths) * case["kv_heads"] * D
        pairs = case["queries"] * case["heads"] * sum(lengths)
        bias = 4 * sum(lengths) if case["bias"] != "none" else 0
        if case["pass"] == "step":  # q, dout in, out, dq out; k, v in, dk, dv out
            return {"bytes": (4 * q + 2 * kv) * e + bias, "flops": 14 * pairs * D}
        return {"bytes": (2 * q + kv) * e + bias, "flops": 4 * pairs * D}
    total = sum(n * size[t] for n, t in zip(_clip_sizes(case), _clip_types(case)))
    return {"bytes": 2 * total, "flops": 3 * sum(_clip_sizes(case))}


# --------------------------------------------------------------------------- #
# What a program has in hand
# --------------------------------------------------------------------------- #
def _table_rows(case):
    return case["tokens"] if case["table"] == "grid" else max(4096, 2 * case["tokens"])


def _table(case):
    """Rotation angles of every position, as cos and sin.  "line": position times a falling
    frequency, stretched fourfold for contexts longer than those trained on; "grid": the
    longitude times whole numbers (the rotation closes around the sphere), then the colatitude."""
    rows, half = _table_rows(case), case["rotary"] // 2
    i = torch.arange(half, dtype=torch.float64)
    p = torch.arange(rows, dtype=torch.float64)[:, None]
    if case["table"] == "line":
        angle = (p / 4.0) * 10000.0 ** (-i / max(1, half))
    else:
        nlat = max(1, int(math.isqrt(max(1, rows // 2))))
        nlon = -(-rows // nlat)
        lon, colat = 2 * math.pi * (p % nlon) / nlon, math.pi * (p // nlon + 0.5) / nlat
        angle = torch.where(i < half / 2, lon * (i + 1), colat * (i + 1))
    return angle.cos().float().to(DEVICE), angle.sin().float().to(DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = TYPES[case.get("dtype", "fp32")]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE)

    state = {"case": case}
    if case["op"] == "rotate":
        B, S, H, D = case["batch"], case["tokens"], case["heads"], case["dim"]
        joint = (1.5 * normal(B, S, case["fused"], H, D)).to(dt)
        state["x"] = joint[:, :, case["fused"] - 1]
        shape = (H, D) if case["weight"] == "per_head" else (D,)
        state["weight"] = (1.0 + 0.2 * normal(*shape)).to(dt) if case["norm"] else None
        state["cos"], state["sin"] = _table(case)
        if case["table"] == "line":
            state["positions"] = torch.randint(0, _table_rows(case), (B, S), generator=g, device=DEVICE,
                                               dtype=torch.int32)
        else:
            state["positions"] = None  # token s stands on row s
        if case["pass"] == "step":
            state["dy"] = normal(B, S, H, D).to(dt)
    elif case["op"] == "attend":
        B, Sq, Sk, H, Hk, D = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "dim"))
        # Normed queries and keys: a score has a spread of about 1.5.
        state["q"] = (1.5 * normal(B, Sq, H, D)).to(dt)
        joint = normal(B, Sk, 2, Hk, D).to(dt)  # one projection gives keys and values
        state["k"], state["v"] = joint[:, :, 0], joint[:, :, 1]
        state["key_bias"] = state["key_lengths"] = None
        if case["bias"] != "none":
            area = torch.rand((B, Sk), generator=g, device=DEVICE) + 0.05
            state["key_bias"] = (area / area.sum(1, keepdim=True)).log()
            if case["bias"] == "holes":
                gone = torch.rand((B, Sk), generator=g, device=DEVICE) < 0.1
                state["key_bias"] = state["key_bias"].masked_fill(gone, -math.inf)
        if case["lengths"] == "ragged" or case["empty"]:
            state["key_lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEVICE)
        if case["pass"] == "step":
            state["dout"] = normal(B, Sq, H, D).to(dt)
    else:
        sizes, types = _clip_sizes(case), _clip_types(case)
        state["grads"] = [(1e-2 * normal(n)).to(TYPES[t]) for n, t in zip(sizes, types)]
        state["max_norm"] = 1e-2 * math.sqrt(sum(sizes)) * (0.3 if case["clipped"] else 3.0)
        state["out"] = [torch.empty_like(t) for t in state["grads"]]
    return state


# --------------------------------------------------------------------------- #
# The plain form, in 32 bits
# --------------------------------------------------------------------------- #
def _angles(state):
    cos, sin = state["cos"], state["sin"]
    if state["positions"] is not None:
        p = state["positions"].long()
        return cos[p][:, :, None], sin[p][:, :, None]  # [B, S, 1, R/2]
    return cos[None, :, None], sin[None, :, None]


def _rotate(u, cos, sin, rotary, layout):
    head, rest = u[..., :rotary], u[..., rotary:]
    if layout == "half":
        a, b = head[..., :rotary // 2], head[..., rotary // 2:]
        return torch.cat((a * cos - b * sin, a * sin + b * cos, rest), -1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2), rest), -1)


def _plain_rotate(state):
    case = state["case"]
    x = state["x"].float()
    cos, sin = _angles(state)
    if case["norm"]:
        w = state["weight"].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * r
        y = _rotate(n * w, cos, sin, case["rotary"], case["layout"])
    else:
        y = _rotate(x, cos, sin, case["rotary"], case["layout"])
    y = y.to(state["x"].dtype)
    if case["pass"] == "forward":
        return [y]
    g = _rotate(state["dy"].float(), cos, -sin, case["rotary"], case["layout"])
    if not case["norm"]:
        return [y, g.to(y.dtype)]
    dw = (g * n).sum((0, 1) if case["weight"] == "per_head" else (0, 1, 2))
    t = g * w
    dx = r * (t - n * (t * n).mean(-1, keepdim=True))
    return [y, dx.to(y.dtype), dw.to(y.dtype)]


def _plain_attend(state):
    case = state["case"]
    dt = state["q"].dtype
    B, Sq, Sk, H, Hk, D = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "dim"))
    G, scale = H // Hk, 1.0 / math.sqrt(D)
    # [B, Hk, G Sq, D] against [B, Hk, Sk, D]
    q = state["q"].float().reshape(B, Sq, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * Sq, D)
    k = state["k"].float().permute(0, 2, 1, 3).contiguous()
    v = state["v"].float().permute(0, 2, 1, 3).contiguous()
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    keep = None
    if state["key_lengths"] is not None:
        keep = torch.arange(Sk, device=DEVICE)[None] < state["key_lengths"][:, None]
    if state["key_bias"] is not None:
        s = s + state["key_bias"][:, None, None]
    if keep is not None:
        s = s.masked_fill(~keep[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    del s
    o = torch.matmul(p, v)

    def back(t, heads, rows):
        return t.reshape(B, Hk, heads // Hk, rows, D).permute(0, 3, 1, 2, 4).reshape(B, rows, heads, D).to(dt)

    out = back(o, H, Sq)
    if case["pass"] == "forward":
        return [out]
    do = state["dout"].float().reshape(B, Sq, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * Sq, D)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (ds - (do * o).sum(-1, keepdim=True)) * scale
    del p
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    return [out, back(dq, H, Sq), back(dk, Hk, Sk), back(dv, Hk, Sk)]


def _plain_clip(state):
    norm = torch.stack([t.float().square().sum() for t in state["grads"]]).sum().sqrt()
    c = torch.clamp(state["max_norm"] / (norm + EPS), max=1.0)
    return [norm] + [(t.float() * c).to(t.dtype) for t in state["grads"]]


# --------------------------------------------------------------------------- #
# One pass
# --------------------------------------------------------------------------- #
def run(state):
    case = state["case"]
    if not own:
        return {"rotate": _plain_rotate, "attend": _plain_attend, "clip": _plain_clip}[case["op"]](state)
    from paper_2209_13603_amd import attention, gradients
    if case["op"] == "rotate":
        how = {"rotation": (state["cos"], state["sin"]), "layout": case["layout"], "positions": state["positions"],
               "norm": case["norm"], "eps": EPS}
        y = attention.norm_rotate(state["x"], state["weight"], **how)
        if case["pass"] == "forward":
            return [y]
        dx, dw = attention.norm_rotate_backward(state["x"], state["weight"], state["dy"], **how)
        return [y, dx] if dw is None else [y, dx, dw]
    if case["op"] == "attend":
        how = {"key_bias": state["key_bias"], "key_lengths": state["key_lengths"]}
        q, k, v = state["q"], state["k"], state["v"]
        if case["pass"] == "forward":
            return [attention.cross_attention(q, k, v, **how)]
        out, stats = attention.cross_attention(q, k, v, return_stats=True, **how)
        return [out, *attention.cross_attention_backward(q, k, v, out, stats, state["dout"], **how)]
    norm, out = gradients.clip(state["grads"], state["max_norm"], eps=EPS, out=state["out"])
    return [norm, *out]


# --------------------------------------------------------------------------- #
# The definition in 64 bits
# --------------------------------------------------------------------------- #
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "rotate":
        return _exact_rotate(case, state)
    if case["op"] == "attend":
        return _exact_attend(case, state)
    total = sum(float(torch.dot(t.double(), t.double())) for t in state["grads"])
    norm = math.sqrt(total)
    factor = min(1.0, state["max_norm"] / (norm + EPS))
    return [torch.tensor(norm, dtype=torch.float64, device=DEVICE)] + [t.double() * factor for t in state["grads"]]


def _exact_rotate(case, state):
    """Pairs as complex numbers, gradients by automatic differentiation."""
    R = case["rotary"]
    x = state["x"].double().requires_grad_(True)
    turn = torch.complex(state["cos"].double(), state["sin"].double())
    if state["positions"] is not None:
        turn = turn[state["positions"].long()]
    else:
        turn = turn[None].expand(case["batch"], -1, -1)
    w = state["weight"].double().requires_grad_(True) if case["norm"] else None
    u = x
    if case["norm"]:
        u = x / (x.pow(2).sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * w
    if R:
        pairs = u[..., :R]
        pairs = pairs.unflatten(-1, (2, R // 2)).transpose(-1, -2) if case["layout"] == "half" \
            else pairs.unflatten(-1, (R // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, :, None])
        z = z.transpose(-1, -2) if case["layout"] == "half" else z
        u = torch.cat((z.flatten(-2), u[..., R:]), -1)
    if case["pass"] == "forward":
        return [u.detach()]
    wrt = [x] if w is None else [x, w]
    return [u.detach(), *torch.autograd.grad(u, wrt, state["dy"].double())]


def _exact_attend(case, state):
    """One head of one item at a time, on the states that the mask leaves."""
    B, Sq, Sk, H, Hk, D = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads", "dim"))
    step = case["pass"] == "step"
    shape_q, shape_k = (B, Sq, H, D), (B, Sk, Hk, D)
    out = torch.zeros(shape_q, dtype=torch.float64, device=DEVICE)
    dq, dk, dv = (torch.zeros(s if step else (0,), dtype=torch.float64, device=DEVICE)
                  for s in (shape_q, shape_k, shape_k))
    for b, n in enumerate(_lengths(case)):
        keep = torch.arange(n, device=DEVICE)
        if state["key_bias"] is not None:
            keep = keep[torch.isfinite(state["key_bias"][b, :n])]
        if keep.numel() == 0:
            continue
        for h in range(H):
            hk = h // (H // Hk)
            q = state["q"][b, :, h].double()
            k, v = state["k"][b, keep, hk].double(), state["v"][b, keep, hk].double()
            logits = (q @ k.t()) / math.sqrt(D)
            if state["key_bias"] is not None:
                logits = logits + state["key_bias"][b, keep].double()
            p = torch.softmax(logits, dim=1)
            del logits
            out[b, :, h] = p @ v
            if not step:
                continue
            do = state["dout"][b, :, h].double()
            dv[b, keep, hk] += p.t() @ do
            dp = do @ v.t()
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            dq[b, :, h] = (ds @ k) / math.sqrt(D)
            dk[b, keep, hk] += (ds.t() @ q) / math.sqrt(D)
    return [out, dq, dk, dv] if step else [out]
