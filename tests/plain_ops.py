"""Plain 64-bit forms of the operators around the attention, with what their tests need to derive tolerances: for every result the
sum of the magnitudes that go into it.  torch on the CPU, no part of the library."""
from math import sqrt

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative: the most that one rounding is off
U32 = 2.0 ** -24


# ---- norm and rotation ---------------------------------------------------------------------------
def row_order(shape):
    """Raster token of every row of a [B, H, L, d] tensor in the shape's order."""
    n = torch.arange(shape.L)
    if not shape.layout:
        return n
    w, h, t = n % shape.Ws, n // shape.Ws % shape.Hs, n // (shape.Ws * shape.Hs)
    block = (t // shape.Ct * (shape.Hs // shape.Ch) + h // shape.Ch) * (shape.Ws // shape.Cw) + w // shape.Cw
    inside = (t % shape.Ct * shape.Ch + h % shape.Ch) * shape.Cw + w % shape.Cw
    return torch.argsort(block * shape.Bk + inside)


def angles(shape, rope, theta, origin):
    """[L, pairs], raster order."""
    n = torch.arange(shape.L)
    coords = (n // (shape.Ws * shape.Hs), n // shape.Ws % shape.Hs, n % shape.Ws)
    parts = []
    for at, first, m in zip(coords, origin, (rope.dt, rope.dh, rope.dw)):
        freq = torch.tensor([theta ** (-2.0 * i / m) for i in range(m // 2)], dtype=torch.float64)
        parts.append((at + first).double()[:, None] * freq)
    return torch.cat(parts, 1)


def pairs_of(rope, d):
    """Index of the first and of the second channel of every pair, and the channels left."""
    n = rope.dt + rope.dh + rope.dw
    i = torch.arange(n // 2)
    return (i, i + n // 2, n) if rope.style else (2 * i, 2 * i + 1, n)


def turn(x, angle, rope, sign=1.0):
    """x [B, L, H, d]; returns the result and the sum of magnitudes of each."""
    a, b, _ = pairs_of(rope, x.shape[-1])
    c, s = angle.cos()[None, :, None], sign * angle.sin()[None, :, None]
    y, mag = x.clone(), x.abs()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    mag[..., a] = mag[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, mag


def norm_rope(shape, rope, X, w, eps, theta=10000.0, origin=(0, 0, 0), dY=None):
    """X [B, L, H, d] float64; returns {"Y": (value, bound of its error without the rounding of the result)} and with dY also "dX", "dw"."""
    d = shape.d
    order = row_order(shape)
    w = torch.ones(d, dtype=torch.float64) if w is None else w
    r = 1.0 / torch.sqrt((X * X).mean(-1, keepdim=True) + eps)
    xhat = X * r
    y, mag = xhat * w, None
    angle = None
    if rope is not None:
        angle = angles(shape, rope, theta, origin)
        y, mag = turn(y, angle, rope)
    else:
        mag = y.abs()
    # r: d products and sums of one sign (half of their relative error counts), its own two roundings; two products, the rotation's
    # three, cosine and sine once
    heads = lambda t: t[:, order].transpose(1, 2)  # noqa: E731
    out = {"Y": (heads(y), heads(mag) * (d / 2 + 10) * U32)}
    if dY is not None:
        g = torch.empty_like(X)
        g[:, order] = dY.transpose(1, 2)
        u, umag = turn(g, angle, rope, -1.0) if rope is not None else (g, g.abs())
        gw, gmag = u * w, umag * w.abs()
        t = (gw * xhat).mean(-1, keepdim=True)
        tmag = (gmag * xhat.abs()).mean(-1, keepdim=True)
        # as above, and the sum t over d products with errors of its own
        out["dX"] = (r * (gw - xhat * t), r * (gmag + xhat.abs() * tmag) * (2 * d + 30) * U32)
        # a lane's own sum, the workgroup's 64 slots at most, factors as above
        rows = X.shape[0] * X.shape[1]
        lanes = shape.H * (rows // 2048 + 1) + 64
        out["dw"] = ((u * xhat).sum((0, 1, 2)), (umag * xhat.abs()).sum((0, 1, 2)) * (lanes + d / 2 + 12) * U32)
    return out


# ---- cross attention -----------------------------------------------------------------------------
def valid_states(B, S, kv_len, kv_mask):
    ok = torch.ones((B, S), dtype=torch.bool)
    if kv_len is not None:
        ok &= torch.arange(S) < kv_len[:, None]
    if kv_mask is not None:
        ok &= kv_mask != 0
    return ok


def cross(Q, K, V, ok, scale, dO=None, half=U32, O_used=None):
    """Q [B, H, L, d], K, V [B, Hkv, S, d] float64, ok [B, S].  Returns {name: (value, bound)}; half: the rounding of the probabilities
    and of dS ahead of a product; O_used: the O that the backward is given."""
    B, H, L, d = Q.shape
    G, S = H // K.shape[1], K.shape[2]
    clean = lambda t: torch.where(ok[:, None, :, None], t, torch.zeros((), dtype=t.dtype)).repeat_interleave(G, 1)  # noqa: E731
    K, V = clean(K), clean(V)
    X = Q @ K.transpose(2, 3) * scale
    X = X.masked_fill(~ok[:, None, None], float("-inf"))
    some = ok.any(1)[:, None, None]
    m = torch.where(some[..., None], X.max(-1, keepdim=True).values, torch.zeros(1, 1, 1, 1, dtype=X.dtype))
    E = torch.exp(X - m)
    l = E.sum(-1)  # noqa: E741
    LSE = torch.where(some, m[..., 0] + torch.log(torch.where(some, l, torch.ones_like(l))), torch.full_like(l, float("-inf")))
    P = torch.where(some[..., None], E / torch.where(some, l, torch.ones_like(l))[..., None], torch.zeros_like(E))
    O = P @ V  # noqa: E741
    # a logit: d products, its scaling; a probability: two logits apart, exp2 and the base (a few steps of the exponent's argument),
    # the sum of S terms of one sign, the division
    es = (d + 4) * U32 * scale * (Q.abs() @ K.abs().transpose(2, 3)).masked_fill(~ok[:, None, None], 0.0).amax(-1, keepdim=True)
    top = torch.where(some[..., None], m.abs(), torch.zeros_like(m)) + es
    ep = 2 * es + (4 * top + S + 10) * U32
    out = {"O": (O, (ep + half + (S + 4) * U32) * (P @ V.abs())), "LSE": (LSE, (es + (4 * top + S + 10) * U32)[..., 0] + 2 * U32 * LSE.abs().nan_to_num(posinf=0))}
    if dO is None:
        return out
    dP = dO @ V.transpose(2, 3)
    dPm = dO.abs() @ V.abs().transpose(2, 3)
    delta = (dO * O).sum(-1, keepdim=True)
    ed = (dO.abs() * ((O_used - O).abs() if O_used is not None else half * O.abs())).sum(-1, keepdim=True)
    dm = (dO * O).abs().sum(-1, keepdim=True)
    dS = P * (dP - delta)
    # a logit's gradient: errors of the probability, of the two sums, of the O that delta was formed with; its rounding
    e = P * ((ep * (dP - delta).abs()) + (d + 4) * U32 * (dPm + dm) + ed) + half * dS.abs()
    group = lambda t: t.view(B, H // G, G, S, d).sum(2)  # noqa: E731
    n = G * L
    acc = lambda k: (k + 4) * U32  # noqa: E731  the product's own sums
    out["dQ"] = (scale * (dS @ K), scale * ((e + acc(S) * dS.abs()) @ K.abs()))
    out["dK"] = (group(scale * (dS.transpose(2, 3) @ Q)), group(scale * ((e + acc(n) * dS.abs()).transpose(2, 3) @ Q.abs())))
    out["dV"] = (group(P.transpose(2, 3) @ dO), group((P * (ep + half + acc(n))).transpose(2, 3) @ dO.abs()))
    return out


def default_scale(d):
    return 1.0 / sqrt(d)


def check(name, got, want, half):
    """Every element within its bound and the rounding of the result; infinities and NaN in the same places."""
    value, bound = want
    got = got.detach().double().cpu()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    fine = torch.isfinite(value)
    assert torch.equal(torch.isnan(got), torch.isnan(value)), f"{name}: NaN"
    assert torch.equal(got[~fine].nan_to_num(nan=0.0), value[~fine].nan_to_num(nan=0.0)), f"{name}: infinities"
    off, most = (got - value).abs()[fine], (bound + half * (value.abs() + bound))[fine]
    bad = off > most
    assert not bad.any(), f"{name}: {int(bad.sum())} of {off.numel()} off, worst {float((off / most.clamp_min(1e-300)).max()):.3g} times its bound"
    return float((off.square().sum() / value[fine].square().sum().clamp_min(1e-300)).sqrt()) if off.numel() else 0.0
