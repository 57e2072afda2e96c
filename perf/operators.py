"""The operators around the sparse self-attention of a video transformer's block, as measurable cases.

    op "rope"    norm of every head's queries and keys with the rotation by grid position in the same pass,
                 from the projection's output [B, L, H, d] to the [B, H, L, d] tensors that attention takes
    op "cross"   attention of the grid's tokens to an encoder's states

Fields of a case (all): mode ("infer": forward alone, "train": forward and backward), dtype, B, H, d.

    rope   T, Hs, Ws (token grid), Ct, Ch, Cw (block), block_major (token order of the results), dt, dh, dw (channels
           rotated by each coordinate), halves (pairs are (i, i + n/2), else (2i, 2i + 1)), packed (queries, keys and
           values are slices of one projection; else queries and keys stand alone, without values), t0 (time
           coordinate of the first frame)
    cross  Hkv (key/value heads), Lq (queries), S (encoder states), lens ("full", "ragged": a valid length for every
           batch entry, "empty": ragged, the last entry without a valid state), mask (a byte for every state),
           token_major (tensors [B, L, H, d] seen as [B, H, L, d])

States that are not valid hold NaN, as memory that nobody wrote may.
"""
from math import log, sqrt

import torch

own = False

EPS, THETA = 1e-6, 10000.0
DEVICE = "cuda:0"


def _rope(name, mode, grid, **kw):
    c = dict(op="rope", mode=mode, dtype="bf16", B=1, H=12, d=128, T=grid[0], Hs=grid[1], Ws=grid[2], Ct=4, Ch=4, Cw=4,
             block_major=False, dt=44, dh=42, dw=42, halves=False, packed=True, t0=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _cross(name, mode, Lq, S, **kw):
    c = dict(op="cross", mode=mode, dtype="bf16", B=1, H=12, Hkv=0, d=128, Lq=Lq, S=S, lens="full", mask=False, token_major=False)
    c.update(kw)
    c["Hkv"] = c["Hkv"] or c["H"]
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest layer, 256 tokens in fp32: launches and host work are what it costs
        _rope("rope_tiny_fp32_train", "train", (4, 8, 8), H=2, d=64, Ct=2, dt=24, dh=20, dw=20, dtype="fp32"),
        # one token of each of eight sequences far along, one axis, keys and queries of separate projections
        _rope("rope_token_infer", "infer", (1, 1, 1), B=8, H=16, Ct=1, Ch=1, Cw=1, dt=128, dh=0, dw=0, halves=True, packed=False, t0=100003),
        # a grid that 4x4x4 blocks do not divide, a head dimension that is no power of two, channels left unrotated
        _rope("rope_odd_grid_train", "train", (21, 30, 52), B=2, H=4, d=72, Ct=3, Ch=5, dt=24, dh=20, dw=20, halves=True),
        # the benchmark layer, 33,280 tokens, training
        _rope("rope_layer33k_train", "train", (20, 32, 52)),
        # a 720p layer at inference, tokens of a block adjacent: 70,400 tokens, 40 heads
        _rope("rope_hd720p_infer", "infer", (20, 44, 80), H=40, block_major=True),
        # one new token of each of four sequences to a short encoder: latency
        _cross("cross_token_infer", "infer", 1, 300, B=4, lens="ragged"),
        # one new token, shared key/value heads, long encoder states of any length: the memory's rate
        _cross("cross_token_long_infer", "infer", 1, 20000, B=8, H=32, Hkv=8, lens="ragged", token_major=True),
        # the smallest layer in fp32, with a masked encoder
        _cross("cross_tiny_fp32_train", "train", 256, 77, H=2, d=64, dtype="fp32", mask=True),
        # a layer checked in fp32, two prompts, one of them empty (unconditional)
        _cross("cross_check_fp32_train", "train", 2520, 333, B=2, lens="empty", dtype="fp32"),
        # an odd head dimension and length, shared heads, batch 3, ragged: training
        _cross("cross_odd_train", "train", 1911, 257, B=3, H=6, Hkv=2, d=72, lens="ragged", mask=True, token_major=True),
        # the benchmark layer's 33,280 tokens to a text encoder's 512 states, training
        _cross("cross_layer33k_train", "train", 33280, 512, lens="ragged"),
        # a 720p layer's 70,400 tokens and 40 heads at inference
        _cross("cross_hd720p_infer", "infer", 70400, 512, H=40),
    ]


def draw(rng):
    over = lambda a, b: int(round(a * (b / a) ** rng.random()))  # noqa: E731
    while True:
        mode = "train" if rng.random() < 0.5 else "infer"
        dtype = "fp32" if rng.random() < 0.25 else "bf16"
        if rng.random() < 0.4:
            ct, ch, cw = rng.choice(((4, 4, 4), (4, 4, 4), (3, 5, 4), (2, 4, 4), (1, 1, 1), (1, 2, 3)))
            n = over(1, 70400) / (ct * ch * cw)
            nt = max(1, round(n ** (1 / 3) * rng.uniform(0.5, 1.0)))
            nh = max(1, round((n / nt) ** 0.5 * rng.uniform(0.75, 1.0)))
            nw = max(1, round(n / (nt * nh)))
            d = rng.choice((32, 64, 72, 80, 96, 128, 128, 128, 160, 256))
            dh = dw = 2 * rng.randint(0, d // 6)
            dt = 2 * rng.randint(0, (d - dh - dw) // 2)
            dt -= (dt + dh + dw) % 8
            if dt < 0:
                continue
            c = _rope("", mode, (nt * ct, nh * ch, nw * cw), B=rng.choice((1, 1, 2, 3)), H=rng.choice((1, 3, 4, 8, 12, 16, 40)), d=d,
                      dtype=dtype, Ct=ct, Ch=ch, Cw=cw, dt=dt, dh=dh, dw=dw, block_major=rng.random() < 0.5, halves=rng.random() < 0.5,
                      packed=rng.random() < 0.7, t0=rng.choice((0, 0, rng.randint(1, 200000))))
        else:
            h = rng.choice((1, 3, 6, 8, 12, 16, 24, 40))
            lq = 1 if rng.random() < 0.2 else over(1, 70400)
            s = over(8 if mode == "train" else 2, 32000)
            c = _cross("", mode, lq, s, dtype=dtype, B=rng.choice((1, 1, 2, 3, 8)), H=h, Hkv=h // rng.choice([g for g in (1, 1, 1, 2, 3, 4, 8) if h % g == 0]),
                       d=rng.choice((32, 64, 64, 72, 80, 96, 128, 128, 128, 160, 256)), lens=rng.choice(("full", "full", "ragged", "empty")),
                       mask=rng.random() < 0.25, token_major=rng.random() < 0.5)
            if c["B"] == 1 and c["lens"] == "empty" or c["B"] * h * lq * s > 1.4e9:
                continue
        w = work(c)
        if w["bytes"] <= 2.5e9 and w["flops"] <= (7e11 if dtype == "bf16" else 7e10):
            return c


def work(c):
    es = 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "rope":
        rows = c["B"] * c["T"] * c["Hs"] * c["Ws"] * c["H"]
        n = rows * c["d"]
        qk, v = 2 * n, n if c["packed"] else 0
        table = 4 * (c["T"] * c["dt"] + c["Hs"] * c["dh"] + c["Ws"] * c["dw"])
        by, flops = es * (2 * qk + 2 * v) + table, 7 * qk  # forward: square, sum, scale, weight, rotate
        if c["mode"] == "train":
            by, flops = by + es * (3 * qk + 2 * v) + table, flops + 17 * qk
        return {"bytes": by + 4 * 4 * c["d"], "flops": flops}
    q, kv = c["B"] * c["H"] * c["Lq"] * c["d"], c["B"] * c["Hkv"] * c["S"] * c["d"]
    valid = {"full": 1.0, "ragged": 0.6, "empty": 0.6 * (c["B"] - 1) / c["B"]}[c["lens"]] * (0.8 if c["mask"] else 1.0)  # in the mean
    lse = 4 * c["B"] * c["H"] * c["Lq"]
    by, flops = es * (2 * q + 2 * kv * valid) + lse, 4 * q * c["S"] * valid
    if c["mode"] == "train":
        by, flops = by + es * (4 * q + 2 * kv * valid + 2 * kv) + lse, flops * 3.5
    return {"bytes": by, "flops": flops}


# ---- what a user's program has in hand -----------------------------------------------------------
def _dtype(c):
    return torch.float32 if c["dtype"] == "fp32" else torch.bfloat16


def _normal(gen, shape, dtype, gain=1.0):
    return (torch.randn(shape, generator=gen, device=DEVICE) * gain).to(dtype)


def _table(c):
    """cos and sin of position * THETA^(-2i/n) for the n channels of every axis, axis after axis: [extent][n/2][2]."""
    parts = []
    for extent, first, n in ((c["T"], c["t0"], c["dt"]), (c["Hs"], 0, c["dh"]), (c["Ws"], 0, c["dw"])):
        if n:
            pos = torch.arange(extent, dtype=torch.float64, device=DEVICE) + first
            angle = pos[:, None] * torch.exp(torch.arange(n // 2, dtype=torch.float64, device=DEVICE) * (-2 * log(THETA) / n))
            parts.append(torch.stack((angle.cos(), angle.sin()), -1).reshape(-1))
    return torch.cat(parts).float() if parts else torch.zeros(0, device=DEVICE)


def _inputs(c, seed):
    gen = torch.Generator(DEVICE)
    gen.manual_seed(seed)
    dt = _dtype(c)
    s = dict(c=c)
    if c["op"] == "rope":
        L = c["T"] * c["Hs"] * c["Ws"]
        if c["packed"]:
            X = _normal(gen, (c["B"], L, 3, c["H"], c["d"]), dt, 1.3)
            s["Xq"], s["Xk"], s["Xv"] = X[:, :, 0], X[:, :, 1], X[:, :, 2]
        else:
            s["Xq"], s["Xk"] = (_normal(gen, (c["B"], L, c["H"], c["d"]), dt, 1.3) for _ in range(2))
            s["Xv"] = None
        s["wq"], s["wk"] = (1 + 0.2 * torch.randn(c["d"], generator=gen, device=DEVICE) for _ in range(2))
        if c["mode"] == "train":
            s["dQ"], s["dK"] = (_normal(gen, (c["B"], c["H"], L, c["d"]), dt) for _ in range(2))
            s["dV"] = _normal(gen, (c["B"], c["H"], L, c["d"]), dt) if c["packed"] else None
        return s
    Bn, S = c["B"], c["S"]

    def heads(h, n, gain=1.0):
        if c["token_major"]:
            return _normal(gen, (Bn, n, h, c["d"]), dt, gain).transpose(1, 2)
        return _normal(gen, (Bn, h, n, c["d"]), dt, gain)

    s["Q"], s["K"], s["V"] = heads(c["H"], c["Lq"]), heads(c["Hkv"], S, 1.5), heads(c["Hkv"], S)
    s["kv_len"] = s["kv_mask"] = None
    valid = torch.ones((Bn, S), dtype=torch.bool, device=DEVICE)
    at = torch.arange(S, device=DEVICE)
    if c["lens"] != "full":
        n = (S * (0.2 + 0.8 * torch.rand(Bn, generator=gen, device=DEVICE))).ceil().clamp(min(S, 2), S)
        if c["lens"] == "empty":
            n[-1] = 0
        s["kv_len"] = n.to(torch.int32)
        valid &= at < n[:, None]
    if c["mask"]:
        keep = (torch.rand((Bn, S), generator=gen, device=DEVICE) < 0.8) | (at < 2)
        s["kv_mask"] = keep.to(torch.uint8)
        valid &= keep
    for name in ("K", "V"):
        s[name].masked_fill_(~valid[:, None, :, None], float("nan"))
    if c["mode"] == "train":
        s["dO"] = heads(c["H"], c["Lq"])
    return s


def prepare(c, seed):
    s = _inputs(c, seed)
    if c["op"] == "rope":
        s["table"] = _table(c)
        L = s["Xq"].shape[1]
        for name in ("Q", "K", "V"):
            s["out" + name] = torch.zeros((c["B"], c["H"], L, c["d"]), dtype=_dtype(c), device=DEVICE) if s["X" + name.lower()] is not None else None
        if c["mode"] == "train":
            if c["packed"]:
                dX = torch.zeros((c["B"], L, 3, c["H"], c["d"]), dtype=_dtype(c), device=DEVICE)
                s["dXq"], s["dXk"], s["dXv"] = dX[:, :, 0], dX[:, :, 1], dX[:, :, 2]
            else:
                s["dXq"], s["dXk"], s["dXv"] = torch.zeros_like(s["Xq"]), torch.zeros_like(s["Xk"]), None
            s["dwq"], s["dwk"] = (torch.zeros(c["d"], device=DEVICE) for _ in range(2))
        return s
    s["O"] = torch.zeros_like(s["Q"])  # (of the same strides)
    s["LSE"] = torch.zeros(s["Q"].shape[:3], device=DEVICE)
    if c["mode"] == "train":
        s["dQ"], s["dK"], s["dV"] = (torch.zeros_like(s[n]) for n in ("Q", "K", "V"))
    return s


# ---- the plain form ------------------------------------------------------------------------------
def _axes(c):
    """Per grid axis: extent, number of channels."""
    return (c["T"], c["dt"]), (c["Hs"], c["dh"]), (c["Ws"], c["dw"])


def _cos_sin(c, table):
    """[L, n/2] cosines and sines of all rotated pairs, tokens in raster order."""
    cos, sin, at = [], [], 0
    grid = (c["T"], c["Hs"], c["Ws"])
    for axis, (extent, n) in enumerate(_axes(c)):
        if n:
            t = table[at:at + extent * n].view(extent, n // 2, 2)
            at += extent * n
            view = [1, 1, 1, n // 2]
            view[axis] = extent
            cos.append(t[..., 0].reshape(view).expand(*grid, n // 2).reshape(-1, n // 2))
            sin.append(t[..., 1].reshape(view).expand(*grid, n // 2).reshape(-1, n // 2))
    return (torch.cat(cos, 1), torch.cat(sin, 1)) if cos else (None, None)


def _turn(c, x, cos, sin):
    """The rotation of x [B, L, H, d]; of the negative angles with -sin."""
    if cos is None:
        return x
    n, y = 2 * cos.shape[1], x.clone()
    cos, sin = cos[None, :, None], sin[None, :, None]
    lo, hi = (slice(0, n // 2), slice(n // 2, n)) if c["halves"] else (slice(0, n, 2), slice(1, n, 2))
    y[..., lo], y[..., hi] = x[..., lo] * cos - x[..., hi] * sin, x[..., lo] * sin + x[..., hi] * cos
    return y


def _to_heads(c, x):
    """[B, L, H, d] in raster order -> [B, H, L, d] in the case's order."""
    if c["block_major"]:
        g = x.reshape(c["B"], c["T"] // c["Ct"], c["Ct"], c["Hs"] // c["Ch"], c["Ch"], c["Ws"] // c["Cw"], c["Cw"], c["H"], c["d"])
        x = g.permute(0, 1, 3, 5, 2, 4, 6, 7, 8).reshape(c["B"], -1, c["H"], c["d"])
    return x.transpose(1, 2).contiguous()


def _from_heads(c, y):
    x = y.transpose(1, 2)
    if c["block_major"]:
        g = x.reshape(c["B"], c["T"] // c["Ct"], c["Hs"] // c["Ch"], c["Ws"] // c["Cw"], c["Ct"], c["Ch"], c["Cw"], c["H"], c["d"])
        x = g.permute(0, 1, 4, 2, 5, 3, 6, 7, 8).reshape(c["B"], -1, c["H"], c["d"])
    return x


def _plain_rope(s):
    c, dt = s["c"], _dtype(s["c"])
    cos, sin = _cos_sin(c, s["table"])
    out = {}
    for name, w in (("q", s["wq"]), ("k", s["wk"])):
        x = s["X" + name].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xhat = x * r
        out[name.upper()] = _to_heads(c, _turn(c, xhat * w, cos, sin).to(dt))
        if c["mode"] == "train":
            u = _turn(c, _from_heads(c, s["d" + name.upper()]).float(), cos, None if sin is None else -sin)
            out["dw" + name] = (u * xhat).sum((0, 1, 2), dtype=torch.float64).float()
            g = u * w
            out["dX" + name] = (r * (g - xhat * (g * xhat).mean(-1, keepdim=True))).to(dt)
    if c["packed"]:
        out["V"] = _to_heads(c, s["Xv"])
        if c["mode"] == "train":
            out["dXv"] = _from_heads(c, s["dV"]).contiguous()
    return out


def _plain_cross(s):
    c, dt = s["c"], _dtype(s["c"])
    Bn, S, d, Hkv = c["B"], c["S"], c["d"], c["Hkv"]
    scale = 1.0 / sqrt(d)
    valid = torch.ones((Bn, S), dtype=torch.bool, device=DEVICE)
    if s["kv_len"] is not None:
        valid = valid & (torch.arange(S, device=DEVICE) < s["kv_len"][:, None])
    if s["kv_mask"] is not None:
        valid = valid & (s["kv_mask"] != 0)
    rows = lambda x: x.float().reshape(Bn, Hkv, -1, d)  # noqa: E731  a group's heads under each other
    zero = torch.zeros((), device=DEVICE)
    Q = rows(s["Q"])
    K, V = (torch.where(valid[:, None, :, None], s[n].float(), zero).contiguous() for n in ("K", "V"))
    Kt, Vt = K.transpose(2, 3).contiguous(), V.transpose(2, 3).contiguous()
    X = torch.matmul(Q, Kt) * scale
    X.masked_fill_(~valid[:, None, None, :], float("-inf"))
    m = X.max(-1, keepdim=True).values
    m = torch.where(m == float("-inf"), zero, m)
    P = torch.exp(X - m)
    l = P.sum(-1, keepdim=True)  # noqa: E741
    LSE = m + torch.log(l)
    P = P / torch.where(l == 0, torch.ones_like(l), l)
    O = torch.matmul(P, V)  # noqa: E741
    like = s["Q"].shape
    out = {"O": O.view(like).to(dt), "LSE": LSE.view(like[:3])}
    if c["mode"] == "train":
        G = rows(s["dO"])
        dS = P * (torch.matmul(G, Vt) - (G * O).sum(-1, keepdim=True)) * scale
        out["dQ"] = torch.matmul(dS, K).view(like).to(dt)
        out["dK"] = torch.matmul(dS.transpose(2, 3).contiguous(), Q).to(dt)
        out["dV"] = torch.matmul(P.transpose(2, 3).contiguous(), G).to(dt)
    return out


# ---- one pass ------------------------------------------------------------------------------------
def _own_rope(s):
    from paper_2509_01085_amd import binding as B

    c = s["c"]
    shp = B.Shape(c["B"], c["H"], c["T"], c["Hs"], c["Ws"], c["Ct"], c["Ch"], c["Cw"], c["d"],
                  B.F32 if c["dtype"] == "fp32" else B.BF16, layout=B.BLOCK_MAJOR if c["block_major"] else B.RASTER)
    rope = B.Rope(c["dt"], c["dh"], c["dw"], B.ROPE_HALVES if c["halves"] else B.ROPE_PAIRS)
    kw = dict(wq=s["wq"], wk=s["wk"], eps=EPS)
    B.qk_norm_rope_fwd(shp, rope, s["table"], s["Xq"], s["Xk"], s["Xv"], Q=s["outQ"], K=s["outK"], V=s["outV"], **kw)
    out = {"Q": s["outQ"], "K": s["outK"]}
    if c["mode"] == "train":
        B.qk_norm_rope_bwd(shp, rope, s["table"], s["Xq"], s["Xk"], s["dQ"], s["dK"], s["dV"], dXq=s["dXq"], dXk=s["dXk"],
                           dXv=s["dXv"], dwq=s["dwq"], dwk=s["dwk"], **kw)
        out.update((n, s[n]) for n in ("dXq", "dXk", "dwq", "dwk"))
    if c["packed"]:
        out["V"] = s["outV"]
        if c["mode"] == "train":
            out["dXv"] = s["dXv"]
    return out


def _own_cross(s):
    from paper_2509_01085_amd import binding as B

    c = s["c"]
    shp = B.CrossShape(c["B"], c["H"], c["Hkv"], c["Lq"], c["S"], c["d"], B.F32 if c["dtype"] == "fp32" else B.BF16)
    B.cross_attn_fwd(shp, s["Q"], s["K"], s["V"], kv_len=s["kv_len"], kv_mask=s["kv_mask"], O=s["O"], LSE=s["LSE"])
    out = {"O": s["O"], "LSE": s["LSE"]}
    if c["mode"] == "train":
        B.cross_attn_bwd(shp, s["Q"], s["K"], s["V"], s["O"], s["LSE"], s["dO"], kv_len=s["kv_len"], kv_mask=s["kv_mask"],
                         dQ=s["dQ"], dK=s["dK"], dV=s["dV"])
        out.update((n, s[n]) for n in ("dQ", "dK", "dV"))
    return out


def run(s):
    if own:
        return _own_rope(s) if s["c"]["op"] == "rope" else _own_cross(s)
    return _plain_rope(s) if s["c"]["op"] == "rope" else _plain_cross(s)


# ---- the definition in 64 bits -------------------------------------------------------------------
def _exact_rope(c, s):
    train = c["mode"] == "train"
    t, h, w = torch.meshgrid(*(torch.arange(n, dtype=torch.float64, device=DEVICE) for n in (c["T"], c["Hs"], c["Ws"])), indexing="ij")
    angles = [pos.reshape(-1, 1) * torch.tensor([THETA ** (-2.0 * i / n) for i in range(n // 2)], dtype=torch.float64, device=DEVICE)
              for pos, n in ((t + c["t0"], c["dt"]), (h, c["dh"]), (w, c["dw"])) if n]
    n = c["dt"] + c["dh"] + c["dw"]
    order = torch.arange(t.numel(), device=DEVICE)  # raster index of every row of the result
    if c["block_major"]:
        block = ((t // c["Ct"]) * (c["Hs"] // c["Ch"]) + h // c["Ch"]) * (c["Ws"] // c["Cw"]) + w // c["Cw"]
        inside = ((t % c["Ct"]) * c["Ch"] + h % c["Ch"]) * c["Cw"] + w % c["Cw"]
        order = torch.argsort((block * (c["Ct"] * c["Ch"] * c["Cw"]) + inside).reshape(-1))
    out = {}
    for name in ("q", "k"):
        x = s["X" + name].double().requires_grad_(train)
        weight = s["w" + name].double().requires_grad_(train)
        y = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["d"] + EPS) * weight
        if n:
            unit = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), torch.cat(angles, 1))[None, :, None]
            if c["halves"]:
                z = torch.complex(y[..., :n // 2], y[..., n // 2:n]) * unit
                y = torch.cat((z.real, z.imag, y[..., n:]), -1)
            else:
                z = torch.view_as_complex(y[..., :n].reshape(*y.shape[:3], n // 2, 2)) * unit
                y = torch.cat((torch.view_as_real(z).flatten(-2), y[..., n:]), -1)
        y = y[:, order].transpose(1, 2)
        out[name.upper()] = y.detach()
        if train:
            out["dX" + name], out["dw" + name] = torch.autograd.grad(y, (x, weight), s["d" + name.upper()].double())
    if c["packed"]:
        out["V"] = s["Xv"][:, order].transpose(1, 2).double()
        if train:
            out["dXv"] = s["dV"].transpose(1, 2)[:, torch.argsort(order)].double()
    return out


def _exact_cross(c, s):
    train, group = c["mode"] == "train", c["H"] // c["Hkv"]
    outs = {n: [] for n in (("O", "LSE", "dQ", "dK", "dV") if train else ("O", "LSE"))}
    for b in range(c["B"]):
        keys = torch.arange(c["S"], device=DEVICE)
        if s["kv_len"] is not None:
            keys = keys[:int(s["kv_len"][b])]
        if s["kv_mask"] is not None:
            keys = keys[s["kv_mask"][b, keys] != 0]
        for k in range(c["Hkv"]):
            K, V = (s[n][b, k, keys].double().requires_grad_(train) for n in ("K", "V"))  # the valid states alone
            dK, dV = (torch.zeros((c["S"], c["d"]), dtype=torch.float64, device=DEVICE) for _ in range(2))
            for h in range(k * group, (k + 1) * group):
                Q = s["Q"][b, h].double().requires_grad_(train)
                X = Q @ K.t() / sqrt(c["d"])
                O = torch.softmax(X, -1) @ V  # noqa: E741
                outs["O"].append(O.detach())
                outs["LSE"].append(torch.logsumexp(X.detach(), -1) if len(keys) else torch.full((c["Lq"],), float("-inf"), dtype=torch.float64, device=DEVICE))
                if train:
                    g = torch.autograd.grad(O, (Q, K, V), s["dO"][b, h].double())
                    outs["dQ"].append(g[0])
                    dK[keys] += g[1]
                    dV[keys] += g[2]
            if train:
                outs["dK"].append(dK)
                outs["dV"].append(dV)
    return {n: torch.stack(v).view(c["B"], -1, *v[0].shape) for n, v in outs.items()}


def exact(c, seed):
    s = _inputs(c, seed)
    return _exact_rope(c, s) if c["op"] == "rope" else _exact_cross(c, s)
