"""Norm of queries and keys with the rotation, forward and backward, against the plain 64-bit form."""
import dataclasses

import pytest
import torch

from paper_2509_01085_amd import binding as B

import gpu_util as U
import plain_ops as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


def shape(grid, block, B_=1, H=2, d=64, dtype=B.BF16, layout=0):
    return B.Shape(B_, H, *grid, *block, d, dtype, layout=layout)


# name: shape, rope (None: no rotation), how the projection's output lies in memory
CASES = {
    "tiny_pairs": (shape((4, 8, 8), (2, 4, 4), d=64, dtype=B.F32), B.Rope(24, 20, 20), "packed"),
    "tiny_halves": (shape((4, 8, 8), (2, 4, 4), d=64, dtype=B.F32), B.Rope(24, 20, 20, 1), "packed"),
    "block_major": (shape((4, 6, 8), (2, 3, 4), 2, 3, 128, layout=1), B.Rope(44, 42, 42), "packed"),
    "block_major_f32": (shape((6, 5, 4), (3, 5, 2), 2, 3, 72, B.F32, 1), B.Rope(8, 14, 10, 1), "heads"),
    "one_token": (shape((1, 1, 1), (1, 1, 1), 1, 1, 128), B.Rope(128, 0, 0, 1), "separate"),
    "text": (shape((333, 1, 1), (1, 1, 1), 2, 5, 96), B.Rope(96, 0, 0, 1), "separate"),
    "d8": (shape((3, 3, 5), (1, 1, 1), 2, 3, 8), B.Rope(4, 2, 2), "packed"),
    "d24": (shape((3, 3, 5), (1, 1, 1), 2, 7, 24, B.F32), B.Rope(8, 4, 4, 1), "separate"),
    "d32": (shape((2, 7, 9), (1, 1, 1), 3, 4, 32), B.Rope(16, 8, 0, 1), "packed"),
    "d40": (shape((2, 7, 9), (2, 1, 3), 1, 9, 40, layout=1), B.Rope(12, 14, 14), "heads"),
    "d160": (shape((5, 4, 6), (1, 2, 2), 1, 3, 160, layout=1), B.Rope(60, 50, 50), "packed"),
    "d256_f32": (shape((2, 3, 5), (1, 1, 1), 2, 2, 256, B.F32), B.Rope(0, 64, 64), "packed"),
    "d256_unturned": (shape((2, 3, 5), (1, 1, 1), 2, 2, 256), B.Rope(32, 0, 0, 1), "padded"),
    "no_rotation": (shape((7, 5, 3), (7, 1, 1), 2, 3, 128), None, "packed"),
    "empty_rotation": (shape((7, 5, 3), (7, 1, 1), 2, 3, 64), B.Rope(0, 0, 0), "packed"),
    "many_groups": (shape((8, 40, 52), (4, 4, 4), 1, 3, 64, layout=1), B.Rope(24, 20, 20), "packed"),
    "many_heads": (shape((1, 3, 3), (1, 1, 1), 1, 40, 128), B.Rope(44, 42, 42), "packed"),
}


def projection(shp, lay, gen):
    """Xq, Xk, Xv of the same strides, and the whole memory they lie in."""
    Bn, L, H, d, dt = shp.B, shp.L, shp.H, shp.d, shp.torch_dtype
    mk = lambda *s: (torch.randn(s, generator=gen) * 1.7).to(dt).to(DEV)  # noqa: E731
    if lay == "packed":
        X = mk(Bn, L, 3, H, d)
        return [X[:, :, i] for i in range(3)], X
    if lay == "separate":
        X = mk(3, Bn, L, H, d)
        return list(X), X
    if lay == "heads":  # heads ahead of tokens
        X = mk(3, Bn, H, L, d)
        return [x.transpose(1, 2) for x in X], X
    X = mk(Bn, L, H, 3, d + 16)  # padded rows
    return [X[..., i, 8:8 + d] for i in range(3)], X


@pytest.mark.parametrize("name", list(CASES))
def test_against_the_plain_form(name):
    shp, rope, lay = CASES[name]
    U.progress(f"qk_norm_rope {name}")
    gen = torch.Generator().manual_seed(sum(map(ord, name)))
    (Xq, Xk, Xv), _ = projection(shp, lay, gen)
    dt, half = shp.torch_dtype, P.HALF[shp.torch_dtype]
    wq = (torch.rand(shp.d, generator=gen) + 0.5).to(DEV)
    wk = torch.randn(shp.d, generator=gen).to(DEV)
    size = (shp.B, shp.H, shp.L, shp.d)
    dQ, dK, dV = (torch.randn(size, generator=gen).to(dt).to(DEV) for _ in range(3))
    theta, origin = 500.0, (7, 100001, -3)
    table = B.rope_table(shp, rope, theta, origin) if rope is not None else None
    Q, K, V = B.qk_norm_rope_fwd(shp, rope, table, Xq, Xk, Xv, wq=wq, wk=wk, eps=EPS)
    (dXq, dXk, dXv), whole = projection(shp, lay, gen)
    before = whole.clone()
    out = B.qk_norm_rope_bwd(shp, rope, table, Xq, Xk, dQ, dK, dV, wq=wq, wk=wk, eps=EPS, dXq=dXq, dXk=dXk, dXv=dXv)
    torch.cuda.synchronize()
    order = P.row_order(shp)
    assert torch.equal(V.cpu(), Xv.cpu()[:, order].transpose(1, 2))
    assert torch.equal(dXv.cpu()[:, order].transpose(1, 2), dV.cpu())
    for X, w, Y, dY, dX, dw in ((Xq, wq, Q, dQ, out[0], out[3]), (Xk, wk, K, dK, out[1], out[4])):
        ref = P.norm_rope(shp, rope, X.double().cpu(), w.double().cpu(), EPS, theta, origin, dY.double().cpu())
        P.check("Y", Y, ref["Y"], half)
        P.check("dX", dX, ref["dX"], half)
        P.check("dw", dw, ref["dw"], P.U32)
    if lay == "padded":  # what lies between the rows is as it was
        assert torch.equal(whole[..., :8], before[..., :8]) and torch.equal(whole[..., 8 + shp.d:], before[..., 8 + shp.d:])


def test_a_table_is_cos_and_sin_of_every_coordinate():
    shp, rope = shape((5, 3, 4), (1, 1, 1), d=32), B.Rope(12, 10, 2)
    origin, theta = (10 ** 6, -17, 2 ** 40), 10000.0
    got = B.rope_table(shp, rope, theta, origin).cpu().double()
    want = []
    for extent, first, n in zip((5, 3, 4), origin, (12, 10, 2)):
        for p in range(extent):
            for i in range(n // 2):
                a = torch.tensor(float(first + p) * theta ** (-2.0 * i / n), dtype=torch.float64)
                want += [a.cos(), a.sin()]
    # one rounding, and an angle of up to 2^40 whose own rounding in 64 bits is 2^-13
    assert (got - torch.stack(want)).abs().max() <= 2.0 ** -24 + 2.0 ** -12
    assert (got - torch.stack(want))[:60].abs().max() <= 2.0 ** -24 + 1e-9


@pytest.mark.parametrize("there", ("q", "k", "v", "qk", "kv", "qv"))
def test_tensors_may_be_left_out(there):
    shp, rope = shape((3, 4, 5), (1, 1, 1), 2, 3, 64), B.Rope(24, 20, 20)
    gen = torch.Generator().manual_seed(3)
    X, _ = projection(shp, "packed", gen)
    dY = [torch.randn((shp.B, shp.H, shp.L, shp.d), generator=gen).to(torch.bfloat16).to(DEV) for _ in range(3)]
    table = B.rope_table(shp, rope)
    every = B.qk_norm_rope_fwd(shp, rope, table, *X)
    grads = B.qk_norm_rope_bwd(shp, rope, table, *X[:2], *dY)
    on = [c in there for c in "qkv"]
    some = B.qk_norm_rope_fwd(shp, rope, table, *(x if f else None for x, f in zip(X, on)))
    g = B.qk_norm_rope_bwd(shp, rope, table, *(x if f else None for x, f in zip(X[:2], on)), *(y if f else None for y, f in zip(dY, on)))
    for got, want, f in zip(some + g, every + grads, on + on + on[:2]):
        assert (got is None) == (not f)
        assert got is None or torch.equal(got, want)


def test_weights_of_one_are_no_weights_and_repeated_inputs_are_read():
    shp = shape((3, 4, 5), (1, 1, 1), 2, 3, 72)
    gen = torch.Generator().manual_seed(4)
    x = torch.randn((1, shp.L, 1, shp.d), generator=gen).to(torch.bfloat16).to(DEV).expand(2, shp.L, 3, shp.d)
    ones = torch.ones(shp.d, device=DEV)
    Q, _, _ = B.qk_norm_rope_fwd(shp, None, None, x)
    Q1, _, _ = B.qk_norm_rope_fwd(shp, None, None, x.contiguous(), wq=ones)
    assert torch.equal(Q, Q1)
    with pytest.raises(B.BsaError) as e:  # a result may not repeat
        B.qk_norm_rope_bwd(shp, None, None, x, None, Q, dXq=x)
    assert e.value.status == -9


def test_rows_of_zeros_infinities_and_nan_stay_in_their_rows():
    shp, rope = shape((1, 8, 8), (1, 1, 1), 1, 2, 64), B.Rope(0, 32, 32)
    gen = torch.Generator().manual_seed(5)
    x = torch.randn((1, shp.L, 2, 64), generator=gen).to(torch.bfloat16)
    y = torch.randn((1, 2, shp.L, 64), generator=gen).to(torch.bfloat16).to(DEV)
    odd = x.clone()
    odd[0, 3, 1], odd[0, 4, 0, 5], odd[0, 9, 1, 63] = 0.0, float("inf"), float("nan")
    table = B.rope_table(shp, rope)
    Q, _, _ = B.qk_norm_rope_fwd(shp, rope, table, x.to(DEV))
    Qo, _, _ = B.qk_norm_rope_fwd(shp, rope, table, odd.to(DEV))
    dX = B.qk_norm_rope_bwd(shp, rope, table, x.to(DEV), None, y)[0]
    dXo = B.qk_norm_rope_bwd(shp, rope, table, odd.to(DEV), None, y)[0]
    clean = torch.ones((shp.L, 2), dtype=torch.bool, device=DEV)
    for n, h in ((3, 1), (4, 0), (9, 1)):
        clean[n, h] = False
    assert torch.equal(Q.transpose(1, 2)[0][clean], Qo.transpose(1, 2)[0][clean])
    assert torch.equal(dX[0][clean], dXo[0][clean])
    assert (Qo[0, 1, 3] == 0).all() and torch.isfinite(dXo[0, 3, 1]).all()  # x = 0: eps keeps it finite
    assert torch.isnan(Qo[0, 0, 4]).any() and torch.isnan(Qo[0, 1, 9]).all()


def test_offsets_past_32_bits():
    """Tokens 2^17 elements apart, 2^16 of them: the last ones lie beyond 2^32 elements."""
    shp = shape((1, 1, 65536), (1, 1, 1), 1, 1, 64)
    big = torch.empty((1, shp.L, 1, 1 << 17), dtype=torch.bfloat16, device=DEV)
    X = big[..., :64]
    gen = torch.Generator().manual_seed(6)
    x = torch.randn((1, shp.L, 1, 64), generator=gen).to(torch.bfloat16).to(DEV)
    X.copy_(x)
    Q, _, _ = B.qk_norm_rope_fwd(shp, None, None, X)
    want, _, _ = B.qk_norm_rope_fwd(shp, None, None, x)
    assert torch.equal(Q, want)
    B.qk_norm_rope_bwd(shp, None, None, X, None, Q, dXq=X)
    assert torch.equal(X, B.qk_norm_rope_bwd(shp, None, None, x, None, Q)[0])


def test_replayed_and_on_other_streams():
    shp, rope, _ = CASES["block_major"]
    gen = torch.Generator().manual_seed(8)
    X, _ = projection(shp, "packed", gen)
    w = torch.rand(shp.d, device=DEV)
    dY = [torch.randn((shp.B, shp.H, shp.L, shp.d), generator=gen).to(torch.bfloat16).to(DEV) for _ in range(3)]
    table = B.rope_table(shp, rope)
    Y = [torch.empty_like(y) for y in dY]
    dX = [torch.empty_like(x) for x in X]
    dw = [torch.empty_like(w) for _ in range(2)]
    ws = torch.empty(B.qk_norm_rope_bwd_workspace_bytes(shp), dtype=torch.uint8, device=DEV)

    def step():
        B.qk_norm_rope_fwd(shp, rope, table, *X, wq=w, wk=w, Q=Y[0], K=Y[1], V=Y[2])
        B.qk_norm_rope_bwd(shp, rope, table, *X[:2], *dY, wq=w, wk=w, dXq=dX[0], dXk=dX[1], dXv=dX[2], dwq=dw[0], dwk=dw[1], workspace=ws)

    step()
    torch.cuda.synchronize()
    outs = Y + dX + dw
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for k in range(3):
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), f"replay {k}"
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), f"stream {k}"


def test_new_inputs_are_seen():
    """Nothing is kept from one call for the next: the same memory with other contents gives other results."""
    shp = shape((1, 4, 8), (1, 1, 1), 1, 2, 64)
    x = torch.randn((1, shp.L, 2, 64), device=DEV).to(torch.bfloat16)
    Q, _, _ = B.qk_norm_rope_fwd(shp, None, None, x)
    x.mul_(-1)
    assert torch.equal(B.qk_norm_rope_fwd(shp, None, None, x)[0], -Q)
    with pytest.raises(ValueError, match="Xq"):
        B.qk_norm_rope_fwd(dataclasses.replace(shp, T=2), None, None, x)
