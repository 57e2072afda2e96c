"""The operators around the attention: what they refuse, on the host and without a GPU, and their plain forms against differences."""
import ctypes as C
import dataclasses

import pytest
import torch

from paper_2509_01085_amd import binding as B

import plain_ops as P

SHAPE = B.Shape(2, 3, 4, 8, 8, 2, 4, 4, 64, B.BF16)
ROPE = B.Rope(24, 20, 20)
p = 4096  # a non-NULL dummy address: these calls must fail validation and never touch it


def strides(b, l, h):  # noqa: E741
    return C.byref(B.StridesStruct(b, l, h))


GOOD_X = (SHAPE.L * SHAPE.H * 64, SHAPE.H * 64, 64)


def fwd(shape=SHAPE, rope=ROPE, table=p, x=(p, p, p), xs=GOOD_X, eps=1e-6, y=(p, p, p), w=(p, p)):
    return B.lib().bsa_qk_norm_rope_fwd(C.byref(shape.c()), C.byref(rope.c()) if rope else None, table, *x, strides(*xs) if xs else None,
                                        *w, eps, *y, None)


def bwd(shape=SHAPE, rope=ROPE, table=p, x=(p, p), xs=GOOD_X, eps=1e-6, dy=(p, p, p), dx=(p, p, p), dxs=GOOD_X, dw=(p, p), ws=p, wsb=None):
    wsb = B.qk_norm_rope_bwd_workspace_bytes(SHAPE) if wsb is None else wsb
    return B.lib().bsa_qk_norm_rope_bwd(C.byref(shape.c()), C.byref(rope.c()) if rope else None, table, *x, strides(*xs) if xs else None, p, p,
                                        eps, *dy, *dx, strides(*dxs) if dxs else None, *dw, ws, wsb, None)


def test_norm_rope_refusals():
    new = dataclasses.replace
    assert fwd(new(SHAPE, dtype=5)) == -5 and fwd(new(SHAPE, d=60)) == -2 and fwd(new(SHAPE, B=0)) == -2 and fwd(new(SHAPE, Ct=3)) == -2
    assert fwd(new(SHAPE, T=4096, Hs=4096, Ws=4096)) == -2  # token numbers are 32 bits
    for rope in (B.Rope(23, 20, 21), B.Rope(24, 20, 18), B.Rope(40, 20, 20), B.Rope(-8, 20, 20), B.Rope(24, 20, 20, 2)):
        assert fwd(rope=rope) == -2 and bwd(rope=rope) == -2, rope
    assert fwd(table=None) == -1 and fwd(xs=None) == -1 and fwd(x=(None,) * 3, y=(None,) * 3) == -1
    assert fwd(x=(p, None, p)) == -1 and fwd(y=(p, p, None)) == -1  # a tensor and its result come together
    for eps in (0.0, -1e-6, float("nan"), float("inf")):
        assert fwd(eps=eps) == -3 and bwd(eps=eps) == -3
    assert fwd(x=(p + 8, p, p)) == -9 and fwd(y=(p, p, p + 4)) == -9
    for xs in ((-8, 192, 64), (GOOD_X[0], 196, 64), (GOOD_X[0], 192, 60), (1 << 40, 192, 64)):
        assert fwd(xs=xs) == -9 and bwd(xs=xs) == -9, xs
    assert fwd(new(SHAPE, dtype=B.F32), xs=(GOOD_X[0], 194, 64)) == -9
    assert bwd(table=None) == -1 and bwd(dxs=None) == -1 and bwd(xs=None) == -1 and bwd(dy=(None,) * 3, dx=(None,) * 3, x=(None, None), dw=(None, None)) == -1
    assert bwd(x=(None, p)) == -1 and bwd(dy=(p, None, p)) == -1 and bwd(dx=(p, p, None)) == -1
    assert bwd(x=(None, p), dy=(None, p, p), dx=(None, p, p)) == -1  # a sum of gradients that are not there
    assert bwd(ws=None) == -7 and bwd(wsb=B.qk_norm_rope_bwd_workspace_bytes(SHAPE) - 1) == -7
    for dxs in ((GOOD_X[0], 192, 56), (GOOD_X[0], 128, 64), (0, 192, 64), (64, 192, 64)):  # elements that would be written twice
        assert bwd(dxs=dxs) == -9, dxs
    assert B.qk_norm_rope_bwd_workspace_bytes(new(SHAPE, d=4)) == 0
    assert b"multiples of 16" in B.lib().bsa_strerror(-9)


def test_rope_table_refusals():
    lib = B.lib()
    table = lambda rope=ROPE, theta=1e4, t=p, shape=SHAPE: lib.bsa_rope_table(C.byref(shape.c()), C.byref(rope.c()) if rope else None, theta, 0, 0, 0, t, None)  # noqa: E731
    assert table(rope=None) == -1 and table(t=None) == -1 and table(B.Rope(1, 2, 5)) == -2
    for theta in (0.0, -1.0, float("nan"), float("inf")):
        assert table(theta=theta) == -3
    assert lib.bsa_rope_table_bytes(C.byref(SHAPE.c()), C.byref(ROPE.c())) == 4 * (4 * 24 + 8 * 20 + 8 * 20)
    assert lib.bsa_rope_table_bytes(C.byref(SHAPE.c()), C.byref(B.Rope(1, 2, 5).c())) == 0


CROSS = B.CrossShape(2, 6, 3, 100, 77, 64, B.BF16)


def cfwd(shape=CROSS, c=None, t=(p, p, p), out=(p, p), scale=0.125, ws=p, wsb=1 << 40):
    return B.lib().bsa_cross_attn_fwd(C.byref(c or shape.c()), *t, None, None, scale, *out, ws, wsb, None)


def cbwd(shape=CROSS, c=None, t=(p,) * 6, out=(p,) * 3, scale=0.125, grads=None, ws=p, wsb=1 << 40):
    return B.lib().bsa_cross_attn_bwd(C.byref(c or shape.c()), *t, None, None, scale, *out, grads, ws, wsb, None)


def test_cross_attention_refusals():
    new = dataclasses.replace
    for bad, status in ((new(CROSS, dtype=2), -5), (new(CROSS, d=12), -2), (new(CROSS, d=264), -2), (new(CROSS, Lq=0), -2), (new(CROSS, S=0), -2),
                        (new(CROSS, B=-1), -2), (new(CROSS, Hkv=4), -2), (new(CROSS, Hkv=0), -2), (new(CROSS, Hkv=1, Lq=1 << 30), -2)):
        assert cfwd(bad) == status and cbwd(bad) == status, bad
        assert B.cross_fwd_workspace_bytes(bad) == 0 and B.cross_bwd_workspace_bytes(bad) == 0
    assert B.lib().bsa_cross_attn_fwd(None, p, p, p, None, None, 0.1, p, p, p, 1 << 40, None) == -1
    for i in range(3):
        assert cfwd(t=[None if k == i else p for k in range(3)]) == -1 and cfwd(t=[p + 8 if k == i else p for k in range(3)]) == -9
        assert cbwd(out=[None if k == i else p for k in range(3)]) == -1 and cbwd(out=[p + 2 if k == i else p for k in range(3)]) == -9
    for i in range(6):
        assert cbwd(t=[None if k == i else p for k in range(6)]) == -1
    assert cfwd(out=(None, p)) == -1 and cfwd(out=(p, None)) == -1
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert cfwd(scale=scale) == -3 and cbwd(scale=scale) == -3
    few = B.CrossShape(1, 1, 1, 1, 100000, 128, B.BF16)  # one row: its keys are split, which needs scratch
    need = B.cross_fwd_workspace_bytes(few)
    assert need > 0 and cfwd(few, ws=None) == -7 and cfwd(few, wsb=need - 1) == -7
    need = B.cross_bwd_workspace_bytes(CROSS)
    assert need > 0 and cbwd(ws=None) == -7 and cbwd(wsb=need - 1) == -7
    assert B.cross_fwd_workspace_bytes(B.CrossShape(1, 12, 12, 33280, 512, 128, B.BF16)) == 0


def test_cross_attention_strides():
    def with_strides(which, **kw):
        c = CROSS.c()
        for k, v in kw.items():
            setattr(getattr(c, which), k, v)
        return c

    for which in "qkv":
        for kw in (dict(l=68), dict(h=-64), dict(b=1 << 40)):
            assert cfwd(c=with_strides(which, **kw)) == -9 and cbwd(c=with_strides(which, **kw)) == -9, (which, kw)
    for kw in (dict(l=56), dict(h=0), dict(b=0), dict(l=64, h=64)):  # O: elements that would be written twice
        assert cfwd(c=with_strides("o", **kw)) == -9, kw
    # repeated inputs are read as they are; their gradients need memory of their own
    assert cbwd(c=with_strides("k", b=0)) == -9
    good = [B.StridesStruct(h * n * 64, 64, n * 64) for h, n in ((6, 100), (6, 100), (3, 77), (3, 77))]
    for i in range(4):
        for bad in (dict(l=60), dict(b=-8)) + (() if i == 0 else (dict(b=0), dict(h=64), dict(l=32))):
            g = [B.StridesStruct(s.b, s.l, s.h) for s in good]
            for k, v in bad.items():
                setattr(g[i], k, v)
            assert cbwd(grads=(B.StridesStruct * 4)(*g)) == -9, (i, bad)


def test_the_binding_refuses_what_a_pointer_cannot_tell():
    x = torch.zeros((2, SHAPE.L, 3, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current GPU"):
        B.qk_norm_rope_fwd(SHAPE, None, None, x, x, None)
    with pytest.raises(ValueError, match="must be given"):
        B.qk_norm_rope_fwd(SHAPE, None, None)
    with pytest.raises(ValueError, match="must be given"):
        B.qk_norm_rope_bwd(SHAPE, None, None)
    q, k = torch.zeros((2, 6, 100, 64)), torch.zeros((2, 3, 77, 64))
    with pytest.raises(ValueError, match="current GPU"):
        B.cross_attn_fwd(CROSS, q, k, k)
    dev = torch.device("cpu")
    take = lambda t, **kw: B._take(t, "Q", (2, 6, 100, 64), torch.float32, dev, **kw)  # noqa: E731
    assert take(None) is None and take(q) == q.data_ptr()
    for bad in (q[:1], q.double(), torch.zeros((2, 6, 64, 100)).transpose(2, 3)):
        with pytest.raises(ValueError, match="Q"):
            take(bad)
    with pytest.raises(ValueError, match="contiguous"):
        take(torch.zeros((2, 100, 6, 64)).transpose(1, 2), dense=True)
    with pytest.raises(ValueError, match="same strides"):
        B._same_strides((x, torch.zeros((2, SHAPE.L, 2, 3, 64))[:, :, 0]), "Xq and Xk")
    one = torch.zeros((1, 5, 3, 64))
    B._same_strides((one, torch.zeros((2, 5, 3, 64))[:1]), "Xq and Xk")  # the stride of an extent of 1 counts for nothing


@pytest.mark.parametrize("style", (0, 1))
def test_plain_norm_rope_gradient_against_differences(style):
    torch.manual_seed(1)
    shape, rope = B.Shape(1, 2, 2, 2, 3, 1, 2, 3, 16, B.F32, layout=1), B.Rope(4, 2, 2, style)
    X, dY = torch.randn(1, shape.L, 2, 16).double(), torch.randn(1, 2, shape.L, 16).double()
    w = torch.rand(16).double() + 0.5
    f = lambda X, w: float((P.norm_rope(shape, rope, X, w, 1e-3)["Y"][0] * dY).sum())  # noqa: E731
    out = P.norm_rope(shape, rope, X, w, 1e-3, dY=dY)
    vx, vw, h = torch.randn_like(X), torch.randn_like(w), 1e-5
    want = (f(X + h * vx, w + h * vw) - f(X - h * vx, w - h * vw)) / (2 * h)
    got = float((out["dX"][0] * vx).sum() + (out["dw"][0] * vw).sum())
    assert abs(got - want) < 1e-7 * (1 + abs(want))


def test_plain_cross_gradient_against_differences():
    torch.manual_seed(2)
    Q, K, V, dO = (torch.randn(2, h, n, 16).double() for h, n in ((4, 5), (2, 9), (2, 9), (4, 5)))
    ok = P.valid_states(2, 9, torch.tensor([9, 6]), torch.tensor([[1, 0, 1, 1, 1, 1, 1, 1, 1]] * 2))
    f = lambda Q, K, V: float((P.cross(Q, K, V, ok, 0.3)["O"][0] * dO).sum())  # noqa: E731
    out = P.cross(Q, K, V, ok, 0.3, dO)
    v, h = [torch.randn_like(t) for t in (Q, K, V)], 1e-5
    want = (f(*(t + h * x for t, x in zip((Q, K, V), v))) - f(*(t - h * x for t, x in zip((Q, K, V), v)))) / (2 * h)
    got = sum(float((out[n][0] * x).sum()) for n, x in zip(("dQ", "dK", "dV"), v))
    assert abs(got - want) < 1e-7 * (1 + abs(want))


def test_more_work_than_a_launch_takes_is_refused():
    for d, most in ((32, 30), (64, 29), (128, 28), (256, 27)):
        wide = B.Shape(1, 1, 1 << most, 1, 1, 1, 1, 1, d, B.BF16)
        assert fwd(wide, rope=None, xs=(0, d, d)) == -2 and bwd(wide, rope=None, xs=(0, d, d), dxs=(0, d, d)) == -2, d
    rows, keys = B.CrossShape(1, 1, 1, 1 << 30, 1, 8, B.BF16), B.CrossShape(1, 1, 1, 1, 1 << 29, 8, B.BF16)
    assert cfwd(rows) == -2 and cbwd(rows) == -2 and cbwd(keys) == -2
    assert B.cross_fwd_workspace_bytes(rows) == 0 and B.cross_fwd_workspace_bytes(keys) > 0
