"""Calls of the operators around the attention on several streams at once, each with a workspace of its own, give what they give alone."""
import pytest
import torch

from paper_2509_01085_amd import binding as B

import gpu_util as U
from test_gpu_cross_attn import DEV, tensors

pytestmark = pytest.mark.gpu


def cross(shape, lens, seed):
    Q, K, V, dO, _, valid = tensors(dict(shape=shape, lens=lens, mask=False, lay="heads"), seed)

    def run():
        O, LSE = B.cross_attn_fwd(shape, Q, K, V, **valid)
        return (O, LSE, *B.cross_attn_bwd(shape, Q, K, V, O, LSE, dO, **valid))

    return run


def rope(seed):
    shp, r = B.Shape(2, 4, 8, 16, 20, 4, 4, 4, 128, B.BF16, layout=B.BLOCK_MAJOR), B.Rope(44, 42, 42)
    gen = torch.Generator(DEV).manual_seed(seed)
    X = torch.randn((2, shp.L, 3, 4, 128), generator=gen, device=DEV).to(torch.bfloat16)
    w = torch.rand(128, generator=gen, device=DEV)
    table = B.rope_table(shp, r)

    def run():
        Y = B.qk_norm_rope_fwd(shp, r, table, *X.unbind(2), wq=w, wk=w)
        return (*Y, *B.qk_norm_rope_bwd(shp, r, table, X[:, :, 0], X[:, :, 1], *Y, wq=w, wk=w))

    return run


def test_streams_do_not_meet():
    U.progress("operators on several streams")
    calls = [cross(B.CrossShape(2, 12, 12, 1000, 4096, 128, B.BF16), [4096, 100], 1), cross(B.CrossShape(3, 8, 2, 1, 1500, 128, B.BF16), [1500, 70, 700], 2),
             cross(B.CrossShape(1, 2, 2, 300, 161, 64, B.F32), None, 3), rope(4)]
    want = [[t.clone() for t in f()] for f in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for turn in range(3):
        got = []
        for f, s in zip(calls, streams):
            with torch.cuda.stream(s):
                got.append(f())
        torch.cuda.synchronize()
        for i, (g, w) in enumerate(zip(got, want)):
            assert all(torch.equal(a, b) for a, b in zip(g, w)), (turn, i)
