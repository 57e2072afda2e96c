"""Norm and rotation of rows of zeros and of tiny elements, where eps decides."""
import pytest
import torch

from paper_2509_01085_amd import binding as B

import plain_ops as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("eps", (2.0 ** -126, 1e-30, 1e-6))
@pytest.mark.parametrize("dtype,d", ((B.F32, 64), (B.BF16, 128), (B.F32, 24)))
def test_rows_that_eps_decides(dtype, d, eps):
    shp = B.Shape(1, 2, 1, 2, 4, 1, 1, 1, d, dtype)
    gen = torch.Generator().manual_seed(91)
    # squares of these and their sums are normal floats, or zero
    size = torch.tensor([0.0, 1e-18, 1e-15, 1e-8, 1e-3, 1.0, 1e6, 1e17])[None, :, None, None]
    x = (torch.randn((1, 8, 2, d), generator=gen).clamp(-3, 3).sign() * (1 + torch.rand((1, 8, 2, d), generator=gen)) * size).to(shp.torch_dtype)
    dY = torch.randn((1, 2, 8, d), generator=gen).to(shp.torch_dtype)
    Q = B.qk_norm_rope_fwd(shp, None, None, x.to(DEV), eps=eps)[0]
    dX, *_, dw, _ = B.qk_norm_rope_bwd(shp, None, None, x.to(DEV), None, dY.to(DEV), eps=eps)
    ref = P.norm_rope(shp, None, x.double(), None, float(torch.tensor(eps, dtype=torch.float32)), dY=dY.double())
    half = P.HALF[shp.torch_dtype]
    for n, t in (("Y", Q), ("dX", dX)):
        P.check(n, t, ref[n], half)
    P.check("dw", dw, ref["dw"], P.U32)
