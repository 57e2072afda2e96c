"""The bf16 cross attention's error against 64 bits is that of the roundings the data type asks for: P to bf16 relative to the row's maximum,
so that the key at the maximum has none, and the stored O.  P relative to a maximum that lags by up to 2^6 has 1.09 to 1.15 times that error over 300 to 512 states."""
from math import log2, e, sqrt

import pytest
import torch

from paper_2509_01085_amd import binding as B

import gpu_util as U
from test_gpu_cross_attn import DEV

pytestmark = pytest.mark.gpu


def rounded(x):
    return x.to(torch.bfloat16).double()


# A running maximum moves from tile to tile, and keys ahead of the last move are rounded relative to an earlier one: in an emulation of the
# walk 0.97 to 0.99 of the error, less where shares of the keys are joined.  The roundings of the stored O are the same nearly everywhere, so the ratio scatters by less than 1 %: what
# is above 1.03 is an error that the roundings do not explain.
@pytest.mark.parametrize("spread", (1.5, 3.0))
@pytest.mark.parametrize("H,Lq,S,d", ((2, 512, 512, 128), (2, 512, 300, 64), (40, 512, 512, 64), (1, 600, 2000, 128), (2, 300, 2000, 64), (2, 512, 512, 256),
                                      (2, 512, 300, 72), (8, 1, 9000, 128)))
def test_error_is_that_of_the_roundings(H, Lq, S, d, spread):
    s = B.CrossShape(1, H, 1, Lq, S, d, B.BF16)
    U.progress(f"cross attention precision {s} {spread}")
    gen = torch.Generator().manual_seed(71)
    mk = lambda h, n, gain=1.0: (torch.randn((1, h, n, d), generator=gen) * gain).to(torch.bfloat16).to(DEV)  # noqa: E731
    Q, K, V = mk(H, Lq), mk(1, S, spread), mk(1, S)
    O, _ = B.cross_attn_fwd(s, Q, K, V)  # noqa: E741
    got = model = 0.0
    k, v = K[0, 0].double().cpu(), V[0, 0].double().cpu()
    for h in range(min(H, 8)):
        y = Q[0, h].double().cpu() @ k.T * (log2(e) / sqrt(d))
        p = torch.exp2(y - y.max(1, keepdim=True).values)
        l = p.sum(1, keepdim=True)  # noqa: E741
        ref = p @ v / l
        got += float((O[0, h].double().cpu() - ref).square().sum())
        model += float((rounded((rounded(p.float()) @ v / l).float()) - ref).square().sum())
    U.record(f"cross_precision_{H}_{Lq}_{S}_{d}_{spread}", "O", {"error_over_model": float(f"{sqrt(got / model):.4f}")})
    print("error over model", sqrt(got / model))
    assert got <= 1.03 ** 2 * model, sqrt(got / model)
