"""Cross attention: an infinity in a valid state's values is the result's in its channel, wherever the state stands in a tile of keys and
however the valid states are told."""
import pytest
import torch

from paper_2509_01085_amd import binding as B

import gpu_util as U
import plain_ops as P
from test_gpu_cross_attn import reference, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("how", ("length", "mask", "both"))
@pytest.mark.parametrize("dtype", (B.BF16, B.F32))
@pytest.mark.parametrize("Lq,S,d,last", ((40, 100, 64, 63), (40, 100, 64, 64), (40, 100, 128, 37), (33, 100, 256, 70), (200, 300, 72, 299), (1, 20, 96, 0),
                                         (1, 3000, 64, 2100), (5, 2000, 128, 1999)))
def test_the_last_valid_state_holds_an_infinity(dtype, Lq, S, d, last, how):
    s = B.CrossShape(2, 2, 1, Lq, S, d, dtype)
    U.progress(f"infinite values {s} {last} {how}")
    lens = [last + 1, S]
    Q, K, V, dO, ok, valid = tensors(dict(shape=s, lens=lens, mask=False, lay="heads"), 61)
    V[0, 0, last, 5] = float("inf")
    V[1, 0, S // 2, 3] = float("-inf")
    if how != "length":
        valid["kv_mask"] = ok.to(torch.uint8).to(Q.device)
    if how == "mask":
        valid["kv_len"] = None
    O, LSE = B.cross_attn_fwd(s, Q, K, V, **valid)
    dV = B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, **valid)[2]
    ref = reference(s, Q, K, V, ok, dO)
    assert torch.isposinf(ref["O"][0][0, :, :, 5]).all() and torch.isneginf(ref["O"][0][1, :, :, 3]).all()
    for n, t in (("O", O), ("LSE", LSE), ("dV", dV)):
        P.check(n, t, ref[n], P.U32 if n == "LSE" else P.HALF[s.torch_dtype])
