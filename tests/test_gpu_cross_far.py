"""Cross attention of tensors whose tokens lie so far apart that a tile's offsets need more than 31 bits, and of ones just below that."""
import pytest
import torch

from paper_2509_01085_amd import binding as B

import gpu_util as U
import plain_ops as P
from test_gpu_cross_attn import DEV, reference, tensors

pytestmark = pytest.mark.gpu


def apart(n, h, d, stride, dt, count):
    """`count` tensors [1, h, n, d] in one memory whose tokens are `stride` elements apart."""
    memory = torch.empty(((n - 1) * stride + count * h * d,), dtype=dt, device=DEV)
    return [memory[i * h * d:].as_strided((1, h, n, d), (0, d, stride, 1)) for i in range(count)]


# 64 tokens a 64th of 2^31 bytes apart reach past it
@pytest.mark.parametrize("beyond", (False, True))
@pytest.mark.parametrize("far", ("states", "queries"))
@pytest.mark.parametrize("dtype,d,H,Hkv,Lq,S,lens", (
    (B.BF16, 64, 2, 1, 33, 70, None), (B.BF16, 128, 1, 1, 70, 66, [65]), (B.BF16, 128, 1, 1, 20, 64, None), (B.BF16, 72, 2, 2, 64, 41, [33]),
    (B.BF16, 256, 1, 1, 35, 40, None), (B.F32, 64, 1, 1, 40, 70, [66]), (B.F32, 128, 2, 1, 33, 32, None)))
def test_tokens_far_apart(dtype, d, H, Hkv, Lq, S, lens, far, beyond):
    s = B.CrossShape(1, H, Hkv, Lq, S, d, dtype)
    U.progress(f"far apart {s} {far} {beyond}")
    Q, K, V, dO, ok, valid = tensors(dict(shape=s, lens=lens, mask=False, lay="heads"), 51)
    dt = s.torch_dtype
    most = 0x7fffffff // (64 * dt.itemsize)
    stride = most + 1 if beyond else (most - d - 1) // 8 * 8
    if far == "states":
        Kf, Vf, dK, dV = apart(S, Hkv, d, stride, dt, 4)
        Qf, dOf, O, dQ = Q, dO, torch.empty_like(Q), torch.empty_like(Q)
        Kf.copy_(K), Vf.copy_(V)
    else:
        Qf, dOf, O, dQ = apart(Lq, H, d, stride, dt, 4)
        Kf, Vf, dK, dV = K, V, torch.empty_like(K), torch.empty_like(V)
        Qf.copy_(Q), dOf.copy_(dO)
    _, LSE = B.cross_attn_fwd(s, Qf, Kf, Vf, O=O, **valid)
    B.cross_attn_bwd(s, Qf, Kf, Vf, O, LSE, dOf, dQ=dQ, dK=dK, dV=dV, **valid)
    ref = reference(s, Q, K, V, ok, dO)
    for n, t in (("O", O), ("LSE", LSE), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        P.check(n, t, ref[n], P.U32 if n == "LSE" else P.HALF[dt])
