"""Cross attention where a workgroup's share of the key tiles has pieces of several units, among them whole units of few keys behind
longer ones: a padded batch of prompts."""
import pytest
import torch

from paper_2509_01085_amd import binding as B

import gpu_util as U
import plain_ops as P
from test_gpu_cross_attn import tensors

pytestmark = pytest.mark.gpu

# Two tiles of 64 keys: lengths of 65 to 128.  The walks of the units before them end in the tile place that the second one arrives in.
SHORT_UNITS = {  # shape, lengths
    "one_short_prompt": (B.CrossShape(2, 12, 12, 1000, 4096, 128, B.BF16), (4096, 100)),
    "seven_short_prompts_and_wavefronts_without_rows": (B.CrossShape(8, 12, 12, 416, 4096, 128, B.BF16), (4096,) + (100,) * 7),
    "one_wavefront_with_rows": (B.CrossShape(3, 40, 40, 32, 4000, 128, B.BF16), (4000, 100, 100)),
    "all_short_d64": (B.CrossShape(16, 40, 40, 32, 1088, 64, B.BF16), (1088, 65) + (100,) * 14),
    "shared_heads_d96": (B.CrossShape(4, 12, 3, 500, 2500, 96, B.BF16), (90, 2500, 128, 65)),
    "d64": (B.CrossShape(5, 24, 24, 130, 3000, 64, B.BF16), (128, 128, 3000, 70, 65)),
}


@pytest.mark.parametrize("name", list(SHORT_UNITS))
def test_short_units_behind_others(name):
    s, lens = SHORT_UNITS[name]
    U.progress(f"cross attention in shares, {name}")
    Q, K, V, dO, ok, valid = tensors(dict(shape=s, lens=list(lens), mask=False, lay="heads"), 41)
    O, LSE = B.cross_attn_fwd(s, Q, K, V, **valid)
    grads = B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, **valid)
    again = B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, **valid)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    f = lambda t: t.double().cpu()  # noqa: E731
    for b, n in enumerate(lens):  # the valid states alone: an entry's reference is as long as they are
        ref = P.cross(f(Q[b:b + 1]), f(K[b:b + 1, :, :n]), f(V[b:b + 1, :, :n]), ok[b:b + 1, :n], P.default_scale(s.d), f(dO[b:b + 1]), P.HALF[torch.bfloat16])
        for what, t in (("O", O), ("LSE", LSE), ("dQ", grads[0]), ("dK", grads[1][:, :, :n]), ("dV", grads[2][:, :, :n])):
            P.check(f"{what} of entry {b}", t[b:b + 1], ref[what], P.U32 if what == "LSE" else P.HALF[torch.bfloat16])
        assert (grads[1][b, :, n:] == 0).all() and (grads[2][b, :, n:] == 0).all()
