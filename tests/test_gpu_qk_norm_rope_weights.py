"""Norm and rotation, backward, for weights that need no gradient."""
import pytest
import torch

from paper_2509_01085_amd import binding as B

from test_gpu_qk_norm_rope import CASES, DEV, projection

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("weights", (True, False))
@pytest.mark.parametrize("name", ("block_major", "tiny_halves", "one_token"))
def test_gradients_of_weights_are_left_out(name, weights):
    shp, rope, lay = CASES[name]
    gen = torch.Generator().manual_seed(81)
    (Xq, Xk, _), _ = projection(shp, lay, gen)
    dY = [torch.randn((shp.B, shp.H, shp.L, shp.d), generator=gen).to(shp.torch_dtype).to(DEV) for _ in range(3)]
    wq, wk = (torch.rand(shp.d, generator=gen).to(DEV) if weights else None for _ in range(2))
    table = B.rope_table(shp, rope)
    run = lambda **kw: B.qk_norm_rope_bwd(shp, rope, table, Xq, Xk, *dY, wq=wq, wk=wk, **kw)  # noqa: E731
    every, some = run(), run(weight_grads=False)
    assert some[3] is None and some[4] is None
    assert all(torch.equal(a, b) for a, b in zip(every[:3], some[:3]))
    mine = torch.full((shp.d,), float("nan"), device=DEV)  # memory that is given asks for its own
    one = run(weight_grads=False, dwk=mine)
    assert one[3] is None and one[4] is mine and torch.equal(mine, every[4]) and torch.equal(one[0], every[0])


def test_without_them_no_sums_are_left():
    shp, rope, lay = CASES["block_major"]
    gen = torch.Generator().manual_seed(82)
    (Xq, Xk, _), _ = projection(shp, lay, gen)
    dY = [torch.randn((shp.B, shp.H, shp.L, shp.d), generator=gen).to(shp.torch_dtype).to(DEV) for _ in range(3)]
    table = B.rope_table(shp, rope)
    ws = torch.empty(B.qk_norm_rope_bwd_workspace_bytes(shp), dtype=torch.uint8, device=DEV)
    for weight_grads in (False, True):  # the workgroups' shares of them are all that the workspace holds
        ws.fill_(0x5a)
        B.qk_norm_rope_bwd(shp, rope, table, Xq, Xk, *dY, weight_grads=weight_grads, workspace=ws)
        assert bool((ws == 0x5a).all()) != weight_grads
