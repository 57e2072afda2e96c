"""The stream that the operators around the attention launch on is torch's current one, with and without torch's short cut to it."""
import pytest
import torch

from paper_2509_01085_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("short_cut", (True, False))
def test_calls_go_to_the_current_stream(short_cut, monkeypatch):
    if not short_cut:
        monkeypatch.setattr(B, "_raw_stream", None)
    device, side = torch.device("cuda:0"), torch.cuda.Stream()
    assert B._stream_of(device) == torch.cuda.current_stream().cuda_stream
    shp = B.Shape(1, 2, 1, 4, 8, 1, 1, 1, 64, B.BF16)
    x = torch.randn((1, shp.L, 2, 64), device=device).to(torch.bfloat16)
    want = B.qk_norm_rope_fwd(shp, None, None, x)[0]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        assert B._stream_of(device) == side.cuda_stream
        got = B.qk_norm_rope_fwd(shp, None, None, x)[0]
    side.synchronize()
    assert torch.equal(got, want)
