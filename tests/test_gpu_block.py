"""The attention part of a transformer block as bench.py runs it: norm and rotation into block-major order, selection and sparse
attention, cross attention, and all of it backward."""
import numpy as np
import pytest
import torch

from bsa_workloads import WORKLOADS, Workload
from oracle import bsa_oracle as o
from paper_2509_01085_amd import binding as B

import bench
import gpu_util as U
import plain_ops as P

pytestmark = pytest.mark.gpu

CASES = {
    "tiny": (WORKLOADS["tiny"].replace(threshold=0.6), 77, [50]),
    "ragged_f32": (Workload("ragged_f32", 2, 2, 72, "fp32", (6, 6, 10), (3, 2, 5), threshold=0.7, keep_ratio=0.4), 130, [130, 0]),
    "mini_wan": (Workload("mini_wan", 1, 2, 128, "bf16", (8, 8, 12), (4, 4, 4), threshold=0.6), 512, None),
    "ragged_bf16": (Workload("ragged_bf16", 2, 2, 64, "bf16", (4, 8, 16), (2, 4, 4), threshold=0.7, keep_ratio=0.3), 257, [257, 31]),
}
RESULTS = ("Q", "K", "V", "O", "LSE", "Oc", "LSEc", "dXc", "dKV", "dQ", "dK", "dV", "dX", "dwq", "dwk")


def block_of(name):
    wl, states, lens = CASES[name]
    return bench.BlockAttention(wl, states, torch, B, kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda") if lens else None)


@pytest.mark.parametrize("name", list(CASES))
def test_every_stage_against_its_plain_form(name):
    U.progress(f"block {name}")
    b = block_of(name)
    b.step()
    torch.cuda.synchronize()
    wl, shp = b.wl, b.shape
    half = P.HALF[shp.torch_dtype]
    f = lambda t: t.double().cpu()  # noqa: E731
    # norm and rotation of what the projection gave, and back from the gradients that the sparse attention left
    for i, (Y, w, dY, dw) in enumerate(((b.Q, b.wq, b.dQ, b.dwq), (b.K, b.wk, b.dK, b.dwk))):
        ref = P.norm_rope(shp, b.rope, f(b.X[:, :, i]), f(w), b.EPS, dY=f(dY))
        P.check("Y", Y, ref["Y"], half)
        P.check("dX", b.dX[:, :, i], ref["dX"], half)
        P.check("dw", dw, ref["dw"], P.U32)
    order = P.row_order(shp)
    assert torch.equal(b.V.cpu(), b.X[:, :, 2].cpu()[:, order].transpose(1, 2))
    assert torch.equal(b.dX[:, :, 2].cpu()[:, order].transpose(1, 2), b.dV.cpu())
    # sparse attention on the rotated queries and keys
    host, part = U.lists_to_host(shp, b.lists), U.part_of(wl)
    for bb in range(wl.B):
        for h in range(wl.H):
            Q, K, V, dO = (U.host_f64(t[bb, h]) for t in (b.Q, b.K, b.V, b.dO))
            ix, O, LSE, dQ, dK, dV = o.bsa_head(Q, K, V, dO, part, wl.threshold, wl.keep_ratio)
            assert np.array_equal(b.keep[bb, h].cpu().numpy(), ix.keep_idx)
            ptr, idx = U.head_csr(host, shp, bb, h)
            assert np.array_equal(ptr, ix.q2k_ptr) and np.array_equal(idx, ix.q2k_idx)
            pairs = [(n, U.host_f64(t[bb, h]), r) for n, t, r in (("O", b.O, O), ("dQ", b.dQ, dQ), ("dK", b.dK, dK), ("dV", b.dV, dV))]
            if wl.dtype == "fp32":
                U.check_tensors(f"block_{name}", f"b{bb}h{h}", "fp32", pairs, lse=(U.host_f64(b.LSE[bb, h]), LSE))
            else:  # bf16: the criterion in RMS, 5e-3
                for n, got, ref in pairs:
                    assert np.sqrt(np.mean((got - ref) ** 2) / np.mean(ref ** 2)) < 5e-3, n
    # cross attention
    ok = P.valid_states(wl.B, b.cross.S, None if b.kv_len is None else b.kv_len.cpu(), None)
    heads = lambda t: f(t).transpose(1, 2)  # noqa: E731
    ref = P.cross(heads(b.Xc), heads(b.KV[:, :, 0]), heads(b.KV[:, :, 1]), ok, P.default_scale(wl.d), heads(b.dOc), half)
    for n, t in (("O", b.Oc), ("dQ", b.dXc), ("dK", b.dKV[:, :, 0]), ("dV", b.dKV[:, :, 1])):
        P.check(n, t.transpose(1, 2), ref[n], half)
    P.check("LSE", b.LSEc, ref["LSE"], P.U32)


@pytest.mark.parametrize("name", ["ragged_f32", "mini_wan"])
def test_a_captured_block_replays_with_new_inputs(name):
    U.progress(f"block, captured {name}")
    b, other = block_of(name), block_of(name)
    b.step()
    other.step()
    torch.cuda.synchronize()
    graphs = []
    for x in (b, other):  # each graph has workspaces of its own
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            x.step()
    gen = torch.Generator(device="cuda").manual_seed(9)
    for turn in range(3):
        for x in (b, other):
            for t in (x.X, x.Xc, x.KV, x.dO, x.dOc):
                t.copy_(torch.randn(t.shape, generator=gen, device="cuda").to(t.dtype))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x in (b, other):
            got = {n: getattr(x, n).clone() for n in RESULTS}
            for n in RESULTS:
                getattr(x, n).zero_()
            x.step()
            torch.cuda.synchronize()
            for n in RESULTS:
                assert torch.equal(got[n], getattr(x, n)), (turn, n)


def test_the_command_reports_every_call(capsys, monkeypatch):
    import json
    import sys

    monkeypatch.setattr(sys, "argv", ["bench.py", "--block", "--workload", "tiny", "--steps", "2", "--warmup", "1", "--states", "33"])
    bench.main()
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert set(line["ms_per_call"]) == set(bench.BlockAttention.CALLS) and line["config"]["states"] == 33
    assert all(v > 0 for v in line["ms_per_call"].values()) and line["value"] > 0
