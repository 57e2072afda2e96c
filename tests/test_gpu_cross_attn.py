"""Cross attention, forward and backward, against the plain 64-bit form."""
import pytest
import torch

from paper_2509_01085_amd import binding as B

import gpu_util as U
import plain_ops as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


def case(dtype, B_, H, Hkv, Lq, S, d, lens=None, mask=False, lay="heads"):
    return dict(shape=B.CrossShape(B_, H, Hkv, Lq, S, d, dtype), lens=lens, mask=mask, lay=lay)


F, H16 = B.F32, B.BF16
CASES = {
    "one_of_each": case(H16, 1, 1, 1, 1, 1, 64),
    "one_of_each_f32": case(F, 1, 1, 1, 1, 1, 8),
    "one_key_of_many": case(H16, 2, 2, 2, 40, 70, 64, [1, 70]),
    "tile": case(H16, 1, 2, 2, 32, 64, 64),
    "tile_and_one": case(H16, 1, 2, 1, 33, 65, 64),
    "tile_less_one": case(F, 1, 2, 1, 127, 31, 64),
    "two_tiles": case(H16, 2, 3, 3, 129, 128, 128, [128, 65]),
    "three_tiles": case(H16, 2, 2, 2, 200, 129, 128, [129, 128]),
    "d8": case(H16, 1, 2, 2, 50, 40, 8),
    "d24_f32": case(F, 2, 2, 1, 45, 70, 24, [70, 33], True),
    "d72": case(H16, 3, 6, 2, 191, 257, 72, [257, 100, 199], True, "tokens"),
    "d72_f32": case(F, 2, 4, 2, 91, 157, 72, [157, 100], True, "tokens"),
    "d80": case(H16, 2, 40, 5, 3, 19, 80, [19, 0], False, "tokens"),
    "d96": case(H16, 1, 3, 3, 300, 77, 96, None, True, "packed"),
    "d128": case(H16, 1, 3, 3, 515, 333, 128, None, False, "packed"),
    "d128_f32": case(F, 1, 2, 2, 300, 161, 128, None, True, "packed"),
    "d160": case(H16, 2, 2, 1, 100, 150, 160, [150, 149]),
    "d256": case(H16, 1, 2, 2, 140, 200, 256, None, True),
    "d256_f32": case(F, 1, 2, 2, 70, 90, 256, [65], False, "tokens"),
    "empty": case(H16, 3, 2, 2, 70, 90, 64, [0, 90, 0]),
    "empty_f32": case(F, 2, 2, 1, 70, 90, 128, [0, 55], True),
    "token_serving": case(H16, 3, 8, 2, 1, 1500, 128, [1500, 1, 700], False, "tokens"),
    "token_serving_d64": case(H16, 2, 12, 12, 1, 2111, 64, [2111, 2000]),
    "token_serving_f32": case(F, 2, 8, 1, 1, 700, 64, [700, 3]),
    "tokens_long": case(H16, 1, 4, 1, 7, 9001, 128, None, True),
    "group_crosses_tiles": case(H16, 1, 6, 2, 45, 130, 64, [130], False, "tokens"),
    "long_queries": case(H16, 1, 1, 1, 9000, 100, 128),
    "long_queries_d64": case(H16, 1, 2, 1, 5003, 300, 64, [299], False, "tokens"),
    "whole_tiles": case(H16, 2, 2, 2, 512, 512, 128, [512, 320]),
    "whole_tiles_d64": case(H16, 1, 2, 2, 512, 256, 64),
}


def tensors(c, seed, dO_lay=None):
    s = c["shape"]
    gen = torch.Generator().manual_seed(seed)

    def mk(h, n, lay, gain=1.0):
        if lay == "tokens":
            return (torch.randn((s.B, n, h, s.d), generator=gen) * gain).to(s.torch_dtype).to(DEV).transpose(1, 2)
        return (torch.randn((s.B, h, n, s.d), generator=gen) * gain).to(s.torch_dtype).to(DEV)

    lay = c["lay"]
    Q = mk(s.H, s.Lq, lay)
    if lay == "packed":  # keys and values of one projection
        KV = (torch.randn((s.B, s.S, 2, s.Hkv, s.d), generator=gen) * 1.5).to(s.torch_dtype).to(DEV)
        K, V = KV[:, :, 0].transpose(1, 2), KV[:, :, 1].transpose(1, 2)
    else:
        K, V = mk(s.Hkv, s.S, lay, 1.5), mk(s.Hkv, s.S, lay)
    dO = mk(s.H, s.Lq, dO_lay or lay)
    kv_len = torch.tensor(c["lens"], dtype=torch.int32) if c["lens"] else None
    kv_mask = None
    if c["mask"]:
        kv_mask = (torch.rand((s.B, s.S), generator=gen) < 0.7).to(torch.uint8) * 3
        kv_mask[:, 0] = 1
    ok = P.valid_states(s.B, s.S, kv_len, kv_mask)
    for t in (K, V):  # nobody wrote there
        t.masked_fill_(~ok.to(DEV)[:, None, :, None], NAN)
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    return Q, K, V, dO, ok, dict(kv_len=dev(kv_len), kv_mask=dev(kv_mask))


def reference(s, Q, K, V, ok, dO=None, O_used=None, scale=None):
    f = lambda t: None if t is None else t.double().cpu()  # noqa: E731
    return P.cross(f(Q), f(K), f(V), ok, scale or P.default_scale(s.d), f(dO), P.HALF[s.torch_dtype], f(O_used))


@pytest.mark.parametrize("name", list(CASES))
def test_against_the_plain_form(name):
    c = CASES[name]
    s = c["shape"]
    U.progress(f"cross attention {name}")
    Q, K, V, dO, ok, valid = tensors(c, sum(map(ord, name)))
    half = P.HALF[s.torch_dtype]
    O, LSE = B.cross_attn_fwd(s, Q, K, V, **valid)
    dQ, dK, dV = B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, **valid)
    torch.cuda.synchronize()
    ref = reference(s, Q, K, V, ok, dO)
    rms = {n: P.check(n, t, ref[n], P.U32 if n == "LSE" else half) for n, t in (("O", O), ("LSE", LSE), ("dQ", dQ), ("dK", dK), ("dV", dV))}
    U.progress(f"  rms {rms}")
    if s.dtype == B.BF16 and ok.sum(1).min() >= 16 and s.Lq * s.H // s.Hkv >= 16:
        # two to four independent roundings of at most half a step, rms 2^-8 / sqrt(3) / sqrt(2) of a value anywhere in its binade
        assert max(v for n, v in rms.items() if n != "LSE") < 5e-3, rms


@pytest.mark.parametrize("dtype", (H16, F))
def test_strides_outputs_within_larger_tensors_and_gradients_of_repetitions(dtype):
    s = B.CrossShape(2, 4, 2, 50, 70, 64, dtype)
    c = dict(shape=s, lens=[70, 41], mask=False, lay="heads")
    Q, K, V, dO, ok, valid = tensors(c, 11, "tokens")
    K, V = K[:1].expand(2, -1, -1, -1), V[:1].expand(2, -1, -1, -1)  # one prompt for both
    dt = s.torch_dtype
    wide = lambda h, n: torch.full((2, n + 3, h + 1, s.d + 16), 7.0, dtype=dt, device=DEV)  # noqa: E731
    inner = lambda t, h, n: t[:, 2:2 + n, :h, 8:8 + s.d].transpose(1, 2)  # noqa: E731
    Ow, dQw, dKw, dVw = wide(4, 50), wide(4, 50), wide(2, 70), wide(2, 70)
    O, dQ, dK, dV = inner(Ow, 4, 50), inner(dQw, 4, 50), inner(dKw, 2, 70), inner(dVw, 2, 70)
    _, LSE = B.cross_attn_fwd(s, Q, K, V, O=O, **valid)
    B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, dQ=dQ, dK=dK, dV=dV, **valid)
    ref = reference(s, Q, K, V, ok, dO)
    for n, t in (("O", O), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        P.check(n, t, ref[n], P.HALF[dt])
    for t, h, n in ((Ow, 4, 50), (dQw, 4, 50), (dKw, 2, 70), (dVw, 2, 70)):
        inner(t, h, n).fill_(7.0)
        assert (t == 7.0).all()  # nothing else was written
    got = B.cross_attn_bwd(s, Q, K, V, O.copy_(ref["O"][0].to(dt)), LSE, dO, **valid)  # memory for the gradients from the binding
    for n, t in zip(("dQ", "dK", "dV"), got):
        P.check(n, t, ref[n], P.HALF[dt])


def test_a_length_outside_its_range_is_taken_as_the_nearest():
    s = B.CrossShape(3, 2, 2, 40, 50, 64, H16)
    Q, K, V, dO, ok, _ = tensors(dict(shape=s, lens=None, mask=False, lay="heads"), 12)
    odd = torch.tensor([-5, 51, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    plain = torch.tensor([0, 50, 50], dtype=torch.int32, device=DEV)
    for a, b in zip(B.cross_attn_fwd(s, Q, K, V, kv_len=odd), B.cross_attn_fwd(s, Q, K, V, kv_len=plain)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", (H16, F))
@pytest.mark.parametrize("S", (40, 300, 3000))
def test_lengths_and_masks_say_the_same(dtype, S):
    """(Not bit for bit: where the walk over the keys is cut goes by the lengths, and with it the order of the sums.)"""
    s = B.CrossShape(2, 2, 1, 37, S, 64, dtype)
    Q, K, V, dO, ok, valid = tensors(dict(shape=s, lens=[S - 3, S // 2], mask=False, lay="heads"), 13)
    ref = reference(s, Q, K, V, ok, dO)
    for how in (valid, dict(kv_mask=ok.to(DEV)), dict(valid, kv_mask=torch.ones_like(ok).to(DEV))):
        O, LSE = B.cross_attn_fwd(s, Q, K, V, **how)
        for n, t in zip(("O", "LSE", "dQ", "dK", "dV"), (O, LSE, *B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, **how))):
            P.check(n, t, ref[n], P.U32 if n == "LSE" else P.HALF[s.torch_dtype])


@pytest.mark.parametrize("dtype", (H16, F))
def test_large_logits_and_infinities(dtype):
    s = B.CrossShape(1, 1, 1, 40, 100, 64, dtype)
    Q, K, V, dO, ok, _ = tensors(dict(shape=s, lens=None, mask=False, lay="heads"), 14)
    Q.mul_(30)
    O, LSE = B.cross_attn_fwd(s, Q, K, V)
    ref = reference(s, Q, K, V, ok)
    P.check("O", O, ref["O"], P.HALF[s.torch_dtype])
    P.check("LSE", LSE, ref["LSE"], P.U32)
    # a valid key whose logits are -inf weighs nothing; where all are, a row has no softmax
    Q.fill_(1.0)
    K[0, 0, 5] = float("-inf")
    O, LSE = B.cross_attn_fwd(s, Q, K, V)
    keep = ok.clone()
    keep[0, 5] = False
    O1, LSE1 = B.cross_attn_fwd(s, Q, K, V, kv_mask=keep.to(DEV))
    assert torch.equal(O, O1) and torch.equal(LSE, LSE1)
    K.fill_(float("-inf"))
    O, LSE = B.cross_attn_fwd(s, Q, K, V)
    assert torch.isnan(O).all() and (LSE == float("-inf")).all()
    # NaN in a valid key spreads to all rows of its head, NaN in a query stays in its row
    K.normal_()
    Q.normal_()
    Q[0, 0, 3, 7] = NAN
    O, LSE = B.cross_attn_fwd(s, Q, K, V)
    bad = torch.isnan(O).all(-1)[0, 0]
    assert bad[3] and int(bad.sum()) == 1 and torch.isnan(LSE[0, 0, 3])
    K[0, 0, 99, 0] = NAN
    assert torch.isnan(B.cross_attn_fwd(s, Q, K, V)[0]).all()


@pytest.mark.parametrize("Lq,S", ((1, 3000), (70, 100), (600, 100), (3000, 600)))
def test_a_large_scale_a_small_one_and_the_same_bits_twice(Lq, S):
    s = B.CrossShape(1, 2, 2, Lq, S, 64, H16)
    Q, K, V, dO, ok, _ = tensors(dict(shape=s, lens=None, mask=False, lay="heads"), 15)
    for scale in (1e-4, 0.7):
        O, LSE = B.cross_attn_fwd(s, Q, K, V, sm_scale=scale)
        ref = reference(s, Q, K, V, ok, dO, scale=scale)
        P.check("O", O, ref["O"], P.HALF[s.torch_dtype])
        P.check("LSE", LSE, ref["LSE"], P.U32)
        first = (O, LSE, *B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, sm_scale=scale))
        for n, t in zip(("dQ", "dK", "dV"), first[2:]):
            P.check(n, t, ref[n], P.HALF[s.torch_dtype])
        O2, LSE2 = B.cross_attn_fwd(s, Q, K, V, sm_scale=scale)
        again = (O2, LSE2, *B.cross_attn_bwd(s, Q, K, V, O2, LSE2, dO, sm_scale=scale))
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_offsets_past_32_bits():
    """States 2^16 elements apart, 70,000 of them: the last ones lie beyond 2^32 elements."""
    s = B.CrossShape(1, 1, 1, 3, 70000, 64, H16)
    Q, K, V, dO, ok, _ = tensors(dict(shape=s, lens=None, mask=False, lay="heads"), 16)
    big = torch.empty((1, 1, s.S, 1 << 16), dtype=torch.bfloat16, device=DEV)
    Kb, Vb, dKb, dVb = (big[..., 64 * i:64 * i + 64] for i in range(4))
    Kb.copy_(K)
    Vb.copy_(V)
    a, b = B.cross_attn_fwd(s, Q, K, V), B.cross_attn_fwd(s, Q, Kb, Vb)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    x = B.cross_attn_bwd(s, Q, K, V, *a, dO)
    y = B.cross_attn_bwd(s, Q, Kb, Vb, *a, dO, dK=dKb, dV=dVb)
    assert all(torch.equal(p, q) for p, q in zip(x, y))


@pytest.mark.parametrize("name", ("d72", "token_serving", "whole_tiles", "d72_f32"))
def test_replayed_and_on_other_streams(name):
    c = CASES[name]
    s = c["shape"]
    Q, K, V, dO, ok, valid = tensors(c, 17)
    O, LSE = torch.empty_like(Q), torch.empty((s.B, s.H, s.Lq), device=DEV)
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
    ws = [torch.empty(max(1, n), dtype=torch.uint8, device=DEV) for n in (B.cross_fwd_workspace_bytes(s), B.cross_bwd_workspace_bytes(s))]

    def step():
        B.cross_attn_fwd(s, Q, K, V, O=O, LSE=LSE, workspace=ws[0], **valid)
        B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, dQ=dQ, dK=dK, dV=dV, workspace=ws[1], **valid)

    step()
    torch.cuda.synchronize()
    outs = (O, LSE, dQ, dK, dV)
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for k in range(3):
        for t in outs:
            t.fill_(NAN)
        for w in ws:
            w.fill_(255)  # nothing is kept there
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), f"replay {k}"
        for t in outs:
            t.fill_(NAN)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), f"stream {k}"


@pytest.mark.parametrize("dtype", (H16, F))
@pytest.mark.parametrize("Lq,S", ((1, 900), (40, 100), (300, 300)))
def test_a_mask_that_leaves_nothing_of_an_entry_or_of_a_tile(Lq, S, dtype):
    s = B.CrossShape(4, 4, 2, Lq, S, 64, dtype)
    Q, K, V, dO, _, _ = tensors(dict(shape=s, lens=None, mask=False, lay="heads"), 31)
    mask = torch.ones((4, S), dtype=torch.bool)
    mask[0] = False          # nothing, and no length says so
    mask[1, :70] = False     # not the first tile
    mask[2, 1:] = False      # one state
    lens = torch.tensor([S, S, S, 64], dtype=torch.int32)
    mask[3, :64] = False     # nothing up to the length
    ok = P.valid_states(4, S, lens, mask)
    for t in (K, V):
        t.masked_fill_(~ok.to(DEV)[:, None, :, None], NAN)
    valid = dict(kv_len=lens.to(DEV), kv_mask=mask.to(DEV))
    O, LSE = B.cross_attn_fwd(s, Q, K, V, **valid)
    grads = B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, **valid)
    ref = reference(s, Q, K, V, ok, dO)
    for n, t in zip(("O", "LSE", "dQ", "dK", "dV"), (O, LSE, *grads)):
        P.check(n, t, ref[n], P.U32 if n == "LSE" else P.HALF[s.torch_dtype])
    assert (O[0] == 0).all() and (O[3] == 0).all() and torch.isneginf(LSE[0]).all() and all((g[0] == 0).all() for g in grads)


@pytest.mark.parametrize("dtype", (H16, F))
@pytest.mark.parametrize("Lq,S,d", ((1, 500, 128), (35, 70, 64), (150, 33, 40), (5, 90, 256)))
def test_more_entries_than_a_wavefront_has_lanes(Lq, S, d, dtype):
    s = B.CrossShape(131, 2, 1, Lq, S, d, dtype)
    gen = torch.Generator().manual_seed(S)
    lens = torch.randint(0, S + 1, (131,), generator=gen)
    lens[60:70] = 0
    c = dict(shape=s, lens=lens.tolist(), mask=False, lay="heads")
    Q, K, V, dO, ok, valid = tensors(c, S)
    O, LSE = B.cross_attn_fwd(s, Q, K, V, **valid)
    grads = B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, **valid)
    ref = reference(s, Q, K, V, ok, dO)
    for n, t in zip(("O", "LSE", "dQ", "dK", "dV"), (O, LSE, *grads)):
        P.check(n, t, ref[n], P.U32 if n == "LSE" else P.HALF[s.torch_dtype])


@pytest.mark.parametrize("dtype", (H16, F))
@pytest.mark.parametrize("B_,H,Lq,S,d", ((1, 4, 700, 200, 64), (2, 8, 500, 300, 256), (1, 3, 64, 1500, 128), (2, 2, 40, 700, 96)))
def test_workspaces_of_the_size_that_is_asked_for_are_not_exceeded(B_, H, Lq, S, d, dtype):
    s = B.CrossShape(B_, H, H, Lq, S, d, dtype)
    for lens in (None, [S // 2 + 1] * B_):
        Q, K, V, dO, ok, valid = tensors(dict(shape=s, lens=lens, mask=False, lay="heads"), 5)
        wide = lambda n: torch.full((n + 4096,), 0x5a, dtype=torch.uint8, device=DEV)  # noqa: E731
        nf, nb = B.cross_fwd_workspace_bytes(s), B.cross_bwd_workspace_bytes(s)
        wf, wb = wide(nf), wide(nb)
        O, LSE = B.cross_attn_fwd(s, Q, K, V, workspace=wf[:nf], **valid)
        grads = B.cross_attn_bwd(s, Q, K, V, O, LSE, dO, workspace=wb[:nb], **valid)
        assert (wf[nf:] == 0x5a).all() and (wb[nb:] == 0x5a).all()
        ref = reference(s, Q, K, V, ok, dO)
        for n, t in zip(("O", "dQ", "dK", "dV"), (O, *grads)):
            P.check(n, t, ref[n], P.HALF[s.torch_dtype])
