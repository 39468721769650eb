"""Gated linear attention on the GPU against the 64-bit plain form.

Bounds, per element, of the magnitude M of the value's terms (the plain form of absolute values):
  bf16 results: a rounding is off by 2^-8 of the value at most; the result's own and, on the tensor cores, one of the operand it is a sum
  over (P or the state; dS, P^T): 2 x 2^-8 M, and a little for what is below.
  fp32 results: sums of fewer than 2^9 terms, in two or three levels, 2^-24 each: 2^-15 M at most; two bf16 pieces leave out 2^-16 of an operand.
  dg is a sum of flows that cross a token, plus the difference of two sums over all pairs of the chunk, which are off by their own roundings:
  2^-15 of its magnitude and 2^-18 of the pairs'.
"""
import pytest
import torch

from tests import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def memory_given_back():
    """The large tensors' segments, which other tests' small ones would be put into."""
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def _ha():
    import paper_2609_32114_b200 as ha

    return ha


def inputs(T, HK, HV, D, dtype, B=1, cu=None, h0=True, shift=2.0, seed=0, unit=True):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    u = (lambda x: torch.nn.functional.normalize(x, dim=-1)) if unit else (lambda x: x)
    N = B if cu is None else len(cu) - 1
    t = dict(q=u(r(B, T, HK, D)).to(dtype), k=u(r(B, T, HK, D)).to(dtype), v=r(B, T, HV, D).to(dtype),
             g=-torch.nn.functional.softplus(r(B, T, HV) + shift), h0=0.5 * r(N, HV, D, D) if h0 else None)
    return t, r(B, T, HV, D).to(dtype), (0.5 * r(N, HV, D, D) if h0 else None)


def cuda(t):
    return {k: None if x is None else x.cuda() for k, x in t.items()} if isinstance(t, dict) else None if t is None else t.cuda()


def close(name, got, want, bound):
    """Within the bound everywhere; the largest excess in the message."""
    got = got.double().cpu()
    assert bool(torch.isfinite(got).all()), name
    off = (got - want).abs() - bound - 1e-30
    assert bool((off <= 0).all()), (name, float(off.max()), float((got - want).abs().max()), float(want.abs().max()))


def check(t, do, dhT, cu=None, scale=1.0, **kw):
    ha, D, HV, HK = _ha(), t["q"].shape[3], t["v"].shape[2], t["q"].shape[2]
    ct, cdo, cdh = cuda(t), cuda(do), cuda(dhT)
    dcu = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    rcu = None if cu is None else torch.tensor(cu)
    half = 2 ** -8 if t["q"].dtype == torch.bfloat16 else 2 ** -15
    o, hT, st, _ = ha.ha_la_gla_prefill(ct["q"], ct["k"], ct["v"], ct["g"], h0=ct["h0"], cu_seqlens=dcu, scale=scale, **kw)
    dq, dk, dv, dg, dh0, st2, _ = ha.ha_la_gla_backward(cdo, ct["q"], ct["k"], ct["v"], ct["g"], h0=ct["h0"], dhT=cdh, cu_seqlens=dcu, scale=scale, **kw)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and int(st2.item()) == 0
    ro, rh = ref.gla(**t, cu=rcu, scale=scale)
    mo, mh = ref.gla(**t, cu=rcu, scale=scale, magnitude=True)
    close("o", o, ro, 2.1 * half * mo)
    close("hT", hT, rh, 2 ** -15 * mh)
    r = ref.gla_backward(do, **t, dhT=dhT, cu=rcu, scale=scale)
    m = ref.gla_backward(do, **t, dhT=dhT, cu=rcu, scale=scale, magnitude=True)
    for name, got, a, b in zip(("dq", "dk"), (dq, dk), r[:2], m[:2]):
        close(name, got, ref.heads_sum(a, HK), 2.1 * half * ref.heads_sum(b, HK))
    close("dv", dv, r[2], 2.1 * half * m[2])
    close("dh0", dh0, r[4], 2 ** -15 * m[4])
    # all pairs that the token's chunk can have: what the outputs of 128 tokens around it are made of
    x = (t["q"].double().abs().repeat_interleave(HV // HK, 2) * m[0]).sum(-1).reshape(-1, HV)
    pairs = torch.stack([x[max(0, i - 127):i + 128].sum(0) for i in range(x.shape[0])]).reshape(m[3].shape) if x.shape[0] else m[3]
    close("dg", dg, r[3], 2 ** -15 * m[3] + 2 ** -18 * pairs)


LENGTHS = [1, 2, 63, 64, 65, 127, 128, 129, 200, 300]


@pytest.mark.parametrize("T", LENGTHS)
@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.float32, 128), (torch.bfloat16, 64), (torch.bfloat16, 128)],
                         ids=["fp32_64", "fp32_128", "bf16_64", "bf16_128"])
def test_lengths(T, dtype, D):
    check(*inputs(T, 1, 2, D, dtype, seed=T), scale=0.5 if T % 2 else 1.0)


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_128"])
@pytest.mark.parametrize("HK,HV,B,h0", [(1, 1, 1, False), (2, 2, 3, True), (1, 4, 2, True), (3, 6, 1, False)])
def test_heads_and_rows(HK, HV, B, h0, dtype, D):
    check(*inputs(150, HK, HV, D, dtype, B=B, h0=h0, seed=HV))


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_64", "bf16_128"])
@pytest.mark.parametrize("cu", [[0, 1], [0, 0, 5, 5], [0, 128, 256, 300], [0, 1, 2, 130, 130, 400], [0, 257, 258]])
def test_packed(cu, dtype, D):
    check(*inputs(cu[-1], 1, 2, D, dtype, cu=cu, seed=len(cu)), cu=cu, max_seqlen=max(b - a for a, b in zip(cu, cu[1:])))


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_128"])
@pytest.mark.parametrize("gates", ["none", "tiny", "closed", "mixed", "underflow"])
def test_gates(gates, dtype, D):
    """No decay at all, hardly any, exp(g) = 0 in one token, open and closed ones in turn, and sums that underflow."""
    t, do, dhT = inputs(260, 1, 2, D, dtype, seed=5)
    g = t["g"]
    if gates == "none":
        g.zero_()
    elif gates == "tiny":
        g.mul_(1e-4)
    elif gates == "closed":
        g[:, 70] = -1e4
        g[:, 130] = -1e30
    elif gates == "mixed":
        g[:, ::2] = 0
        g[:, 1::16] = -200
    else:
        g.fill_(-20.0)
    check(t, do, dhT)


def test_long_sums_keep_their_gates():
    """A cumulative gate of 1e3 and more with small steps behind it: what e^{G_i - G_j} is made of must not lose them."""
    t, do, dhT = inputs(256, 1, 1, 128, torch.bfloat16, seed=8)
    t["g"][:, :20] = -300.0
    t["g"][:, 20:] = -1e-3 * torch.rand(1, 236, 1)
    check(t, do, dhT)
    t, do, dhT = inputs(128, 1, 1, 64, torch.float32, seed=9)
    t["g"][:, :20] = -300.0
    t["g"][:, 20:] = -1e-3 * torch.rand(1, 108, 1)
    check(t, do, dhT)


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_128"])
def test_large_values(dtype, D):
    t, do, dhT = inputs(140, 1, 1, D, dtype, seed=3, unit=False)
    t["v"] *= 100
    check(t, do, dhT, scale=-3.0)


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_64", "bf16_128"])
def test_one_sequence_does_not_reach_another(dtype, D):
    """NaN and infinities in a sequence: the others' results are the same bits as without them."""
    ha, cu = _ha(), [0, 100, 230, 231, 400]
    t, do, dhT = inputs(400, 1, 2, D, dtype, cu=cu, seed=4)
    ct, cdo, cdh = cuda(t), cuda(do), cuda(dhT)
    dcu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    call = lambda: (*ha.ha_la_gla_prefill(**ct, cu_seqlens=dcu)[:2], *ha.ha_la_gla_backward(cdo, **ct, dhT=cdh, cu_seqlens=dcu)[:5])
    clean = [x.clone() for x in call()]
    for x, bad in ((ct["q"], float("nan")), (ct["k"], float("inf")), (ct["v"], float("nan")), (cdo, float("-inf")), (ct["g"], float("nan"))):
        x[:, 100:230] = bad
    ct["h0"][1] = float("nan")
    cdh[1] = float("inf")
    for a, b in zip(clean, call()):
        if a.shape[0] == 4:
            a, b = a[[0, 2, 3]], b[[0, 2, 3]]
        else:
            a, b = (torch.cat([x[:, :100], x[:, 230:]], 1) for x in (a, b))
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,D,T", [(torch.float32, 64, 0), (torch.bfloat16, 128, 0)], ids=["fp32_64", "bf16_128"])
def test_no_token(dtype, D, T):
    ha = _ha()
    t, do, dhT = inputs(0, 1, 2, D, dtype, B=2)
    ct = cuda(t)
    o, hT, st, _ = ha.ha_la_gla_prefill(**ct)
    assert o.numel() == 0 and torch.equal(hT, ct["h0"])
    assert torch.equal(ha.ha_la_gla_backward(cuda(do), **ct, dhT=cuda(dhT))[4], cuda(dhT))
    assert not ha.ha_la_gla_prefill(ct["q"], ct["k"], ct["v"], ct["g"])[1].any()
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    h0 = torch.randn(3, 2, D, D, device="cuda")
    one = {k: x[:1] for k, x in ct.items() if k != "h0"}
    o, hT, st, _ = ha.ha_la_gla_prefill(**one, h0=h0, cu_seqlens=cu)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and torch.equal(hT, h0)


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_128"])
def test_in_place_without_batch_and_given_outputs(dtype, D):
    ha = _ha()
    t, do, dhT = inputs(170, 1, 2, D, dtype, seed=6)
    ct, cdo, cdh = cuda(t), cuda(do), cuda(dhT)
    o, hT, _, ws = ha.ha_la_gla_prefill(**ct)
    back = ha.ha_la_gla_backward(cdo, **ct, dhT=cdh)
    h, dh = ct["h0"].clone(), cdh.clone()
    flat = {k: x[0] for k, x in ct.items() if k != "h0"}
    o2, h2, st, ws2 = ha.ha_la_gla_prefill(**flat, h0=h, hT=h, workspace=ws)
    assert h2 is h and ws2 is ws and torch.equal(o2, o[0]) and torch.equal(h, hT)
    outs = [torch.empty_like(x) for x in back[:4]]
    b2 = ha.ha_la_gla_backward(cdo, **ct, dhT=dh, dq=outs[0], dk=outs[1], dv=outs[2], dg=outs[3], dh0=dh)
    assert all(a is b for a, b in zip(b2[:4], outs)) and b2[4] is dh
    assert all(torch.equal(a, b) for a, b in zip(b2[:5], back[:5]))
    assert ha.ha_la_gla_prefill(**ct, want_hT=False)[1] is None and ha.ha_la_gla_backward(cdo, **ct, want_dh0=False)[4] is None
    b3 = ha.ha_la_gla_backward(cdo[0], **flat, h0=ct["h0"], dhT=cdh)
    assert all(torch.equal(a.flatten(), b.flatten()) for a, b in zip(b3[:5], back[:5]))


def test_lengths_that_do_not_fit_are_reported():
    ha = _ha()
    for dtype, D in ((torch.float32, 64), (torch.bfloat16, 128)):
        t, do, _ = inputs(100, 1, 1, D, dtype, h0=False)
        ct = cuda({k: x for k, x in t.items() if k != "h0"})
        for cu, most in (([0, 60, 40, 100], 0), ([0, 90, 101], 0), ([0, 50, 90], 0), ([1, 100], 0), ([0, 80, 100], 70), ([-5, 100], 0)):
            dcu = torch.tensor(cu, dtype=torch.int32, device="cuda")
            assert int(ha.ha_la_gla_prefill(**ct, cu_seqlens=dcu, max_seqlen=most)[2].item()) == 6, cu
            assert int(ha.ha_la_gla_backward(cuda(do), **ct, cu_seqlens=dcu, max_seqlen=most)[5].item()) == 6, cu


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_128"])
def test_captured_and_on_another_stream(dtype, D):
    """Replayed on new contents; on a named stream while the current one is busy; a workspace of its own to each of two graphs."""
    ha = _ha()
    t, do, dhT = inputs(300, 1, 2, D, dtype, seed=7)
    ct, cdo, cdh = cuda(t), cuda(do), cuda(dhT)
    call = lambda **kw: (*ha.ha_la_gla_prefill(**ct, **kw)[:2], *ha.ha_la_gla_backward(cdo, **ct, dhT=cdh, **kw)[:5])
    first = [x.clone() for x in call()]
    assert all(torch.equal(a, b) for a, b in zip(first, call()))
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            graphs.append((gr, call()))
            graphs[-1][1]
    for gr, outs in graphs:
        gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
    t2, do2, dhT2 = inputs(300, 1, 2, D, dtype, seed=70)
    for k, x in t2.items():
        ct[k].copy_(x)
    cdo.copy_(do2)
    cdh.copy_(dhT2)
    second = call()
    for gr, outs in graphs:
        gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for _, outs in graphs for a, b in zip(second, outs))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    there = call(stream=side.cuda_stream)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(second, there))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("N,HK,HV,D", [(1, 1, 1, 64), (1, 2, 2, 128), (5, 1, 4, 128), (37, 2, 2, 64), (0, 1, 1, 64)])
def test_decode(N, HK, HV, D, dtype):
    ha = _ha()
    t, _, _ = inputs(1, HK, HV, D, dtype, B=max(N, 1), seed=N)
    t = {k: x[:N] for k, x in t.items()}
    one = {k: x[:, 0].cuda() for k, x in t.items() if k != "h0"}
    h0 = t["h0"].cuda()
    o, h = ha.ha_la_gla_decode(**one, state=h0, scale=0.5, state_out=torch.empty_like(h0))
    torch.cuda.synchronize()
    ro, rh = ref.gla(**t, scale=0.5)
    mo, mh = ref.gla(**t, scale=0.5, magnitude=True)
    # fp32 sums of at most 128 terms in two levels, one rounding of the result
    close("o", o, ro[:, 0], (2 ** -19 + (2 ** -8 if dtype == torch.bfloat16 else 0)) * mo[:, 0])
    close("state", h, rh, 2 ** -21 * mh)
    keep = h0.clone()
    o2, h2 = ha.ha_la_gla_decode(**one, state=keep, scale=0.5)
    assert h2 is keep and torch.equal(h2, h) and torch.equal(o2, o)
    o3, h3 = ha.ha_la_gla_decode(**one, state=None)
    ro, rh = ref.gla(**{**t, "h0": None})
    close("fresh", h3, rh, 2 ** -21 * rh.abs())


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_128"])
def test_prefill_then_decode(dtype, D):
    """A prompt, then token by token: the same as one longer prompt."""
    ha = _ha()
    t, _, _ = inputs(135, 1, 2, D, dtype, B=2, seed=11)
    ct = cuda(t)
    part = {k: x[:, :131].contiguous() for k, x in ct.items() if k != "h0"}
    _, h, _, _ = ha.ha_la_gla_prefill(**part, h0=ct["h0"])
    ro, rh = ref.gla(**t)
    mo, mh = ref.gla(**t, magnitude=True)
    half = 2 ** -8 if dtype == torch.bfloat16 else 2 ** -15
    for i in range(131, 135):
        o, h = ha.ha_la_gla_decode(**{k: x[:, i].contiguous() for k, x in ct.items() if k != "h0"}, state=h)
        close("o", o, ro[:, i], 2.1 * half * mo[:, i])
    close("hT", h, rh, 2 ** -14 * mh)


def test_long_cache_of_offsets():
    """More than 2^31 elements of q, k, v and o: the last tokens of a long row against a call on a part of it."""
    ha = _ha()
    T, H, D = 140_000, 128, 128                            # 2.3e9 elements
    free = torch.cuda.mem_get_info()[0]
    if free < 120e9:
        pytest.skip("needs 120 GB")
    cu = torch.tensor([0, T - 300, T], dtype=torch.int32, device="cuda")
    x = torch.empty(1, T, H, D, dtype=torch.bfloat16, device="cuda").normal_()
    g = -torch.rand(1, T, H, device="cuda")
    o, hT, st, ws = ha.ha_la_gla_prefill(x, x, x, g, cu_seqlens=cu, scale=0.01)
    s = lambda t: t[:, T - 300:].contiguous()
    o2, hT2, _, _ = ha.ha_la_gla_prefill(s(x), s(x), s(x), s(g), scale=0.01)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and torch.equal(s(o), o2) and torch.equal(hT[1], hT2[0])
