"""The short convolution on the GPU against the 64-bit form.

Bounds, per element: one rounding r of the result (bf16 2^-8, fp32 2^-24).  The sums have five terms at the most, 2^-21 of their magnitudes M with what the
inputs' products round; the activation is off by 2^-20 of itself and passes that on with a slope of 1.1 at the most (2^-20 M).  Gradients: e = dy act'(s) is off by
2^-19 |dy| (1 + M), sums over tokens add 2^-24 for each of the tokens that a thread adds up, fewer than 512: 2^-15 of the terms' magnitudes in all."""
import pytest
import torch

from tests import mixer_reference as ref

pytestmark = pytest.mark.gpu
ROUND = {torch.bfloat16: 2 ** -8, torch.float32: 2 ** -24}
TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])


def _ha():
    import paper_2609_32114_b200 as ha

    return ha


def off(name, got, want, bound):
    got = got.double().cpu().reshape(want.shape)
    assert bool(torch.isfinite(got).all()), name
    d = (got - want).abs() - bound - 1e-37
    assert d.numel() == 0 or bool((d <= 0).all()), (name, float(d.max()), int(d.argmax()))


def inputs(B, T, C, K, dtype, cu=None, seed=0, bias=True, h0=True, pitch=0, lift=0):
    """x as rows of a tensor that is `pitch` channels wider and starts `lift` elements behind a boundary."""
    gen = torch.Generator().manual_seed(seed)
    N = B if cu is None else len(cu) - 1

    def rows(*shape):
        wide = torch.randn(B * T * (C + pitch) + lift, generator=gen).to(dtype).cuda()[lift:].view(B, T, C + pitch)
        return wide[..., :C]

    t = dict(x=rows(), dy=torch.randn(B, T, C, generator=gen).to(dtype).cuda(), w=(0.5 * torch.randn(C, K, generator=gen)).cuda(),
             bias=torch.randn(C, generator=gen).cuda() if bias else None, h0=torch.randn(N, K - 1, C, generator=gen).to(dtype).cuda() if h0 else None,
             dhT=torch.randn(N, K - 1, C, generator=gen).to(dtype).cuda() if h0 else None)
    t["cu"] = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    t["seqs"] = ref.spans(T, cu, B)
    return t


def check(t, act="silu", max_seqlen=0):
    ha, dtype, C = _ha(), t["x"].dtype, t["x"].shape[-1]
    kw = dict(bias=t["bias"], activation=act, h0=t["h0"], cu_seqlens=t["cu"], max_seqlen=max_seqlen)
    y, hT, status = ha.ha_la_conv(t["x"], t["w"], **kw)
    dx, dw, db, dh0, status2, _ = ha.ha_la_conv_backward(t["dy"], t["x"], t["w"], dhT=t["dhT"], **kw)
    again = ha.ha_la_conv_backward(t["dy"], t["x"], t["w"], dhT=t["dhT"], **kw)
    torch.cuda.synchronize()
    assert int(status) == 0 == int(status2)
    assert all(a is None or torch.equal(a, b) for a, b in zip((dx, dw, db, dh0), again))
    x, r = ref.d(t["x"]).reshape(-1, C), ROUND[dtype]
    want, last, mag = ref.conv(x, ref.d(t["w"]), ref.d(t["bias"]), ref.d(t["h0"]), act == "silu", t["seqs"])
    off("y", y, want, (r + 2 ** -20) * want.abs() + 2 ** -20 * mag)
    assert torch.equal(hT.double().cpu(), last)
    grads = ref.conv_grads(t["dy"].reshape(-1, C), x, t["w"], t["bias"], t["h0"], t["dhT"], act == "silu", t["seqs"])
    for name, got in (("dx", dx), ("dw", dw), ("dh0", dh0), ("db", db)):
        if got is None:
            assert name == "db" and t["bias"] is None
            continue
        g, m = grads[name]
        off(name, got, g, (r if name in ("dx", "dh0") else 2 ** -24) * g.abs() + 2 ** -15 * m)


@TYPES
@pytest.mark.parametrize("K", [2, 3, 4])
@pytest.mark.parametrize("T,C", [(1, 8), (2, 1), (3, 130), (9, 1024), (70, 515), (333, 72)])
def test_rows(T, C, K, dtype):
    check(inputs(2, T, C, K, dtype, seed=T + C))
    check(inputs(1, T, C, K, dtype, seed=T, bias=False, h0=False), act=None)


@TYPES
@pytest.mark.parametrize("cu", [[0, 1, 2, 3, 5, 8, 8, 40, 41], [0, 0, 77], [0, 300, 300], [0, 5, 5, 5, 6, 200, 202]], ids=str)
def test_packed(cu, dtype):
    for K in (2, 4):
        check(inputs(1, cu[-1], 264, K, dtype, cu=cu, seed=cu[-1]))
        check(inputs(1, cu[-1], 33, K, dtype, cu=cu, seed=cu[1], h0=False), act=None, max_seqlen=max(b - a for a, b in zip(cu, cu[1:])))


@TYPES
@pytest.mark.parametrize("pitch,lift", [(8, 0), (3, 0), (0, 1), (64, 8), (5, 2)])
def test_rows_of_a_wider_tensor(pitch, lift, dtype):
    check(inputs(1, 45, 264, 4, dtype, pitch=pitch, lift=lift, seed=pitch))
    check(inputs(3, 20, 264, 3, dtype, pitch=pitch, lift=lift, seed=lift))


@TYPES
def test_many_tokens(dtype):
    """Runs of the largest length, several CTAs to a sequence."""
    check(inputs(1, 3000, 24, 4, dtype, cu=[0, 1290, 1291, 3000], seed=3))


@TYPES
@pytest.mark.parametrize("N,C,K", [(1, 8, 4), (3, 515, 4), (200, 128, 2), (7, 1030, 3)])
def test_tokens_one_by_one(N, C, K, dtype):
    """From a state in place, against the same tokens as rows."""
    ha = _ha()
    t = inputs(N, 6, C, K, dtype, seed=N)
    kw = dict(bias=t["bias"])
    want, last, _ = ha.ha_la_conv(t["x"], t["w"], h0=t["h0"], **kw)
    state = t["h0"].clone()
    for i in range(6):
        y, new = ha.ha_la_conv_decode(t["x"][:, i], t["w"], state, **kw)
        assert new is state and torch.equal(y, want[:, i])
    assert torch.equal(state, last)
    y, new = ha.ha_la_conv_decode(t["x"][:, 0], t["w"], None, state_out=torch.empty_like(state), **kw)
    first, _, _ = ha.ha_la_conv(t["x"][:, :1].contiguous(), t["w"], **kw)
    assert torch.equal(y, first[:, 0])


@TYPES
def test_what_one_sequence_holds_stays_there(dtype):
    ha = _ha()
    cu = [0, 30, 31, 64]
    t = inputs(1, 64, 136, 4, dtype, cu=cu, seed=5)
    kw = dict(bias=t["bias"], h0=t["h0"], cu_seqlens=t["cu"])
    want = ha.ha_la_conv(t["x"], t["w"], **kw)[:2]
    wback = ha.ha_la_conv_backward(t["dy"], t["x"], t["w"], dhT=t["dhT"], **kw)
    for bad in (float("nan"), float("inf")):
        x, dy, h0, dhT = t["x"].clone(), t["dy"].clone(), t["h0"].clone(), t["dhT"].clone()
        x[:, 30:31], dy[:, 30:31], h0[1], dhT[1] = bad, bad, bad, bad
        got = ha.ha_la_conv(x, t["w"], **dict(kw, h0=h0))
        back = ha.ha_la_conv_backward(dy, x, t["w"], dhT=dhT, **dict(kw, h0=h0))
        keep = [i for i in range(64) if i != 30]
        assert torch.equal(got[0][:, keep], want[0][:, keep]) and torch.equal(got[1][[0, 2]], want[1][[0, 2]])
        assert torch.equal(back[0][:, keep], wback[0][:, keep]) and torch.equal(back[3][[0, 2]], wback[3][[0, 2]])


@TYPES
def test_no_token(dtype):
    ha = _ha()
    w, h0 = torch.ones(40, 4, device="cuda"), torch.randn(2, 3, 40, device="cuda").to(dtype)
    x = torch.empty(2, 0, 40, dtype=dtype, device="cuda")
    y, hT, status = ha.ha_la_conv(x, w, h0=h0)
    dx, dw, db, dh0, _, _ = ha.ha_la_conv_backward(x, x, w, h0=h0, dhT=h0, dw=torch.full((40, 4), 7.0, device="cuda"))
    assert y.shape == x.shape and torch.equal(hT, h0) and torch.equal(dh0, h0) and not dw.any() and int(status) == 0
    y, st = ha.ha_la_conv_decode(x[:, 0:0].reshape(0, 40), w, None)
    assert y.shape == (0, 40) and st.shape == (0, 3, 40)


def test_lengths_that_do_not_fit_are_reported():
    ha = _ha()
    x, w = torch.randn(1, 50, 64, device="cuda").bfloat16(), torch.ones(64, 4, device="cuda")
    for cu, most in (([0, 20, 49], 0), ([1, 20, 50], 0), ([0, 30, 20, 50], 0), ([0, 20, 50], 25), ([0, -5, 50], 0), ([0, 2 ** 31 - 1, 50], 0)):
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        assert int(ha.ha_la_conv(x, w, cu_seqlens=c, max_seqlen=most)[2]) == 6, cu
        assert int(ha.ha_la_conv_backward(x, x, w, cu_seqlens=c, max_seqlen=most)[4]) == 6, cu


def test_in_place_is_refused_for_prompts():
    ha = _ha()
    x, w, h = torch.randn(1, 50, 64, device="cuda"), torch.ones(64, 4, device="cuda"), torch.zeros(1, 3, 64, device="cuda")
    with pytest.raises(ha.HaLaError):
        ha.ha_la_conv(x, w, h0=h, hT=h)


def test_long_offsets():
    """More than 2^31 elements: the last rows against a call on them alone."""
    ha, T, C = _ha(), 300_000, 8192
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB")
    x = torch.empty(1, T, C, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.randn(C, 4, device="cuda")
    cu = torch.tensor([0, T - 100, T], dtype=torch.int32, device="cuda")
    y, hT, _ = ha.ha_la_conv(x, w, cu_seqlens=cu)
    tail = x[:, T - 100:].contiguous()
    want = ha.ha_la_conv(tail, w)
    assert torch.equal(y[:, T - 100:], want[0]) and torch.equal(hT[1], want[1][0])
    del y
    dx, *_ = ha.ha_la_conv_backward(x, x, w, cu_seqlens=cu)
    assert torch.equal(dx[:, T - 100:], ha.ha_la_conv_backward(tail, tail, w)[0])
    del dx, x
    torch.cuda.empty_cache()
