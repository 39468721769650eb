"""The selective scan on the GPU against the 64-bit form.

Bounds, per element: one rounding r of the result, and 2^-19 of what a relative error of one in every factor of every step comes to (mixer_reference): a step's decay is
off by 2^-22 (the exponential) and by 2^-20 of its exponent (delta by 2^-21, two roundings), delta x by 2^-21, sums of up to 64 states by 2^-21, gates by 2^-20.  Sums over
a group's channels or over tokens have up to a few hundred terms, added in parts of at most 64 in 32 bits: another 2^-18."""
import pytest
import torch

from tests import mixer_reference as ref
from tests.test_gpu_conv import ROUND, TYPES, off

pytestmark = pytest.mark.gpu


def _ha():
    import paper_2609_32114_b200 as ha

    return ha


def inputs(B, T, ch, S, G, dtype, cu=None, seed=0, D=True, z=True, bias=True, h0=True, pitch=0, strong=1.0):
    gen = torch.Generator().manual_seed(seed)
    N = B if cu is None else len(cu) - 1

    def rows(*inner, std=1.0):
        n = 1
        for i in inner:
            n *= i
        wide = (std * torch.randn(B, T, n + pitch, generator=gen)).to(dtype).cuda()
        return wide[..., :n].unflatten(-1, inner)

    f = lambda *s: torch.randn(*s, generator=gen).cuda()      # noqa: E731
    t = dict(x=rows(ch), dt=rows(ch), A=-strong * f(ch, S).abs(), B=rows(G, S), C=rows(G, S), D=f(ch) if D else None, z=rows(ch) if z else None,
             dt_bias=f(ch) - 2 if bias else None, h0=f(N, ch, S) if h0 else None, dhT=f(N, ch, S) if h0 else None)
    t["dy"] = torch.randn(B, T, ch, generator=gen).to(dtype).cuda()
    t["cu"] = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    t["seqs"] = ref.spans(T, cu, B)
    return t


def flat(t):
    return None if t is None else ref.d(t).reshape(-1, *t.shape[2:])


def check(t, softplus=True, back=True, max_seqlen=0):
    ha, r = _ha(), ROUND[t["x"].dtype]
    a = [t[k] for k in ("x", "dt", "A", "B", "C")]
    kw = dict(D=t["D"], z=t["z"], dt_bias=t["dt_bias"], softplus=softplus, cu_seqlens=t["cu"], max_seqlen=max_seqlen)
    y, hT, status, _ = ha.ha_la_scan(*a, h0=t["h0"], **kw)
    torch.cuda.synchronize()
    assert int(status) == 0
    args = (flat(t["x"]), flat(t["dt"]), ref.d(t["A"]), flat(t["B"]), flat(t["C"]), ref.d(t["D"]), flat(t["z"]), ref.d(t["dt_bias"]), softplus)
    want, last, e, elast = ref.scan(*args, ref.d(t["h0"]), t["seqs"])
    off("y", y, want, r * want.abs() + 2 ** -19 * e)
    off("hT", hT, last, 2 ** -19 * elast)
    if t["h0"] is not None:                                  # in place
        h = t["h0"].clone()
        y2, h2, _, _ = ha.ha_la_scan(*a, h0=h, hT=h, **kw)
        assert h2 is h and torch.equal(y2, y) and torch.equal(h, hT)
    if not back:
        return
    got = ha.ha_la_scan_backward(t["dy"], *a, h0=t["h0"], dhT=t["dhT"], **kw)
    again = ha.ha_la_scan_backward(t["dy"], *a, h0=t["h0"], dhT=t["dhT"], **kw)
    torch.cuda.synchronize()
    assert int(got[9]) == 0 and all(p is None or torch.equal(p, q) for p, q in zip(got[:9], again[:9]))
    grads = ref.scan_grads(flat(t["dy"]), *args, ref.d(t["h0"]), t["dhT"], t["seqs"])
    for name, g in zip(("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias", "dh0"), got):
        if g is None:
            assert t[{"dD": "D", "dz": "z", "ddt_bias": "dt_bias"}[name]] is None
            continue
        w, m = grads[name]
        off(name, g, w, (r if name in ("dx", "ddt", "dB", "dC", "dz") else 2 ** -24) * w.abs() + 2 ** -17 * m)


@TYPES
@pytest.mark.parametrize("T,ch,S,G", [(1, 1, 1, 1), (2, 8, 16, 1), (33, 70, 16, 2), (8, 32, 5, 4), (40, 65, 33, 1), (17, 24, 64, 3), (65, 130, 17, 1)])
def test_rows(T, ch, S, G, dtype):
    check(inputs(2, T, ch, S, G, dtype, seed=T + ch))
    check(inputs(1, T, ch, S, G, dtype, seed=S, D=False, z=False, bias=False, h0=False))


@TYPES
@pytest.mark.parametrize("cu", [[0, 1, 2, 10, 10, 33, 70], [0, 0, 31], [0, 64, 64], [0, 8, 16, 17, 90]], ids=str)
def test_packed(cu, dtype):
    check(inputs(1, cu[-1], 40, 16, 2, dtype, cu=cu, seed=cu[-1]))
    check(inputs(1, cu[-1], 24, 20, 1, dtype, cu=cu, seed=cu[1], h0=False, z=False), max_seqlen=max(b - a for a, b in zip(cu, cu[1:])))


@TYPES
@pytest.mark.parametrize("ch,G,rows", [(4096, 1, 1), (2048, 2, 2), (1024, 1, 1), (300, 1, 1)])
def test_states_to_a_thread(ch, G, rows, dtype):
    """Each of the ways that channels are shared out, by how many there are."""
    check(inputs(rows, 12, ch, 16, G, dtype, seed=ch, D=False))
    check(inputs(rows, 11, ch, 32, G, dtype, seed=ch + 1, z=False), back=rows == 1)
    if ch >= 1024:
        check(inputs(rows, 10, ch, 64, G, dtype, seed=ch + 2, D=False), back=False)


@TYPES
@pytest.mark.parametrize("cu", [None, [0, 700, 701, 1600], [0, 1600, 1600]], ids=str)
def test_segments(cu, dtype):
    """Few channels, long sequences: states of segments first, by all at once."""
    check(inputs(1, 1600, 16, 16, 1, dtype, cu=cu, seed=7, strong=0.05), back=False)
    check(inputs(1, 1600, 9, 40, 1, dtype, cu=cu, seed=8, strong=0.02, h0=False), back=False)


@TYPES
@pytest.mark.parametrize("pitch", [8, 3])
def test_rows_of_a_wider_tensor(pitch, dtype):
    check(inputs(2, 20, 48, 16, 2, dtype, pitch=pitch, seed=pitch))


@TYPES
def test_steps_of_every_size(dtype):
    """softplus from 2^-40 to 60, and steps given as they are."""
    t = inputs(1, 64, 32, 16, 1, dtype, seed=11, bias=False)
    t["dt"] = torch.linspace(-28, 60, 64 * 32).reshape(1, 64, 32).to(dtype).cuda()
    check(t)
    t["dt"] = torch.rand(1, 64, 32).to(dtype).cuda()
    t["dt"][:, 5] = 0
    check(t, softplus=False)


@TYPES
@pytest.mark.parametrize("N,ch,S,G", [(1, 64, 16, 1), (3, 70, 16, 1), (9, 130, 7, 2), (2, 36, 64, 4), (5, 20, 32, 1), (200, 8, 48, 1)])
def test_tokens_one_by_one(N, ch, S, G, dtype):
    ha, r = _ha(), ROUND[dtype]
    t = inputs(N, 4, ch, S, G, dtype, seed=N)
    rest = dict(D=t["D"], dt_bias=t["dt_bias"])
    state = t["h0"].clone()
    ys = []
    for i in range(4):
        y, new = ha.ha_la_scan_decode(*(t[k][:, i] if k != "A" else t[k] for k in ("x", "dt", "A", "B", "C")), state, z=t["z"][:, i], **rest)
        assert new is state
        ys.append(y)
    want, last, e, elast = ref.scan(flat(t["x"]), flat(t["dt"]), ref.d(t["A"]), flat(t["B"]), flat(t["C"]), ref.d(t["D"]), flat(t["z"]), ref.d(t["dt_bias"]), True,
                                    ref.d(t["h0"]), t["seqs"])
    off("y", torch.stack(ys, 1), want, r * want.abs() + 2 ** -19 * e)
    off("state", state, last, 2 ** -19 * elast)
    y0, s0 = ha.ha_la_scan_decode(*(t[k][:, 0] if k != "A" else t[k] for k in ("x", "dt", "A", "B", "C")), None)
    y1, s1 = ha.ha_la_scan_decode(*(t[k][:, 0] if k != "A" else t[k] for k in ("x", "dt", "A", "B", "C")), torch.zeros_like(state))
    assert torch.equal(y0, y1) and torch.equal(s0, s1)


@TYPES
@pytest.mark.parametrize("N,ch,S,G", [(1, 64, 16, 1), (7, 70, 32, 2), (130, 24, 64, 3)])
def test_token_wherever_b_and_c_lie(N, ch, S, G, dtype):
    ha = _ha()
    t, names = inputs(N, 1, ch, S, G, dtype, seed=N), ("x", "dt", "A", "B", "C")
    got = []
    for pitch, shift in ((0, 0), (4, 4), (4, 1), (3, 0)):
        s = {k: t[k] if k == "A" else t[k][:, 0] for k in names}
        for k in ("B", "C"):
            wide = torch.full((N, G * S + pitch + shift), float("nan"), dtype=dtype, device="cuda")
            s[k] = wide[:, shift:shift + G * S].unflatten(-1, (G, S))
            s[k].copy_(t[k][:, 0])
        got.append(ha.ha_la_scan_decode(*(s[k] for k in names), t["h0"].clone(), z=t["z"][:, 0], D=t["D"], dt_bias=t["dt_bias"]))
    want, last, e, elast = ref.scan(flat(t["x"]), flat(t["dt"]), ref.d(t["A"]), flat(t["B"]), flat(t["C"]), ref.d(t["D"]), flat(t["z"]), ref.d(t["dt_bias"]), True,
                                    ref.d(t["h0"]), t["seqs"])
    off("y", got[0][0][:, None], want, ROUND[dtype] * want.abs() + 2 ** -19 * e)
    off("state", got[0][1], last, 2 ** -19 * elast)
    for y, state in got[1:]:
        assert torch.equal(y, got[0][0]) and torch.equal(state, got[0][1])


@TYPES
def test_what_one_sequence_holds_stays_there(dtype):
    ha = _ha()
    cu = [0, 30, 37, 70]
    t = inputs(1, 70, 48, 16, 1, dtype, cu=cu, seed=5)
    names, kw = ("x", "dt", "A", "B", "C"), dict(D=t["D"], z=t["z"], dt_bias=t["dt_bias"], cu_seqlens=t["cu"])
    want = ha.ha_la_scan(*(t[k] for k in names), h0=t["h0"], **kw)
    wback = ha.ha_la_scan_backward(t["dy"], *(t[k] for k in names), h0=t["h0"], dhT=t["dhT"], **kw)
    s = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
    for k in ("x", "dt", "B", "C", "z", "dy"):
        s[k][:, 30:37] = float("nan")
    s["h0"][1], s["dhT"][1] = float("nan"), float("inf")
    kw["z"] = s["z"]
    got = ha.ha_la_scan(*(s[k] for k in names), h0=s["h0"], **kw)
    back = ha.ha_la_scan_backward(s["dy"], *(s[k] for k in names), h0=s["h0"], dhT=s["dhT"], **kw)
    keep = [i for i in range(70) if not 30 <= i < 37]
    assert torch.equal(got[0][:, keep], want[0][:, keep]) and torch.equal(got[1][[0, 2]], want[1][[0, 2]])
    for i in (0, 1, 3, 4, 6):
        assert torch.equal(back[i][:, keep], wback[i][:, keep]), i
    assert torch.equal(back[8][[0, 2]], wback[8][[0, 2]])


@TYPES
def test_no_token(dtype):
    ha = _ha()
    x, B = torch.empty(2, 0, 40, dtype=dtype, device="cuda"), torch.empty(2, 0, 1, 16, dtype=dtype, device="cuda")
    A, h0 = -torch.ones(40, 16, device="cuda"), torch.randn(2, 40, 16, device="cuda")
    y, hT, status, _ = ha.ha_la_scan(x, x, A, B, B, h0=h0)
    assert y.shape == x.shape and torch.equal(hT, h0) and int(status) == 0
    got = ha.ha_la_scan_backward(x, x, x, A, B, B, D=torch.ones(40, device="cuda"), h0=h0, dhT=h0, dA=torch.full((40, 16), 7.0, device="cuda"))
    assert not got[2].any() and not got[5].any() and torch.equal(got[8], h0)
    y, st = ha.ha_la_scan_decode(x.reshape(0, 40), x.reshape(0, 40), A, B.reshape(0, 1, 16), B.reshape(0, 1, 16), None)
    assert y.shape == (0, 40) and st.shape == (0, 40, 16)


def test_lengths_that_do_not_fit_are_reported():
    ha = _ha()
    x, B, A = torch.randn(1, 50, 64, device="cuda"), torch.randn(1, 50, 1, 16, device="cuda"), -torch.ones(64, 16, device="cuda")
    for cu, most in (([0, 20, 49], 0), ([1, 20, 50], 0), ([0, 30, 20, 50], 0), ([0, 20, 50], 25), ([0, -5, 50], 0), ([0, 2 ** 31 - 1, 50], 0)):
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        assert int(ha.ha_la_scan(x, x, A, B, B, cu_seqlens=c, max_seqlen=most)[2]) == 6, cu
        assert int(ha.ha_la_scan_backward(x, x, x, A, B, B, cu_seqlens=c, max_seqlen=most)[9]) == 6, cu
    long = torch.randn(1, 2000, 8, device="cuda")            # (in segments)
    Bl, c = torch.randn(1, 2000, 1, 16, device="cuda"), torch.tensor([0, 1500, 700, 2000], dtype=torch.int32, device="cuda")
    assert int(ha.ha_la_scan(long, long, A[:8], Bl, Bl, cu_seqlens=c)[2]) == 6


def test_long_offsets():
    """More than 2^31 elements of x and of the states: the last sequences against a call on them alone."""
    ha, T, ch = _ha(), 600_000, 4096
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB")
    x = torch.empty(1, T, ch, dtype=torch.bfloat16, device="cuda").normal_()
    B = torch.randn(1, T, 1, 16, device="cuda").bfloat16()
    A = -torch.rand(ch, 16, device="cuda")
    cu = torch.tensor([0, T // 2, T - 50, T], dtype=torch.int32, device="cuda")
    y, hT, _, _ = ha.ha_la_scan(x, x, A, B, B, cu_seqlens=cu)
    tail, tb = x[:, T - 50:].contiguous(), B[:, T - 50:].contiguous()
    # (as one of three sequences, so that the channels are shared out alike)
    three = torch.tensor([0, 50, 100, 150], dtype=torch.int32, device="cuda")
    want = ha.ha_la_scan(*(t.repeat(1, 3, 1) for t in (tail, tail)), A, *(t.repeat(1, 3, 1, 1) for t in (tb, tb)), cu_seqlens=three)
    assert torch.equal(y[:, T - 50:], want[0][:, 100:]) and torch.equal(hT[2], want[1][2])
    del y, x
    N = 33_000
    x = torch.randn(N, ch, device="cuda").bfloat16()
    st = torch.randn(N, ch, 16, device="cuda")
    b = torch.randn(N, 1, 16, device="cuda").bfloat16()
    last = st[-3:].clone()
    want = ha.ha_la_scan_decode(x[-3:].contiguous(), x[-3:].contiguous(), A, b[-3:].contiguous(), b[-3:].contiguous(), last)
    got = ha.ha_la_scan_decode(x, x, A, b, b, st)
    assert torch.equal(got[0][-3:], want[0]) and torch.equal(st[-3:], want[1])
    del st, x
    torch.cuda.empty_cache()
