"""The short convolution where a thread goes through as many tokens one behind the other as it ever does (32 forwards, 270 to 512 backwards), sequences starting
and ending inside its run, against 64 bits on the GPU; and bounds without the room that such runs need where they are short.

Whole numbers, no activation: every product and sum is below 2^24, so nothing is rounded and results are the 64-bit ones.  With silu: y as elsewhere, e = dy act'(s) off by
2^-19 |dy| (1 + M), M the magnitude of the sum ahead of the activation; dx and dh0 add up 4 terms and a gradient at the most (5 2^-24): 2^-18 of the terms' magnitudes.  dw and db
add up a run's tokens in 32 bits, runs in 64: 8 of them 8 2^-24, 2^-18 in all, 512 of them 2^-15."""
import pytest
import torch

from tests.test_gpu_conv import ROUND, TYPES

pytestmark = pytest.mark.gpu
CU = [0, 1, 1, 3, 700, 701, 5000, 5002, 12345, 12345, 20011]


def plain(t, act):
    """y, hT, dx, dw, db, dh0 in 64 bits, and the magnitudes of the sums ahead of the activation and of the gradients' terms."""
    w, K, C = t["w"].double(), t["w"].shape[1], t["x"].shape[-1]
    bias = t["bias"].double()
    out = {k: [] for k in ("y", "hT", "dx", "dh0", "M", "m_dx", "m_dh0")}
    dw, db, m_dw, m_db = 0, 0, 0, 0
    for n, (a, b) in enumerate(zip(t["cu"], t["cu"][1:])):
        m = b - a
        full = torch.cat([t["h0"][n].double(), t["x"][0, a:b].double()])
        out["hT"].append(full[m:])
        s = bias + sum(w[:, j] * full[j:j + m] for j in range(K))
        M = bias.abs() + sum(w[:, j].abs() * full[j:j + m].abs() for j in range(K))
        g = torch.sigmoid(s)
        e = t["dy"][0, a:b].double() * (g * (1 + s * (1 - g)) if act else 1)
        out["y"].append(s * g if act else s)
        out["M"].append(M)
        for sign, ee, name in ((1, e, "d"), (0, t["dy"][0, a:b].double().abs() * (1 + M), "m_d")):
            f = (lambda v: v) if sign else torch.abs
            back = torch.zeros_like(full)
            back[m:] += f(t["dhT"][n].double())
            for j in range(K):
                back[j:j + m] += f(w[:, j]) * ee
            out[name + "h0"].append(back[:K - 1])
            out[name + "x"].append(back[K - 1:])
            to_w = torch.stack([(ee * f(full[j:j + m])).sum(0) for j in range(K)], -1)
            if sign:
                dw, db = dw + to_w, db + ee.sum(0)
            else:
                m_dw, m_db = m_dw + to_w, m_db + ee.sum(0)
    out = {k: (torch.stack if k in ("hT", "dh0", "m_dh0") else torch.cat)(v) for k, v in out.items()}
    return dict(out, dw=dw, db=db, m_dw=m_dw, m_db=m_db)


def inputs(cu, C, K, dtype, whole, pitch=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, N = cu[-1], len(cu) - 1

    def n(*s, top=3):
        t = torch.randn(*s, generator=gen, device="cuda")
        return t.round().clamp(-top, top) if whole else t

    return dict(x=n(1, T, C + pitch).to(dtype)[..., :C], dy=n(1, T, C).to(dtype), w=n(C, K) * (1 if whole else 0.5), bias=n(C), h0=n(N, K - 1, C).to(dtype), dhT=n(N, K - 1, C).to(dtype), cu=cu)


def run(t, act):
    import paper_2609_32114_b200 as ha

    cu = torch.tensor(t["cu"], dtype=torch.int32, device="cuda")
    kw = dict(bias=t["bias"], activation="silu" if act else None, h0=t["h0"], cu_seqlens=cu)
    y, hT, s1 = ha.ha_la_conv(t["x"], t["w"], **kw)
    dx, dw, db, dh0, s2, ws = ha.ha_la_conv_backward(t["dy"], t["x"], t["w"], dhT=t["dhT"], **kw)
    assert int(s1) == 0 == int(s2)
    return dict(y=y[0], hT=hT, dx=dx[0], dw=dw, db=db, dh0=dh0), ws


def check(t, act, long):
    got, ws = run(t, act)
    want, r = plain(t, act), ROUND[t["x"].dtype]
    assert torch.equal(got["hT"].double(), want["hT"])
    bound = {"y": (r + 2 ** -20) * want["y"].abs() + 2 ** -20 * want["M"]}
    for name in ("dx", "dh0"):
        bound[name] = r * want[name].abs() + 2 ** -18 * want["m_" + name]
    for name in ("dw", "db"):
        bound[name] = 2 ** -24 * want[name].abs() + (2 ** -15 if long else 2 ** -18) * want["m_" + name]
    for name, b in bound.items():
        off = (got[name].double() - want[name]).abs() - b - 1e-37
        assert bool((off <= 0).all()), (name, float(off.max()))
    return ws


def runs(ws, t):
    """How many runs the gradients' workspace has room for."""
    return (ws.numel() - 256) // (4 * (t["w"].shape[1] + 1) * t["x"].shape[-1])


@TYPES
@pytest.mark.parametrize("K", [2, 3, 4])
@pytest.mark.parametrize("C,pitch", [(4096, 0), (4096, 8), (1030, 0)])
def test_whole_numbers_in_long_runs(C, pitch, K, dtype):
    t = inputs(CU, C, K, dtype, True, pitch=pitch, seed=C + K)
    got, ws = run(t, False)
    assert CU[-1] / runs(ws, t) > (70 if C == 1030 else 200)  # (1030 go element by element, in longer runs than the workspace has to have room for)
    want = plain(t, False)
    for name, g in got.items():
        assert torch.equal(g.double(), want[name]), name


@TYPES
@pytest.mark.parametrize("K", [2, 3, 4])
def test_long_runs(K, dtype):
    t = inputs(CU, 4096, K, dtype, False, seed=K)
    assert CU[-1] / runs(check(t, True, True), t) > 200


@TYPES
@pytest.mark.parametrize("cu,C,K", [([0, 1, 2, 3, 5, 8, 8, 40, 41], 264, 4), ([0, 0, 77], 33, 3), ([0, 300, 300], 72, 2), ([0, 1290, 1291, 3000], 24, 4), ([0, 333], 515, 4)], ids=str)
def test_short_runs(cu, C, K, dtype):
    for act in (False, True):
        check(inputs(cu, C, K, dtype, False, pitch=8 if C % 8 == 0 else 0, seed=C), act, False)
