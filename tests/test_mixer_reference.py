"""The 64-bit forms that the mixers' kernels are compared with, themselves: gradients against differences, the scan against its closed form, attention
against explicit sums, the absorbed form against the expanded one."""
import math

import torch

from tests import mixer_reference as ref


def make(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def test_convolution_by_hand():
    x = torch.tensor([[1.0], [2.0], [3.0]], dtype=torch.float64)
    y, hT, mag = ref.conv(x, torch.tensor([[10.0, 1.0]], dtype=torch.float64), torch.tensor([0.5], dtype=torch.float64), torch.tensor([[[7.0]], [[-1.0]]], dtype=torch.float64), False,
                          [(0, 1), (1, 2)])
    assert y[:, 0].tolist() == [71.5, -7.5, 23.5] and hT[:, 0, 0].tolist() == [1.0, 3.0] and mag[:, 0].tolist() == [71.5, 12.5, 23.5]


def test_a_sequence_shorter_than_the_state():
    h0 = make(1, 3, 2)
    _, hT, _ = ref.conv(make(1, 2, seed=1), make(2, 4, seed=2), None, h0, True, [(0, 1)])
    assert torch.equal(hT[0, :2], h0[0, 1:]) and torch.equal(hT[0, 2], make(1, 2, seed=1)[0])


def difference(f, t, i, h=1e-6):
    a, b = t.clone(), t.clone()
    a.view(-1)[i] += h
    b.view(-1)[i] -= h
    return (f(a) - f(b)) / (2 * h)


def test_gradients_of_the_convolution_against_differences():
    seqs = [(0, 2), (2, 0), (2, 5)]
    t = dict(x=make(7, 3), w=make(3, 4, seed=1), bias=make(3, seed=2), h0=make(3, 3, 3, seed=3))
    dy, dhT = make(7, 3, seed=4), make(3, 3, 3, seed=5)
    grads = ref.conv_grads(dy, t["x"], t["w"], t["bias"], t["h0"], dhT, True, seqs)
    for name, key in (("dx", "x"), ("dw", "w"), ("db", "bias"), ("dh0", "h0")):
        def loss(v):
            s = dict(t, **{key: v})
            y, hT, _ = ref.conv(s["x"], s["w"], s["bias"], s["h0"], True, seqs)
            return float((y * dy).sum() + (hT * dhT).sum())
        g, mag = grads[name]
        for i in range(t[key].numel()):
            assert abs(difference(loss, t[key], i) - g.reshape(-1)[i]) < 1e-7 and mag.reshape(-1)[i] >= abs(g.reshape(-1)[i]) * 0.5


def test_one_channel_of_the_scan_in_closed_form():
    """Constant steps: h_t = sum_j e^{(t - j) delta A} delta B x_j."""
    T, delta, A = 6, 0.3, -0.7
    x = make(T, 1)
    one = torch.ones(T, 1, 1, dtype=torch.float64)
    y, hT, _, _ = ref.scan(x, torch.full((T, 1), delta, dtype=torch.float64), torch.tensor([[A]], dtype=torch.float64), one, 2 * one, None, None, None, False, None, [(0, T)])
    want = [sum(math.exp((t - j) * delta * A) * delta * float(x[j]) for j in range(t + 1)) for t in range(T)]
    assert torch.allclose(y[:, 0], 2 * torch.tensor(want, dtype=torch.float64), atol=1e-12) and abs(float(hT) - want[-1]) < 1e-12


def test_gradients_of_the_scan_against_differences():
    seqs = [(0, 3), (3, 0), (3, 4)]
    t = dict(x=make(7, 4), dt=make(7, 4, seed=1), A=-make(4, 3, seed=2).abs(), B=make(7, 2, 3, seed=3), C=make(7, 2, 3, seed=4), D=make(4, seed=5), z=make(7, 4, seed=6),
             dt_bias=make(4, seed=7), h0=make(3, 4, 3, seed=8))
    dy, dhT = make(7, 4, seed=9), make(3, 4, 3, seed=10)
    grads = ref.scan_grads(dy, *(t[k] for k in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias")), True, t["h0"], dhT, seqs)
    for key in t:
        def loss(v):
            s = dict(t, **{key: v})
            y, hT, _, _ = ref.scan(*(s[k] for k in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias")), True, s["h0"], seqs)
            return float((y * dy).sum() + (hT * dhT).sum())
        g, e = grads["d" + key]
        for i in range(0, t[key].numel(), 3):
            assert abs(difference(loss, t[key], i) - g.reshape(-1)[i]) < 1e-7, key
        assert bool((e >= g.abs()).all())


def test_attention_by_hand_and_rows_that_see_nothing():
    q, k, v = make(3, 4), make(5, 4, seed=1), make(5, 2, seed=2)
    v[4] = math.nan
    o, lse, mag, top = ref.attend(q, k, v, torch.tensor([0, 2, 4]), 0.5)
    w = torch.exp(0.5 * q[1] @ k[:2].T)
    assert torch.allclose(o[1], (w @ v[:2]) / w.sum()) and torch.allclose(lse[1], torch.log(w.sum()))
    assert not o[0].any() and lse[0] == -math.inf and bool(torch.isfinite(o).all()) and bool((mag >= o.abs() - 1e-12).all()) and top[0] == 0


def test_absorbed_is_expanded():
    """Scores against W c are scores of W^T q against c, and the values' product may come behind the sum."""
    c, r, uk, uv, qn, qr = make(6, 8), make(6, 2, seed=1), make(3, 8, seed=2), make(4, 8, seed=3), make(5, 3, seed=4), make(5, 2, seed=5)
    limit = torch.arange(2, 7)
    o, lse, _, _ = ref.attend(torch.cat([qn, qr], -1), torch.cat([c @ uk.T, r], -1), c @ uv.T, limit, 0.3)
    o2, lse2, _, _ = ref.attend(torch.cat([qn @ uk, qr], -1), torch.cat([c, r], -1), c, limit, 0.3)
    assert torch.allclose(o, o2 @ uv.T) and torch.allclose(lse, lse2)
