"""How exact the selective scan is where 2^-19 of everything would hide it: steps of every size by themselves, and sums over many tokens."""
import numpy as np
import pytest
import torch

from tests import test_gpu_scan as scan

pytestmark = pytest.mark.gpu


def _ha():
    import paper_2609_32114_b200 as ha

    return ha


def test_steps_by_themselves():
    """One token with x = B = 1 from a state of zero leaves the step itself.  For small steps, relative: e 2^-22 (the exponential), its rounded exponent |v| (2^-24 + 2^-26), 2 + e
    one rounding and its reciprocal 2^-23, the quotient, four of the polynomial and the last product one each: 4 + 1 + 2 + 6 of 2^-24, below 2^-20, and |v| 1.25 2^-24."""
    v = torch.linspace(-80, 30, 4096 * 8).view(8, 4096)
    one = torch.ones(8, 1, 1, device="cuda")
    x = torch.ones(8, 4096, device="cuda")
    _, state = _ha().ha_la_scan_decode(x, v.cuda(), -torch.ones(4096, 1, device="cuda"), one, one, None)
    v = v.double()
    want = v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))
    off = (state[..., 0].double().cpu() - want).abs() / want - 2 ** -20 - 1.25 * 2 ** -24 * v.abs()
    assert float(off.max()) <= 0


def test_steps_that_end():
    """No step at all, steps that are their argument, and NaN, which stays."""
    v = torch.tensor([[-3e38, -float("inf"), -200.0, 200.0, 3e38, float("nan"), 0.0, -0.0]], device="cuda")
    one = torch.ones(1, 1, 1, device="cuda")
    _, state = _ha().ha_la_scan_decode(torch.ones_like(v), v, -torch.zeros(8, 1, device="cuda"), one, one, None)
    got = state[0, :, 0].cpu()
    assert got[:5].tolist() == [0, 0, 0, 200.0, v[0, 4].item()] and bool(got[5].isnan())
    assert float((got[6:].double() - 0.6931471805599453).abs().max()) <= 2 ** -20


def test_decays_on_the_average():
    """x = 0: what is left of a state of one is the decay by itself.  Its average error decides how far a state that lasts n tokens is off, n times as much: less than 2^-26, a
    quarter of a rounding, in every octave of exponents below one, with 2^19 decays in each, whose roundings (2^-24.5 each) average out to 2^-34."""
    one, gen = torch.ones(128, 1, 1, device="cuda"), torch.Generator(device="cuda").manual_seed(1)
    A, st = -torch.ones(4096, 1, device="cuda"), torch.ones(128, 4096, 1, device="cuda")
    zero = torch.zeros(128, 4096, device="cuda")
    for octave in range(-18, 0):
        delta = (1 + torch.rand(128, 4096, generator=gen, device="cuda")) * 2.0 ** octave * 0.693
        _, state = _ha().ha_la_scan_decode(zero, delta, A, one, one, st, softplus=False, state_out=torch.empty_like(st))
        error = state[..., 0].double() * torch.exp(delta.double()) - 1
        assert abs(float(error.mean())) <= 2 ** -26, octave
        assert float(error.abs().max()) <= 2 ** -22 + 2 ** -23 * 2 ** max(octave, 0)
    _, state = _ha().ha_la_scan_decode(zero, zero, A, one, one, st, softplus=False, state_out=torch.empty_like(st))
    assert torch.equal(state, st)                            # nothing passes: not one bit changes


def test_gradients_that_add_up_over_many_tokens():
    """The same token 65,536 times: from the sum's size on, what each adds would be rounded alike, so 32 bits lose what 64 keep.  All terms are positive but one.  Relative:
    decays of 0.05 to 0.6 are off by 2^-21, which states and their gradients carry on 1.5 times each, so their product by 2^-19; products 2^-21; sums of 8 tokens 8 times 2^-20."""
    ha, T, ch, S = _ha(), 65536, 6, 3
    gen = torch.Generator().manual_seed(4)
    r = lambda *s: 0.5 + 0.5 * torch.rand(*s, generator=gen)                   # noqa: E731
    x, dt, dy, B, C, D, A = r(ch), r(ch), r(ch), r(1, S), r(1, S), r(ch), -2 * r(ch, S)
    rows = lambda t: t.cuda().expand(1, T, *t.shape).contiguous()              # noqa: E731
    got = ha.ha_la_scan_backward(rows(dy), rows(x), rows(dt), A.cuda(), rows(B), rows(C), D=D.cuda(), dt_bias=torch.zeros(ch, device="cuda"), softplus=False)
    x, dt, dy, B, C, D, A = (t.double().numpy() for t in (x, dt, dy, B, C, D, A))
    a, u = np.exp(dt[:, None] * A), (dt * x)[:, None] * B
    h = np.zeros((T + 1, ch, S))
    for t in range(T):
        h[t + 1] = a * h[t] + u
    dh, flow, to_b = np.zeros((ch, S)), np.zeros((ch, S)), np.zeros(ch)
    for t in reversed(range(T)):
        dh = C * dy[:, None] + dh
        to_b += (dh * B).sum(1)
        dh = dh * a
        flow += dh * h[t]
    dA, from_a, from_b = flow * dt[:, None], (flow * A).sum(1), x * to_b
    off = lambda g, w, m=None: float(((g.double().cpu() - torch.tensor(w)).abs() / torch.tensor(w if m is None else m)).max())       # noqa: E731
    assert off(got[2], dA) <= 2 ** -18
    assert off(got[5], T * x * dy) <= 2 ** -21
    assert off(got[7], from_a + from_b, from_b - from_a) <= 2 ** -18


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_gradients_of_long_sequences(dtype):
    """Everything of a few thousand random tokens, to the bounds that short sequences keep (sums over tokens in parts of at most 64 in 32 bits, the parts in 64)."""
    scan.check(scan.inputs(1, 3300, 5, 16, 1, dtype, cu=[0, 1300, 1301, 3300], seed=21, strong=0.3))
