"""The 64-bit plain forms that the kernels are compared with: gradients against differences, the norms' against torch's."""
import pytest
import torch

from tests import layer_reference as ref


def _inputs(seed=0, HK=2, HV=4, D=4, T=9, cu=None):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    N = 1 if cu is None else len(cu) - 1
    return dict(q=r(1, T, HK, D), k=r(1, T, HK, D), v=r(1, T, HV, D), g=-r(1, T, HV).abs(), h0=r(N, HV, D, D)), r(1, T, HV, D), r(N, HV, D, D)


@pytest.mark.parametrize("cu", [None, [0, 4, 4, 9]])
def test_gradients_of_the_recurrence_against_differences(cu):
    t, do, dhT = _inputs(cu=cu)
    cu = None if cu is None else torch.tensor(cu)
    loss = lambda a: sum((x * y).sum() for x, y in zip(ref.gla(**a, cu=cu, scale=0.7), (do, dhT)))
    dq, dk, dv, dg, dh0 = ref.gla_backward(do, **t, dhT=dhT, cu=cu, scale=0.7)
    got = dict(q=ref.heads_sum(dq, 2), k=ref.heads_sum(dk, 2), v=dv, g=dg, h0=dh0)
    for name, x in t.items():
        for i in range(0, x.numel(), 7):
            step = torch.zeros_like(x).flatten()
            step[i] = 1e-6
            step = step.reshape(x.shape)
            slope = (loss({**t, name: x + step}) - loss({**t, name: x - step})) / 2e-6
            assert abs(float(slope) - float(got[name].flatten()[i])) < 1e-7 * (1 + abs(float(slope))), (name, i)


def test_magnitudes_bound_the_values():
    t, do, dhT = _inputs(seed=2)
    for x, m in zip(ref.gla(**t, scale=-0.3), ref.gla(**t, scale=-0.3, magnitude=True)):
        assert bool((x.abs() <= m * (1 + 1e-12)).all())
    for x, m in zip(ref.gla_backward(do, **t, dhT=dhT), ref.gla_backward(do, **t, dhT=dhT, magnitude=True)):
        assert bool((x.abs() <= m * (1 + 1e-12)).all())


@pytest.mark.parametrize("name", [None, "silu", "sigmoid"])
def test_gated_norm_against_autograd(name):
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    x, w, z, dy = r(5, 7).requires_grad_(), r(7).requires_grad_(), r(5, 7).requires_grad_(), r(5, 7)
    y = torch.nn.functional.rms_norm(x, (7,), w, 1e-3)
    if name:
        y = y * (torch.nn.functional.silu(z) if name == "silu" else torch.sigmoid(z))
    assert torch.allclose(y, ref.gated_norm(x, w, z if name else None, name, 1e-3), rtol=1e-12)
    got = ref.gated_norm_backward(dy, x, w, z if name else None, name, 1e-3)
    want = torch.autograd.grad(y, [x, w] + ([z] if name else []), dy)
    for (a, m), b in zip((got[n] for n in ("dx", "dw", "dz")[:len(want)]), want):
        assert torch.allclose(a, b, rtol=1e-10, atol=1e-12) and bool((a.abs() <= m * (1 + 1e-12)).all())


@pytest.mark.parametrize("post", [False, True])
def test_add_norm_against_autograd(post):
    gen = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    x, res, w, wp, dy, dr = r(5, 7).requires_grad_(), r(5, 7).requires_grad_(), r(7).requires_grad_(), r(7).requires_grad_(), r(5, 7), r(5, 7)
    f = torch.nn.functional.rms_norm(x, (7,), wp, 1e-3) if post else x
    out = res + 0.5 * f
    y = torch.nn.functional.rms_norm(out, (7,), w, 1e-3)
    y2, out2, _ = ref.add_norm(x, res, w, wp if post else None, 0.5, 1e-3)
    assert torch.allclose(y, y2, rtol=1e-12) and torch.allclose(out, out2, rtol=1e-12)
    got = ref.add_norm_backward(dy, dr, x, out, w, wp if post else None, 0.5, 1e-3)
    want = torch.autograd.grad([y, out], [x, res, w] + ([wp] if post else []), [dy, dr])
    for n, b in zip(("dx", "dr", "dw", "dw_post"), want):
        a, m = got[n]
        assert torch.allclose(a, b, rtol=1e-10, atol=1e-12) and bool((a.abs() <= m * (1 + 1e-12)).all()), n
