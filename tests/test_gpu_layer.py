"""The operators run together, as a layer of a hybrid model runs them, and where only large calls go.

Bounds of the runs, in the norm of a whole tensor: each operator is off by 2^-15 of its result in fp32 at most (test_gpu_gla, test_gpu_norm) and by
2^-8 in bf16, and a norm passes on at most twice what it is given (its Jacobian is rs (1 - n n^T / cols) w, |w| < 2 |mean w| here).  Four operators one behind the
other: 8 x 2^-15 and 8 x 2^-8; back through the same four, from values that are off by that: twice as much."""
import pytest
import torch

from tests import layer_reference as ref
from tests.test_gpu_gla import check, close, cuda, inputs

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


def near(name, got, want, bound):
    got, want = got.detach().double().cpu(), want.detach().double()
    assert got.shape == want.shape and bool(torch.isfinite(got).all()), name
    assert float((got - want).norm()) <= bound * float(want.norm()), (name, float((got - want).norm() / want.norm()))


# ---------------------------------------------------------------- a layer

def weights(T, HK, HV, D, dtype, seed=0, N=1):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    C = HV * D
    return dict(x=r(T, C).to(dtype), res=r(T, C).to(dtype), z=r(T, HV, D).to(dtype), g=-torch.nn.functional.softplus(r(T, HV) + 2), beta=torch.sigmoid(r(T, HV)),
                qk=torch.nn.functional.normalize(r(2, T, HK, D), dim=-1).to(dtype), h0=0.2 * r(N, HV, D, D),
                **{n: 1 + 0.1 * r(C if n in "ac" else D) for n in "abc"}, post=1 + 0.1 * r(C))


def plain_layer(p, cu, delta=False, scale=0.125):
    """Token by token, in 64 bits, recorded for autograd."""
    C, (T, HV, D) = p["x"].shape[1], p["z"].shape
    norm = lambda x, w: x * ref.rms_scale(x, 1e-6) * w
    r1 = p["res"] + p["x"]
    v = norm(r1, p["a"]).reshape(T, HV, D)
    q, k = (t.repeat_interleave(HV // t.shape[1], 1) for t in p["qk"])
    o, hT = [], []
    for n, (a, b) in enumerate(zip(cu, cu[1:])):
        h = p["h0"][n]
        for t in range(a, b):
            h = p["g"][t].exp()[:, None, None] * h
            new = v[t]
            if delta:
                new = p["beta"][t][:, None] * (new - torch.einsum("hkv,hk->hv", h, k[t]))
            h = h + k[t][:, :, None] * new[:, None, :]
            o.append(scale * torch.einsum("hkv,hk->hv", h, q[t]))
        hT.append(h)
    n = norm(torch.stack(o), p["b"]) * torch.nn.functional.silu(p["z"])
    r2 = r1 + 0.5 * norm(n.reshape(T, C), p["post"])
    return norm(r2, p["c"]), r2, torch.stack(hT)


def layer(ha, p, cu, delta=False, scale=0.125):
    T, HV, D = p["z"].shape
    y1, r1 = ha.ha_la_add_norm(p["x"], p["res"], p["a"])
    v, (q, k) = y1.view(1, T, HV, D), p["qk"][:, None]
    if delta:
        o, hT, st, _ = ha.ha_la_prefill(q, k, v, p["g"][None], p["beta"][None], h0=p["h0"], cu_seqlens=cu, scale=scale)
    else:
        o, hT, st, _ = ha.ha_la_gla_prefill(q, k, v, p["g"][None], h0=p["h0"], cu_seqlens=cu, scale=scale)
    o = o.view(T, HV, D)
    n = ha.ha_la_gated_norm(o, p["b"], p["z"])
    y, r2 = ha.ha_la_add_norm(n.view(T, HV * D), r1, p["c"], w_post=p["post"], scale=0.5)
    return (y, r2, hT), (v, r1, o, n, st)


def layer_backward(ha, p, cu, kept, r2, dy, dr, dhT, scale=0.125):
    v, r1, o, n, _ = kept
    T, HV, D = p["z"].shape
    dn, dr1, dc, dpost = ha.ha_la_add_norm_backward(dy, dr, n.view(T, HV * D), r2, p["c"], w_post=p["post"], scale=0.5)
    do, db, dz = ha.ha_la_gated_norm_backward(dn.view(T, HV, D), o, p["b"], p["z"])
    q, k = p["qk"][:, None]
    dq, dk, dv, dg, dh0, st, _ = ha.ha_la_gla_backward(do[None], q, k, v, p["g"][None], h0=p["h0"], dhT=dhT, cu_seqlens=cu, scale=scale)
    dx, dres, da, _ = ha.ha_la_add_norm_backward(dv.view(T, HV * D), dr1, p["x"], r1, p["a"])
    return dict(x=dx, res=dres, z=dz, g=dg[0], qk=torch.cat([dq, dk]), h0=dh0, a=da, b=db, c=dc, post=dpost), st


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_64", "bf16_128"])
@pytest.mark.parametrize("cu", [[0, 1], [0, 150], [0, 100, 100, 101, 290]])
def test_a_layer_and_its_gradients(cu, dtype, D):
    ha, T, bound = _ha(), cu[-1], 2 ** -12 if dtype == torch.float32 else 2 ** -5
    p = weights(T, 1, 2, D, dtype, seed=T, N=len(cu) - 1)
    gen = torch.Generator().manual_seed(1)
    dy, dr = (torch.randn(T, 2 * D, generator=gen).to(dtype) for _ in range(2))
    dhT = 0.2 * torch.randn(p["h0"].shape, generator=gen)
    plain = {k: x.double().requires_grad_() for k, x in p.items() if k != "beta"}
    want = plain_layer(plain, cu)
    torch.autograd.backward(want, [dy.double(), dr.double(), dhT.double()])
    c, dcu = cuda(p), torch.tensor(cu, dtype=torch.int32, device="cuda")
    got, kept = layer(ha, c, dcu)
    grads, st = layer_backward(ha, c, dcu, kept, got[1], dy.cuda(), dr.cuda(), dhT.cuda())
    torch.cuda.synchronize()
    assert int(kept[-1].item()) == 0 and int(st.item()) == 0
    for name, a, b in zip(("y", "r", "hT"), got, want):
        near(name, a, b, bound)
    for name, a in grads.items():
        near("d" + name, a, plain[name].grad, 2 * bound)


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_128"])
def test_around_the_delta_rule(dtype, D):
    ha, cu = _ha(), [0, 70, 71, 200]
    p = weights(200, 1, 2, D, dtype, seed=3, N=3)
    want = plain_layer({k: x.double() for k, x in p.items()}, cu, delta=True)
    got, kept = layer(ha, cuda(p), torch.tensor(cu, dtype=torch.int32, device="cuda"), delta=True)
    torch.cuda.synchronize()
    assert int(kept[-1].item()) == 0
    for name, a, b in zip(("y", "r", "hT"), got, want):
        near(name, a, b, 2 ** -12 if dtype == torch.float32 else 2 ** -5)


def test_a_training_step_is_captured():
    """Forward and backward of two layers in one graph, replayed on new contents: the bits of the calls one by one."""
    ha, cu = _ha(), torch.tensor([0, 130, 400], dtype=torch.int32, device="cuda")
    p = cuda(weights(400, 2, 4, 128, torch.bfloat16, seed=5, N=2))
    dy = torch.randn(400, 512, device="cuda").bfloat16()

    def step():
        (y, r, hT), kept = layer(ha, p, cu)
        (y2, r2, hT2), kept2 = layer(ha, p | dict(x=y, res=r), cu)
        g2, _ = layer_backward(ha, p | dict(x=y, res=r), cu, kept2, r2, dy, None, None)
        g, _ = layer_backward(ha, p, cu, kept, r, g2["x"], g2["res"], None)
        return [y2, r2, hT, hT2, *g.values(), *g2.values()]

    step()
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        outs = step()
    for k in ("x", "res", "z"):
        p[k].copy_(torch.randn(p[k].shape, device="cuda"))
    want = step()
    gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_tokens_one_by_one_after_a_prompt():
    ha, N, HV, D = _ha(), 3, 2, 128
    p = weights(20 * N, 1, HV, D, torch.float32, seed=9, N=N)
    cu = [20 * i for i in range(N + 1)]
    want, r_want, h_want = plain_layer({k: x.double() for k, x in p.items()}, cu)
    c = cuda(p)
    rows = lambda a, b: torch.cat([torch.arange(20 * n + a, 20 * n + b) for n in range(N)]).cuda()
    part = lambda i: {k: (x[:, i] if k == "qk" else x[i] if k in ("x", "res", "z", "g", "beta") else x).contiguous() for k, x in c.items()}
    (_, _, h), _ = layer(ha, part(rows(0, 18)), torch.tensor([18 * i for i in range(N + 1)], dtype=torch.int32, device="cuda"))
    for t in (18, 19):
        i = rows(t, t + 1)
        s = part(i)
        y1, r1 = ha.ha_la_add_norm(s["x"], s["res"], s["a"])
        o, h = ha.ha_la_gla_decode(s["qk"][0], s["qk"][1], y1.view(N, HV, D), s["g"], h, scale=0.125)
        n = ha.ha_la_gated_norm(o, s["b"], s["z"])
        y, r2 = ha.ha_la_add_norm(n.view(N, HV * D), r1, s["c"], w_post=s["post"], scale=0.5)
        near("y", y, want[i.cpu()], 2 ** -12)
        near("r", r2, r_want[i.cpu()], 2 ** -12)
    near("h", h, h_want, 2 ** -12)


# ---------------------------------------------------------------- what only large calls reach

@pytest.mark.parametrize("HK,HV,N", [(1, 4, 320), (1, 4, 160), (2, 8, 160), (2, 8, 60), (3, 6, 130)])
def test_runs_of_heads(HK, HV, N):
    """Many steps with several V-heads to a q/k head: the gradient kernel takes heads one behind the other, all of them or some."""
    lens = torch.randint(1, 4, (N,), generator=torch.Generator().manual_seed(N))
    lens[N // 2] = 140
    cu = [0, *lens.cumsum(0).tolist()]
    check(*inputs(cu[-1], HK, HV, 128, torch.bfloat16, cu=cu, seed=N, h0=N > 200), cu=cu)


@pytest.mark.parametrize("cu", [[0, 4100], [0, 3000, 3001, 3001, 4500]])
def test_sequences_in_segments(cu):
    """Few long sequences: their states are summed and then walked segment by segment."""
    check(*inputs(cu[-1], 1, 1, 128, torch.bfloat16, cu=cu, seed=cu[1], shift=5.0), cu=cu)


def test_long_rows_on_the_cuda_cores():
    check(*inputs(1500, 1, 1, 64, torch.float32, seed=15, shift=5.0))


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.bfloat16, 128)], ids=["fp32_64", "bf16_128"])
def test_gates_of_minus_infinity(dtype, D):
    t, do, dhT = inputs(260, 1, 2, D, dtype, seed=12)
    t["g"][:, [0, 70, 71, 128, 259]] = float("-inf")
    check(t, do, dhT)


def test_gradients_at_long_offsets():
    """More than 2^31 elements of each gradient: the last tokens against a call on them alone."""
    ha = _ha()
    T, H, D = 140_000, 128, 128
    if torch.cuda.mem_get_info()[0] < 140e9:
        pytest.skip("needs 140 GB")
    cu = torch.tensor([0, T - 300, T], dtype=torch.int32, device="cuda")
    x = torch.empty(1, T, H, D, dtype=torch.bfloat16, device="cuda").normal_()
    g = -torch.rand(1, T, H, device="cuda")
    got = ha.ha_la_gla_backward(x, x, x, x, g, cu_seqlens=cu, scale=0.01)
    s = lambda t: t[:, T - 300:].contiguous()
    want = ha.ha_la_gla_backward(s(x), s(x), s(x), s(x), s(g), scale=0.01)
    torch.cuda.synchronize()
    assert int(got[5].item()) == 0 and all(torch.equal(s(a), b) for a, b in zip(got[:4], want)) and torch.equal(got[4][1], want[4][0])


def test_decode_at_long_offsets():
    """More than 2^31 elements of state."""
    ha, N, H, D = _ha(), 1100, 128, 128
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB")
    state = torch.empty(N, H, D, D, device="cuda").normal_()
    q, k, v = (torch.randn(N, H, D, device="cuda").bfloat16() for _ in range(3))
    g = -torch.rand(N, H, device="cuda")
    tail = lambda t: t[-3:].clone()
    o2, h2 = ha.ha_la_gla_decode(*(tail(t) for t in (q, k, v, g)), tail(state))
    o, h = ha.ha_la_gla_decode(q, k, v, g, state)
    assert torch.equal(o[-3:], o2) and torch.equal(h[-3:], h2)
