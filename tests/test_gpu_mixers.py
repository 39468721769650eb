"""The layers that alternate with the recurrences, run together as a model runs them: a prompt, then token by token; captured and replayed; on another stream; two at once."""
import pytest
import torch

from tests import mixer_reference as ref
from tests.test_gpu_conv import off
from tests.test_gpu_latent import run_tokens, tokens

pytestmark = pytest.mark.gpu


def _ha():
    import paper_2609_32114_b200 as ha

    return ha


# ---------------------------------------------------------------- convolution and scan: a state space layer

def layer_weights(ch, S, G, seed):
    gen = torch.Generator().manual_seed(seed)
    f = lambda *s, std=1.0: (std * torch.randn(*s, generator=gen)).cuda()      # noqa: E731
    return dict(w=f(ch, 4, std=0.5), bias=f(ch), A=-f(ch, S).abs(), D=f(ch), dt_bias=f(ch) - 2, proj=f(ch, ch + 2 * G * S, std=ch ** -0.5)), gen


def state_space(ha, p, xz, ch, S, G, conv0, h0, cu=None):
    """xz [1, T, 2 ch]: x and z as halves of one projection; dt, B and C as slices of another one."""
    x, z = xz[..., :ch], xz[..., ch:]
    u, conv, s1 = ha.ha_la_conv(x, p["w"], bias=p["bias"], h0=conv0, cu_seqlens=cu)
    pr = u @ p["proj"].to(u.dtype)
    B, C = (pr[..., ch + i * G * S:ch + (i + 1) * G * S].unflatten(-1, (G, S)) for i in (0, 1))
    y, h, s2, _ = ha.ha_la_scan(u, pr[..., :ch], p["A"], B, C, D=p["D"], z=z, dt_bias=p["dt_bias"], h0=h0, cu_seqlens=cu)
    assert int(s1) == 0 == int(s2)
    return y, conv, h


def state_space_token(ha, p, xz, ch, S, G, conv, h):
    u, conv = ha.ha_la_conv_decode(xz[:, :ch], p["w"], conv, bias=p["bias"])
    pr = u @ p["proj"].to(u.dtype)
    B, C = (pr[..., ch + i * G * S:ch + (i + 1) * G * S].unflatten(-1, (G, S)) for i in (0, 1))
    y, h = ha.ha_la_scan_decode(u, pr[:, :ch], p["A"], B, C, h, D=p["D"], z=xz[:, ch:], dt_bias=p["dt_bias"])
    return y, conv, h


def test_a_state_space_layer_prompt_and_tokens():
    """fp32: 20 tokens at once, and 17 followed by three one by one.  Both ways round the same sums differ by 2^-24 of their terms in each of the layer's some forty
    operations on a value, the projection's ch-term products among them: 2^-12 of the largest output is far above it and far below any real difference."""
    ha, N, ch, S, G = _ha(), 3, 48, 16, 2
    p, gen = layer_weights(ch, S, G, 1)
    xz = torch.randn(1, 20 * N, 2 * ch, generator=gen).cuda()
    conv0, h0 = torch.randn(N, 3, ch, generator=gen).cuda(), torch.randn(N, ch, S, generator=gen).cuda()
    cu = lambda n: torch.tensor([n * i for i in range(N + 1)], dtype=torch.int32, device="cuda")     # noqa: E731
    want, conv_w, h_w = state_space(ha, p, xz, ch, S, G, conv0, h0, cu(20))
    rows = xz.view(N, 20, 2 * ch)
    y, conv, h = state_space(ha, p, rows[:, :17].reshape(1, 17 * N, 2 * ch).contiguous(), ch, S, G, conv0, h0, cu(17))
    near = lambda a, b: float((a - b).abs().max()) <= 2 ** -12 * float(b.abs().max())                # noqa: E731
    assert near(y.view(N, 17, ch), want.view(N, 20, ch)[:, :17])
    for t in (17, 18, 19):
        y, conv, h = state_space_token(ha, p, rows[:, t].contiguous(), ch, S, G, conv, h)
        assert near(y, want.view(N, 20, ch)[:, t])
    assert torch.equal(conv, conv_w) and near(h, h_w)


def test_gradients_through_the_layer():
    """Of the convolution and the scan one behind the other, against the 64-bit form differentiated: errors of the scan's dx pass through the convolution's transpose."""
    ha, T, ch, S = _ha(), 33, 24, 16
    gen = torch.Generator().manual_seed(3)
    f = lambda *s: torch.randn(*s, generator=gen)            # noqa: E731
    x, w, dt, A, B, C, dy = f(1, T, ch), f(ch, 4), f(1, T, ch) - 2, -f(ch, S).abs(), f(1, T, 1, S), f(1, T, 1, S), f(1, T, ch)
    g = [t.cuda() for t in (x, w, dt, A, B, C, dy)]
    u, _, _ = ha.ha_la_conv(g[0], g[1])
    du, *_ = ha.ha_la_scan_backward(g[6], u, g[2], g[3], g[4], g[5])
    dx, dw, *_ = ha.ha_la_conv_backward(du, g[0], g[1])
    xs, ws = x[0].double().requires_grad_(), w.double().requires_grad_()
    us, _, _ = ref.conv(xs, ws, None, None, True, [(0, T)])
    y, _, _, _ = ref.scan(us, dt[0].double(), A.double(), B[0].double(), C[0].double(), None, None, None, True, None, [(0, T)])
    want = torch.autograd.grad(y, [xs, ws], dy[0].double())
    for got, ww in ((dx[0], want[0]), (dw, want[1])):
        off("gradient", got, ww, 2 ** -12 * ww.abs().max())


# ---------------------------------------------------------------- latent attention: both forms

def test_absorbed_tokens_are_the_prompt_s_last():
    """A prompt by the expanded form; its last tokens by the absorbed one, from a cache of the same latent rows.  Everything but the products around is the library's."""
    ha, H, T, new, page = _ha(), 16, 150, 3, 64
    gen = torch.Generator().manual_seed(5)
    n = lambda *s, std=1.0: std * torch.randn(*s, generator=gen).cuda()        # noqa: E731
    c, kr = n(T, 512), n(T, 64).bfloat16()
    uk, uv = n(H, 128, 512, std=512 ** -0.5), n(H, 128, 512, std=512 ** -0.5)
    q = n(1, T, H, 192).bfloat16()
    cb = c.bfloat16().float()
    kn, v = torch.einsum("tc,hdc->thd", cb, uk).bfloat16(), torch.einsum("tc,hdc->thd", cb, uv).bfloat16()
    o, lse, status = ha.ha_la_latent_prefill(q, kn[None], kr[None], v[None], scale=192 ** -0.5)
    cache = torch.zeros(4, page, 576, device="cuda").bfloat16()
    rows = torch.cat([c.bfloat16(), kr], -1)
    for j, pg in enumerate((2, 0, 3)):
        part = rows[j * page:(j + 1) * page]
        cache[pg, :len(part)] = part
    qa = torch.cat([torch.einsum("thd,hdc->thc", q[0, -new:, :, :128].float(), uk), q[0, -new:, :, 128:].float()], -1).bfloat16()
    oa, la, s2, _ = ha.ha_la_latent_decode(qa[None], cache, torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda"),
                                           torch.tensor([T], dtype=torch.int32, device="cuda"), scale=192 ** -0.5)
    back = torch.einsum("ihc,hdc->ihd", oa[0].float(), uv)
    assert int(status) == 0 == int(s2)
    # keys, values and absorbed queries are rounded to bf16 on one side and not on the other: scores differ by some 192 products off by 2^-8 each
    assert float((la[0] - lse[0, -new:]).abs().max()) < 0.1 and float((back - o[0, -new:].float()).abs().max()) < 0.1 * float(o.float().abs().max())


# ---------------------------------------------------------------- streams, captured calls

def everything(seed, T=300):
    """One call of each entry point on its own buffers; returns (run, outputs)."""
    ha = _ha()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s, dt=torch.bfloat16: torch.randn(*s, generator=gen, device="cuda").to(dt)     # noqa: E731
    f = lambda *s: torch.randn(*s, generator=gen, device="cuda")                               # noqa: E731
    ch, S = 64, 16
    x, dt, z, dy, B, C = n(1, T, ch), n(1, T, ch), n(1, T, ch), n(1, T, ch), n(1, T, 1, S), n(1, T, 1, S)
    w, bias, A, D = f(ch, 4), f(ch), -f(ch, S).abs(), f(ch)
    cu = torch.tensor([0, T // 3, T], dtype=torch.int32, device="cuda")
    q, kn, kr, v = n(1, T, 4, 192), n(1, T, 4, 128), n(1, T, 64), n(1, T, 4, 128)
    tok = tokens([T, 70], 1, 8, 32, torch.bfloat16, seed=seed, junk=0.0)
    st, h = n(2, 3, ch), f(2, ch, S)
    keep = {}

    def run(stream=None):
        kw = dict(stream=stream)
        keep["conv"] = ha.ha_la_conv(x, w, bias=bias, cu_seqlens=cu, **kw)[:2]
        keep["conv_back"] = ha.ha_la_conv_backward(dy, x, w, bias=bias, cu_seqlens=cu, **kw)[:4]
        keep["scan"] = ha.ha_la_scan(x, dt, A, B, C, D=D, z=z, cu_seqlens=cu, **kw)[:2]
        keep["scan_back"] = ha.ha_la_scan_backward(dy, x, dt, A, B, C, D=D, z=z, cu_seqlens=cu, **kw)[:9]
        keep["conv_token"] = ha.ha_la_conv_decode(x[0, :2], w, st, state_out=torch.empty_like(st), **kw)
        keep["scan_token"] = ha.ha_la_scan_decode(x[0, :2], dt[0, :2], A, B[0, :2], C[0, :2], h, state_out=torch.empty_like(h), **kw)
        keep["prompt"] = ha.ha_la_latent_prefill(q, kn, kr, v, scale=0.07, cu_seqlens=cu, **kw)[:2]
        keep["tokens"] = run_tokens(tok, 0.05, **kw)[:2]
        return [t for k in keep for t in keep[k] if t is not None]

    return run, [x, dt, z, dy, q, kn, v, tok["q"], tok["cache"], st, h]


def test_captured_and_replayed():
    """Two graphs of the same calls in one process, replayed in turn on new contents, against eager calls."""
    graphs = []
    for seed in (1, 2):
        run, ins = everything(seed, T=300 if seed == 1 else 700)
        run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = run()
        graphs.append((g, run, ins, outs))
    for scale in (1.0, 0.5, 2.0):
        for g, run, ins, outs in graphs:
            for t in ins:
                t.mul_(scale)
            g.replay()
        torch.cuda.synchronize()
        for g, run, ins, outs in graphs:
            have = [t.clone() for t in outs]
            want = run()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(have, want))


def test_on_another_stream_and_two_at_once():
    runs = [everything(s)[0] for s in (3, 4)]
    want = [[t.clone() for t in r()] for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    got = []
    for r, s in zip(runs, streams):                          # by argument
        got.append([t for t in r(stream=s.cuda_stream)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))
    got = []
    for r, s in zip(runs, streams):                          # as the current one
        with torch.cuda.stream(s):
            got.append(r())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))


def test_native_and_python_marshalling_agree(monkeypatch):
    """The same calls with the native half answering that they are not ordinary."""
    from paper_2609_32114_b200 import binding

    run, _ = everything(5)
    want = [t.clone() for t in run()]

    class Nothing:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(binding, "_native", lambda: Nothing())
    got = run()
    torch.cuda.synchronize()
    assert len(want) == len(got) and all(torch.equal(a, b) for a, b in zip(want, got))
