"""The norms around a block on the GPU against the 64-bit plain form.

Bounds, per element, of the magnitude M of the value's terms: one rounding of the result (bf16 2^-8, fp32 2^-24) and, for what is computed in
fp32 before it, 2^-17: sums over a row of up to 16384 values in threads of 16 and a tree (mean squares: 30 roundings of
2^-24), exponentials and quotients to 2^-21, a handful of products.  Sums over rows for the weights' gradients: 2^-24 for each row that a
thread adds, fewer than 64 here, and what each term is off."""
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

COLS = [1, 2, 7, 8, 9, 40, 64, 100, 127, 128, 129, 248, 249, 256, 257, 1000, 2048, 2049, 4096, 4100, 8192, 8200, 16383, 16384]


def _ha():
    import paper_2609_32114_b200 as ha

    return ha


def make(rows, cols, dtype, n, seed=0, lift=0):
    """n tensors of rows, `lift` elements behind a 16-byte boundary, and two weights."""
    gen = torch.Generator().manual_seed(seed)
    ts = []
    for _ in range(n):
        x = torch.randn(rows * cols + lift, generator=gen).to(dtype).cuda()[lift:].view(rows, cols)
        ts.append(x)
    return ts, [(1 + 0.2 * torch.randn(cols, generator=gen)).cuda() for _ in range(2)]


def close(name, got, want, magnitude, dtype, extra=2 ** -17):
    got, r = got.double().cpu(), {torch.bfloat16: 2 ** -8, torch.float32: 2 ** -24}[dtype]
    assert got.shape == want.shape and bool(torch.isfinite(got).all()), name
    off = (got - want).abs() - (r + extra) * magnitude - 1e-37
    assert bool((off <= 0).all()), (name, float(off.max()), int(off.argmax()))


def gated(rows, cols, dtype, name, lift=0, eps=1e-5, seed=0):
    ha = _ha()
    (x, z, dy), (w, _) = make(rows, cols, dtype, 3, seed=cols + rows, lift=lift)
    z = z if name else None
    kw = dict(activation=name or "silu", eps=eps)
    y = ha.ha_la_gated_norm(x, w, z, **kw)
    dx, dw, dz = ha.ha_la_gated_norm_backward(dy, x, w, z, **kw)
    torch.cuda.synchronize()
    want = ref.gated_norm(x, w, z, name, eps)
    close("y", y, want, want.abs(), dtype)
    grads = ref.gated_norm_backward(dy, x, w, z, name, eps)
    close("dx", dx, *grads["dx"], dtype)
    close("dw", dw, *grads["dw"], torch.float32)
    assert (dz is None) == (name is None)
    if name:
        close("dz", dz, *grads["dz"], dtype)


def added(rows, cols, dtype, post, lift=0, eps=1e-5, scale=0.7, given=True):
    ha = _ha()
    (x, r, dy, dr_out), (w, wp) = make(rows, cols, dtype, 4, seed=cols + rows, lift=lift)
    kw = dict(w_post=wp if post else None, scale=scale, eps=eps)
    y, r_out = ha.ha_la_add_norm(x, r, w, **kw)
    dr_out = dr_out if given else None
    dx, dr, dw, dwp = ha.ha_la_add_norm_backward(dy, dr_out, x, r_out, w, **kw)
    torch.cuda.synchronize()
    want_y, want_r, mag = ref.add_norm(x, r, w, kw["w_post"], scale, eps)
    close("r_out", r_out, want_r, mag, dtype)
    close("y", y, want_y, want_y.abs() + mag * ref.rms_scale(want_r, eps) * w.double().cpu().abs(), dtype)
    grads = ref.add_norm_backward(dy, dr_out, x, r_out, w, kw["w_post"], scale, eps)
    close("dr", dr, *grads["dr"], dtype)
    close("dx", dx, *grads["dx"], dtype)
    close("dw", dw, *grads["dw"], torch.float32)
    assert (dwp is None) == (not post)
    if post:
        close("dw_post", dwp, *grads["dw_post"], torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("cols", COLS)
def test_cols(cols, dtype):
    gated(5, cols, dtype, "silu")
    added(5, cols, dtype, True)
    added(3, cols, dtype, False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(1, 128), (1, 2048), (2, 64), (17, 33), (1111, 128), (20011, 129), (3001, 257), (1999, 2048), (4003, 1030)])
def test_rows(rows, cols, dtype):
    gated(rows, cols, dtype, "sigmoid")
    added(rows, cols, dtype, True, given=False)
    added(rows, cols, dtype, False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("cols", [8, 100, 128, 1030, 2048, 16384])
@pytest.mark.parametrize("lift", [1, 2, 4])
def test_off_a_boundary(lift, cols, dtype):
    gated(37, cols, dtype, None, lift=lift)
    gated(37, cols, dtype, "silu", lift=lift)
    added(37, cols, dtype, True, lift=lift)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_no_row_and_shapes(dtype):
    ha = _ha()
    w = torch.ones(64, device="cuda")
    e = torch.empty(0, 3, 64, dtype=dtype, device="cuda")
    assert ha.ha_la_gated_norm(e, w, e).shape == e.shape
    dx, dw, dz = ha.ha_la_gated_norm_backward(e, e, w, e, dw=torch.full((64,), 7.0, device="cuda"))
    assert dx.shape == e.shape and not dw.any()
    y, r = ha.ha_la_add_norm(e, e, w, w_post=w)
    out = ha.ha_la_add_norm_backward(e, None, e, e, w, w_post=w, dw_post=torch.full((64,), 7.0, device="cuda"))
    assert not out[2].any() and not out[3].any()
    x = torch.randn(2, 5, 3, 64, device="cuda").to(dtype)
    assert torch.equal(ha.ha_la_gated_norm(x, w, x), ha.ha_la_gated_norm(x.view(30, 64), w, x.view(30, 64)).view_as(x))
    assert torch.equal(ha.ha_la_gated_norm(x[0, 0, 0], w), ha.ha_la_gated_norm(x, w)[0, 0, 0])


@pytest.mark.parametrize("cols", [9, 128, 129, 1001])
def test_a_row_does_not_reach_another(cols):
    """NaN and infinities in every third row: the others' results are the same bits as without them."""
    ha = _ha()
    (x, z, dy, r), (w, wp) = make(40, cols, torch.bfloat16, 4)
    call = lambda: (ha.ha_la_gated_norm(x, w, z), *ha.ha_la_gated_norm_backward(dy, x, w, z)[::2], *ha.ha_la_add_norm(x, r, w, w_post=wp),
                    *ha.ha_la_add_norm_backward(dy, z, x, r, w, w_post=wp)[:2])
    clean = [t.clone() for t in call()]
    x[::3], z[::3], dy[::3], r[::3] = float("nan"), float("inf"), float("-inf"), float("nan")
    keep = torch.arange(40, device="cuda") % 3 != 0
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(clean, call()))


@pytest.mark.parametrize("cols", [128, 129, 2048, 2051])
def test_in_place(cols):
    ha = _ha()
    (x, z, dy, r), (w, wp) = make(333, cols, torch.bfloat16, 4)
    c = lambda t: t.clone()
    y = ha.ha_la_gated_norm(x, w, z)
    a = c(x)
    assert ha.ha_la_gated_norm(a, w, z, y=a) is a and torch.equal(a, y)
    a = c(z)
    assert torch.equal(ha.ha_la_gated_norm(x, w, a, y=a), y)
    dx, dw, dz = ha.ha_la_gated_norm_backward(dy, x, w, z)
    a, b = c(dy), c(z)
    g = ha.ha_la_gated_norm_backward(a, x, w, b, dx=a, dz=b)
    assert g[0] is a and g[2] is b and torch.equal(a, dx) and torch.equal(b, dz) and torch.equal(g[1], dw)
    a, b = c(x), c(dy)
    g = ha.ha_la_gated_norm_backward(b, a, w, z, dx=a, dz=b)
    assert torch.equal(a, dx) and torch.equal(b, dz)
    y, ro = ha.ha_la_add_norm(x, r, w, w_post=wp)
    a, b = c(x), c(r)
    assert ha.ha_la_add_norm(a, b, w, w_post=wp, y=a, r_out=b)[1] is b and torch.equal(a, y) and torch.equal(b, ro)
    want = ha.ha_la_add_norm_backward(dy, z, x, ro, w, w_post=wp)
    a, b = c(dy), c(z)
    got = ha.ha_la_add_norm_backward(a, b, x, ro, w, w_post=wp, dx=a, dr=b)
    assert got[0] is a and got[1] is b and all(torch.equal(p, q) for p, q in zip(want, got))


def test_extreme_gates_and_rows():
    ha = _ha()
    w = torch.ones(128, device="cuda")
    x = torch.randn(6, 128, device="cuda")
    z = torch.tensor([0.0, 88.0, 1000.0, -88.5, -1000.0, -60.0], device="cuda")[:, None].expand(6, 128).contiguous()
    for name in ("silu", "sigmoid"):
        y = ha.ha_la_gated_norm(x, w, z, activation=name)
        close(name, y, ref.gated_norm(x, w, z, name, 1e-6), ref.gated_norm(x, w, z, name, 1e-6).abs() + 1e-30, torch.float32)
        assert all(bool(torch.isfinite(t).all()) for t in ha.ha_la_gated_norm_backward(x, x, w, z, activation=name))
    zero = torch.zeros(3, 128, device="cuda")
    assert not ha.ha_la_gated_norm(zero, w, zero).any() and bool(torch.isfinite(ha.ha_la_gated_norm_backward(x[:3], zero, w, zero)[0]).all())
    tiny, huge = 1e-15 * x, 1e15 * x
    for s in (tiny, huge):
        close("y", ha.ha_la_gated_norm(s, w, eps=0.0), ref.gated_norm(s, w, None, None, 0.0), ref.gated_norm(s, w, None, None, 0.0).abs(), torch.float32)


def test_captured_and_on_another_stream():
    ha = _ha()
    (x, z, dy, r), (w, wp) = make(3000, 130, torch.bfloat16, 4)

    def call(**kw):
        return [ha.ha_la_gated_norm(x, w, z, **kw), *ha.ha_la_gated_norm_backward(dy, x, w, z, **kw), *ha.ha_la_add_norm(x, r, w, w_post=wp, **kw),
                *ha.ha_la_add_norm_backward(dy, z, x, r, w, w_post=wp, **kw)]

    first = [t.clone() for t in call()]
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        outs = call()
    for t in (x, z, dy, r):
        t.mul_(0.5)
    second = call()
    gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(second, outs)) and not torch.equal(first[0], second[0])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    there = call(stream=side.cuda_stream)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(second, there))


def test_many_elements():
    """More than 2^31 elements: the last rows against a call on them alone.  Where a row starts within 16 bytes decides which thread adds
    what, so both are roundings of values 2^-17 apart at most: two halves of a step, 2 x 2^-8, and that."""
    ha = _ha()
    rows, cols = 17_000_003, 129
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.rand(cols, device="cuda")
    tail = x[-1000:].contiguous()

    def near(a, b, magnitude):
        assert bool(((a[-1000:].float() - b.float()).abs() <= (2 ** -7 + 2 ** -16) * magnitude + 1e-30).all())

    y = ha.ha_la_gated_norm(x, w, x)
    near(y, ha.ha_la_gated_norm(tail, w, tail), y[-1000:].float().abs())
    dx, dw, dz = ha.ha_la_gated_norm_backward(x, x, w, x)
    a, _, c = ha.ha_la_gated_norm_backward(tail, tail, w, tail)
    grads = ref.gated_norm_backward(tail, tail, w, tail, "silu", 1e-6)
    near(dx, a, grads["dx"][1].float().cuda())
    near(dz, c, grads["dz"][1].float().cuda())
