"""Attention over latent rows on the GPU against the 64-bit form.

Bounds, per element.  A score is a sum of up to 576 products in 32 bits, 40 roundings or truncations deep on the tensor cores and as many as there are channels on
the CUDA cores: 2^-23 each of the sum of magnitudes `top`, so s = 2^-17 top (40) or 2^-13 top (576).  lse: s + 2^-20 (1 + |lse|).  Outputs: weights are off by
2 s + 2^-18 and on the tensor cores by a rounding to bf16, 2^-8, of the sum of weights times |v|; then one rounding of the result."""
import math

import pytest
import torch

from tests import mixer_reference as ref
from tests.test_gpu_conv import ROUND, TYPES, off

pytestmark = pytest.mark.gpu


def _ha():
    import paper_2609_32114_b200 as ha

    return ha


def compare(o, lse, want, dtype, tc):
    w, wl, mag, top = want
    s = (2 ** -17 if tc else 2 ** -13) * top
    none = torch.isinf(wl)
    assert torch.equal(torch.isinf(lse.cpu()), none) and not o.cpu()[none].any()
    off("lse", torch.where(none, torch.zeros_like(wl), lse.double().cpu()), torch.where(none, torch.zeros_like(wl), wl), s + 2 ** -20 * (1 + wl.abs().nan_to_num(posinf=0, neginf=0)))
    off("o", o, w, ROUND[dtype] * w.abs() + ((2 ** -8 if tc else 0) + 2 ** -18 + 2 * s[:, None]) * mag)


# ---------------------------------------------------------------- prompts

def prompt(B, T, Tk, H, dims, dtype, cu=None, cuk=None, seed=0, layout="pair", pitch=0, size=2.0):
    dn, dr, dv = dims
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: (std * torch.randn(*s, generator=gen)).to(dtype).cuda()      # noqa: E731
    q = n(B, T, H * (dn + dr) + pitch, std=size)[..., :H * (dn + dr)].unflatten(-1, (H, dn + dr))
    if layout == "pair":                                     # a head's key and value side by side
        kv = n(B, Tk, H, dn + dv)
        kn, v = kv[..., :dn], kv[..., dn:]
    elif layout == "heads":                                  # head by head, B = 1
        kn, v = n(H, Tk, dn).transpose(0, 1)[None], n(H, Tk, dv).transpose(0, 1)[None]
    else:
        kn, v = n(B, Tk, H, dn), n(B, Tk, H, dv)
    kr = n(B, Tk, dr + pitch)[..., :dr]
    i = lambda c: None if c is None else torch.tensor(c, dtype=torch.int32, device="cuda")   # noqa: E731
    return dict(q=q, kn=kn, kr=kr, v=v, cu=i(cu), cuk=i(cuk), spans=ref.spans(T, cu, B), kspans=ref.spans(Tk, cuk if cuk is not None else cu, B))


def run_prompt(t, scale, **kw):
    return _ha().ha_la_latent_prefill(t["q"], t["kn"], t["kr"], t["v"], scale=scale, cu_seqlens=t["cu"], cu_seqlens_k=t["cuk"], **kw)


def check_prompt(t, scale=None, tc=None, heads=None):
    dtype, H, dq = t["q"].dtype, t["q"].shape[2], t["q"].shape[3]
    scale = dq ** -0.5 if scale is None else scale
    o, lse, status = run_prompt(t, scale)
    again = run_prompt(t, scale)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(o, again[0]) and torch.equal(lse, again[1])
    q, kn, kr, v = (ref.d(t[k]).flatten(0, 1) for k in ("q", "kn", "kr", "v"))
    fo, fl = o.reshape(-1, H, o.shape[-1]), lse.reshape(-1, H)
    for (a, n), (b, m) in zip(t["spans"], t["kspans"]):
        for h in heads or range(H):
            limit = (m - n + 1 + torch.arange(n)).clamp(0, m)
            want = ref.attend(q[a:a + n, h], torch.cat([kn[b:b + m, h], kr[b:b + m]], -1), v[b:b + m, h], limit, scale)
            compare(fo[a:a + n, h], fl[a:a + n, h], want, dtype, tc)


TC = (128, 64, 128)


@pytest.mark.parametrize("T", [1, 2, 63, 127, 128, 129, 200, 256, 257, 385])
def test_prompts_on_the_tensor_cores(T):
    check_prompt(prompt(2, T, T, 2, TC, torch.bfloat16, seed=T), tc=True)


def test_two_tiles_of_queries():
    """Enough heads and sequences that a CTA takes 256 queries."""
    check_prompt(prompt(3, 390, 390, 32, TC, torch.bfloat16, seed=1), tc=True, heads=[0, 13, 31])
    check_prompt(prompt(1, 1090, 1200, 40, TC, torch.bfloat16, seed=2, layout="apart"), tc=True, heads=[39])
    cu, cuk = [0, 100, 100, 357, 358, 700], [0, 130, 260, 517, 700, 900]
    check_prompt(prompt(1, 700, 900, 32, TC, torch.bfloat16, cu=cu, cuk=cuk, seed=3), tc=True, heads=[5, 30])


@TYPES
@pytest.mark.parametrize("cu,cuk", [([0, 1, 130, 130, 300], None), ([0, 3, 140], [0, 200, 400]), ([0, 40, 41, 200], [0, 10, 10, 169]), ([0, 0, 20], [0, 30, 30])], ids=str)
def test_packed_prompts(cu, cuk, dtype):
    """Prompts that go on from earlier keys, and queries in front of all keys, which see nothing."""
    t = prompt(1, cu[-1], (cuk or cu)[-1], 3, TC, dtype, cu=cu, cuk=cuk, seed=cu[1])
    check_prompt(t, tc=dtype == torch.bfloat16)


@pytest.mark.parametrize("layout", ["pair", "apart", "heads"])
@pytest.mark.parametrize("pitch", [0, 8, 4])
def test_layouts(layout, pitch):
    """(rows that are not 16 bytes apart go to the CUDA cores)"""
    t = prompt(1, 150, 150, 3, TC, torch.bfloat16, seed=pitch, layout=layout, pitch=pitch)
    check_prompt(t, tc=pitch % 8 == 0)


@TYPES
@pytest.mark.parametrize("dims", [(1, 0, 1), (16, 8, 24), (64, 0, 64), (128, 64, 128), (256, 128, 256), (33, 5, 65)], ids=str)
def test_other_heads(dims, dtype):
    t = prompt(2, 45, 70, 2, dims, dtype, seed=sum(dims))
    check_prompt(t, tc=dtype == torch.bfloat16 and dims == TC)


def test_large_scores_and_scales():
    """Scores of hundreds, whose maximum moves far while keys go by; a scale that is not positive."""
    t = prompt(1, 300, 300, 2, TC, torch.bfloat16, seed=4, size=60.0)
    t["q"] *= torch.linspace(0.1, 1, 300, device="cuda")[None, :, None, None].bfloat16()
    check_prompt(t, tc=True)
    check_prompt(prompt(1, 140, 140, 2, TC, torch.bfloat16, seed=5), scale=-0.05, tc=False)
    check_prompt(prompt(1, 140, 140, 2, TC, torch.bfloat16, seed=6), scale=0.0, tc=False)


@TYPES
def test_what_one_prompt_holds_stays_there(dtype):
    cu = [0, 100, 170, 300]
    t = prompt(1, 300, 300, 2, TC, dtype, cu=cu, seed=7)
    want = run_prompt(t, 0.07)
    for bad in (math.nan, math.inf):
        s = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
        for k in ("q", "kn", "kr", "v"):
            s[k][:, 100:170] = bad
        got = run_prompt(s, 0.07)
        for i in (0, 1):
            assert torch.equal(got[i][:, :100], want[i][:, :100]) and torch.equal(got[i][:, 170:], want[i][:, 170:])


def test_prompts_without_tokens_or_keys():
    ha = _ha()
    t = prompt(2, 0, 5, 2, TC, torch.bfloat16)
    assert run_prompt(t, 1.0)[0].shape == (2, 0, 2, 128)
    t = prompt(2, 5, 0, 2, TC, torch.bfloat16)
    o, lse, status = run_prompt(t, 1.0)
    assert not o.any() and bool((lse == -math.inf).all()) and int(status) == 0
    t = prompt(1, 50, 60, 2, TC, torch.bfloat16, cu=[0, 20, 50], cuk=[0, 20, 60])
    for cu, cuk in (([0, 20, 49], [0, 20, 60]), ([0, 20, 50], [0, 30, 20]), ([0, 20, 50], [0, 2 ** 31 - 1, 60]), ([0, 60, 50], [0, 20, 60])):
        s = dict(t, cu=torch.tensor(cu, dtype=torch.int32, device="cuda"), cuk=torch.tensor(cuk, dtype=torch.int32, device="cuda"))
        assert int(run_prompt(s, 1.0)[2]) == 6
    assert int(run_prompt(t, 1.0, max_seqlen=25)[2]) == 6
    assert ha.ha_la_latent_prefill_path(ha.ha_la_latent_prefill_args(dtype=0, batch=1, seqlen=1, seqlen_k=1, num_heads=1, d_nope=128, d_rope=64, d_v=128, scale=1.0)) == "tc"


# ---------------------------------------------------------------- new tokens on a paged cache

def tokens(lens, new, H, page, dtype, dims=(512, 64), seed=0, junk=math.nan, size=2.0):
    """Pages of all sequences mixed; rows behind a sequence's, and pages that nobody has, hold `junk`; entries behind the pages are out of range."""
    dl, dr = dims
    gen = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    total = sum(need) + 2
    order = torch.randperm(total, generator=gen)
    cache = torch.full((total, page, dl + dr), junk)
    table = torch.full((len(lens), max(need + [1]) + 1), 2 ** 31 - 1, dtype=torch.int32)
    at, rows = 0, []
    for i, n in enumerate(lens):
        r = torch.randn(n, dl + dr, generator=gen).to(dtype)
        rows.append(r)
        for j in range(need[i]):
            table[i, j] = order[at]
            part = r[j * page:(j + 1) * page]
            cache[order[at], :len(part)] = part.float()
            at += 1
    q = (size * torch.randn(len(lens), new, H, dl + dr, generator=gen)).to(dtype)
    return dict(q=q.cuda(), cache=cache.to(dtype).cuda(), table=table.cuda(), lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"), rows=rows, dl=dl)


def run_tokens(t, scale, **kw):
    return _ha().ha_la_latent_decode(t["q"], t["cache"], t["table"], t["lengths"], scale=scale, d_latent=t["dl"], **kw)


def check_tokens(t, scale=None, tc=None, sequences=None):
    dtype, (N, new, H, d) = t["q"].dtype, t["q"].shape
    scale = d ** -0.5 if scale is None else scale
    o, lse, status, ws = run_tokens(t, scale)
    again = run_tokens(t, scale, workspace=ws)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(o, again[0]) and torch.equal(lse, again[1])
    for n in range(N) if sequences is None else sequences:
        r = ref.d(t["rows"][n])
        limit = (len(r) - new + 1 + torch.arange(new)).clamp(min=0).repeat_interleave(H)
        want = ref.attend(ref.d(t["q"][n]).reshape(new * H, d), r, r[:, :t["dl"]], limit, scale)
        compare(o[n].reshape(new * H, -1), lse[n].reshape(-1), want, dtype, tc)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("H,new", [(1, 1), (16, 1), (8, 3), (32, 1), (33, 1), (64, 1), (128, 2)])
def test_new_tokens_on_the_tensor_cores(H, new, page):
    check_tokens(tokens([1, 70, 0, 300, 64, 17], new, H, page, torch.bfloat16, seed=H + page), tc=True)


@pytest.mark.parametrize("lens,H", [([5000], 16), ([9001], 128), ([3000, 1, 2000], 32), ([129] * 40, 20), ([64] * 300, 16), ([7] * 200 + [4000], 64)], ids=lambda x: str(x)[:20])
def test_parts_of_sequences(lens, H):
    """Contexts that several CTAs share, CTAs that have several contexts, more CTAs than there is work for."""
    check_tokens(tokens(lens, 1, H, 64, torch.bfloat16, seed=len(lens)), tc=True, sequences=range(0, len(lens), max(1, len(lens) // 6)))


def test_a_maximum_that_moves():
    """Scores that grow along the context, by far more than the outputs are held back for."""
    t = tokens([2000, 300], 1, 24, 64, torch.bfloat16, seed=3, size=1.0)
    for r, n in zip(t["rows"], (2000, 300)):
        r[:, 0] = torch.linspace(-30, 30, n).bfloat16()
    t["q"][..., 0] = 20
    for i, n in enumerate((2000, 300)):
        for j in range(-(-n // 64)):
            part = t["rows"][i][j * 64:(j + 1) * 64]
            t["cache"][int(t["table"][i, j]), :len(part)] = part.cuda()
    check_tokens(t, tc=True)


@TYPES
@pytest.mark.parametrize("dims,page", [((512, 64), 8), ((512, 64), 1), ((64, 0), 16), ((100, 28), 32), ((512, 128), 64), ((1, 1), 2)], ids=str)
def test_other_rows(dims, page, dtype):
    check_tokens(tokens([1, 70, 0, 45], 2, 5, page, dtype, dims=dims, seed=page), tc=False)


def test_fp32():
    check_tokens(tokens([33, 260, 1], 2, 16, 64, torch.float32, seed=1), tc=False)


def test_lengths_and_pages_that_do_not_exist():
    ha = _ha()
    for dtype in (torch.bfloat16, torch.float32):
        t = tokens([70, 130], 1, 4, 64, dtype, seed=2, junk=0.0)
        good = run_tokens(t, 0.1)
        for bad in ([70, -1], [70, 10 ** 6], [-2 ** 31, 130], [2 ** 31 - 1, 130]):
            s = dict(t, lengths=torch.tensor(bad, dtype=torch.int32, device="cuda"))
            o, lse, status, _ = run_tokens(s, 0.1)
            assert int(status) == 6
            for i in (0, 1):
                if bad[i] == (70, 130)[i]:
                    assert torch.equal(o[i], good[0][i])
                else:
                    assert not o[i].any() and bool((lse[i] == -math.inf).all())
        for entry in (-1, t["cache"].shape[0], 2 ** 31 - 1, -2 ** 31):
            s = dict(t, table=t["table"].clone())
            s["table"][1, 1] = entry
            o, _, status, _ = run_tokens(s, 0.1)
            assert int(status) == 6 and torch.equal(o[0], good[0][0])
        e = dict(t, cache=t["cache"][:0], lengths=torch.zeros(2, dtype=torch.int32, device="cuda"))
        o, lse, status, _ = run_tokens(e, 0.1)
        assert int(status) == 0 and not o.any()
        none = ha.ha_la_latent_decode(t["q"][:0], t["cache"], t["table"][:0], t["lengths"][:0])
        assert none[0].shape == (0, 1, 4, 512)


def test_a_long_cache():
    """Rows behind 2^31 elements."""
    if torch.cuda.mem_get_info()[0] < 30e9:
        pytest.skip("needs 30 GB")
    pages = 70_000
    cache = torch.empty(pages, 64, 576, dtype=torch.bfloat16, device="cuda").normal_()
    q = torch.randn(2, 1, 16, 576, device="cuda").bfloat16()
    table = torch.tensor([[pages - 1, pages - 2, 5], [0, pages // 2, pages - 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([190, 150], dtype=torch.int32, device="cuda")
    got = _ha().ha_la_latent_decode(q, cache, table, lengths, scale=0.05)
    small = cache[table.long().reshape(-1)].contiguous()
    want = _ha().ha_la_latent_decode(q, small, torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3), lengths, scale=0.05)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    del cache
    torch.cuda.empty_cache()
