"""Packed batches of gated linear attention that hold nothing, or whose offsets are not offsets."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [(torch.float32, 64), (torch.float32, 128), (torch.bfloat16, 64), (torch.bfloat16, 128)],
                         ids=["fp32_64", "fp32_128", "bf16_64", "bf16_128"])
@pytest.mark.parametrize("N", [1, 2, 3, 200])
@pytest.mark.parametrize("HK,HV", [(1, 1), (1, 2), (2, 6)])
def test_packed_without_a_token(HK, HV, N, dtype, D):
    """The states pass through, forward and backward, q/k heads shared or not."""
    import paper_2609_32114_b200 as ha

    e = lambda *s: torch.empty(1, 0, *s, dtype=dtype, device="cuda")
    q, v, g = e(HK, D), e(HV, D), torch.empty(1, 0, HV, device="cuda")
    cu = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    h0, dhT = torch.randn(2, N, HV, D, D, device="cuda")
    o, hT, st, _ = ha.ha_la_gla_prefill(q, q, v, g, h0=h0, cu_seqlens=cu)
    dq, dk, dv, dg, dh0, st2, _ = ha.ha_la_gla_backward(v, q, q, v, g, h0=h0, dhT=dhT, cu_seqlens=cu)
    assert not ha.ha_la_gla_backward(v, q, q, v, g, cu_seqlens=cu)[4].any()
    torch.cuda.synchronize()
    assert int(st.item()) == 0 == int(st2.item())
    assert torch.equal(hT, h0) and torch.equal(dh0, dhT)
    assert all(x.numel() == 0 for x in (o, dq, dk, dv, dg))


@pytest.mark.parametrize("path", ["gla_fp32_64", "gla_fp32_128", "gla_bf16_64", "gla_bf16_128", "gdn_bf16_128", "kda_bf16_128", "gdn_fp32_64", "kda_fp32_128"])
@pytest.mark.parametrize("offsets", [[0, 1000] * 3, [0, 900, 100, 1000, 200, 1000]], ids=["three_times", "pieces"])
def test_sequences_that_overlap(offsets, path):
    """Offsets that go back, between sequences that fit by themselves and hold more chunks than there is room for: reported, nothing is written
    behind the workspace, states pass through, and the next call is as before."""
    import paper_2609_32114_b200 as ha

    op, dtype, D = path.split("_")
    D, T, HV, N = int(D), 1000, 2, 5
    gen = torch.Generator().manual_seed(D)
    r = lambda *s: torch.randn(*s, generator=gen)
    like = lambda *s: (r(*s) / D ** 0.5).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    q, k, v, do = like(1, T, 1, D), like(1, T, 1, D), like(1, T, HV, D), like(1, T, HV, D)
    g = -torch.rand(1, T, HV, D if op == "kda" else 1, generator=gen).cuda() * 0.1
    g = g if op == "kda" else g[..., 0].contiguous()
    beta = torch.rand(1, T, HV, generator=gen).cuda()
    h0, dhT = r(2, N, HV, D, D).cuda()
    bad, good = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in (offsets, [0, 10, 300, 300, 700, 1000]))
    if op == "gla":
        calls = [lambda cu, **kw: ha.ha_la_gla_prefill(q, k, v, g, h0=h0, cu_seqlens=cu, **kw),
                 lambda cu, **kw: ha.ha_la_gla_backward(do, q, k, v, g, h0=h0, dhT=dhT, cu_seqlens=cu, **kw)]
        status, states, room = [2, 5], [1, 4], [3, 6]
    else:
        calls = [lambda cu, **kw: ha.ha_la_prefill(q, k, v, g, beta, variant=op, h0=h0, cu_seqlens=cu, **kw)]
        status, states, room = [2], [1], [3]
    for call, st, h, ws, through in zip(calls, status, states, room, (h0, dhT)):
        want = call(good)
        torch.cuda.synchronize()
        need = want[ws].numel() - 256
        buffer = torch.full((need + (64 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
        assert buffer.data_ptr() % 256 == 0
        out = call(bad, workspace=buffer[:need])
        torch.cuda.synchronize()
        assert int(out[st].item()) == 6 and torch.equal(out[h], through)
        assert bool((buffer[need:] == 0x5A).all())
        again = call(good, workspace=buffer[:need])
        torch.cuda.synchronize()
        assert int(again[st].item()) == 0 and all(torch.equal(a, b) for i, (a, b) in enumerate(zip(again, want)) if i not in (st, ws))
