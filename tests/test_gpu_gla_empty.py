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
