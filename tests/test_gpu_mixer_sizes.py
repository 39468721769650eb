"""The mixers' kernels at the largest sizes that the library takes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_convolution_gradients_of_the_most_tokens():
    """Ones everywhere: every sum is a whole number, exact in runs of 512 and in 64 bits, and rounded once."""
    import paper_2609_32114_b200 as ha

    T = 2 ** 31 - 257
    if torch.cuda.mem_get_info()[0] < 20e9:
        pytest.skip("needs 20 GB")
    x = torch.ones(1, T, 1, dtype=torch.bfloat16, device="cuda")
    w = torch.tensor([[1.0, 2.0, 4.0, 8.0]], device="cuda")
    dx, dw, db, dh0, status, _ = ha.ha_la_conv_backward(x, x, w, bias=torch.zeros(1, device="cuda"), activation=None)
    assert int(status) == 0 and bool((dx[0, :-3] == 15).all()) and dx[0, -3:, 0].tolist() == [14, 12, 8]
    assert dw[0].double().tolist() == torch.tensor([T - 3, T - 2, T - 1, T], dtype=torch.float64).float().double().tolist()
    assert float(db) == float(torch.tensor(T, dtype=torch.float64).float()) and dh0[0, :, 0].tolist() == [1, 3, 7]
    del x, dx
    torch.cuda.empty_cache()


def test_lengths_that_row_numbers_do_not_reach():
    """A table may name a page as often as it likes, so that its row holds 2^31 cached rows; a length whose last tile would pass 2^31 counts as zero."""
    import paper_2609_32114_b200 as ha

    page = 1 << 20
    if torch.cuda.mem_get_info()[0] < 10e9:
        pytest.skip("needs 10 GB")
    cache = torch.zeros(2, page, 576, dtype=torch.bfloat16, device="cuda")
    cache[0, :100] = torch.randn(100, 576, device="cuda").bfloat16()
    q = torch.randn(2, 1, 16, 576, device="cuda").bfloat16()
    table = torch.zeros(2, 2048, dtype=torch.int32, device="cuda")
    want = ha.ha_la_latent_decode(q, cache, table, torch.tensor([100, 0], dtype=torch.int32, device="cuda"), scale=0.05)
    for length in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 255):
        got = ha.ha_la_latent_decode(q, cache, table, torch.tensor([100, length], dtype=torch.int32, device="cuda"), scale=0.05)
        assert int(got[2]) == 6 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
