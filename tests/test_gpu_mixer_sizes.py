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
