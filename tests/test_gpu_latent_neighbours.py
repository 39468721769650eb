"""Attention over latent rows: what a sequence's neighbour in the batch holds, finite and large, does not change one bit of its results.  (NaN and infinities, which
no comparison lets through, are elsewhere.)"""
import pytest
import torch

from tests.test_gpu_latent import TC, prompt, run_prompt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,first", [(2, 200), (2, 333), (40, 200), (40, 1000)])
def test_prompts_beside_large_queries(H, first):
    """The last tile's rows behind the sequence are the next one's queries, here with scores that leave any maximum of before far behind."""
    cu = [0, first, first + 150]
    t = prompt(1, cu[-1], cu[-1], H, TC, torch.bfloat16, cu=cu, seed=first)
    want = run_prompt(t, 0.07)
    for size in (0.0, 5.0, 100.0):
        s = dict(t, q=t["q"].clone())
        s["q"][:, first:] *= size
        got = run_prompt(s, 0.07)
        assert torch.equal(got[0][:, :first], want[0][:, :first]) and torch.equal(got[1][:, :first], want[1][:, :first]), size
