"""Attention over latent rows: what a sequence's neighbour in the batch holds, finite and large, does not change one bit of its results.  (NaN and infinities, which
no comparison lets through, are elsewhere.)"""
import pytest
import torch

from tests.test_gpu_latent import TC, prompt, run_prompt, run_tokens, tokens

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


@pytest.mark.parametrize("H,new,lens", [(24, 1, (700, 500, 64)), (9, 1, (2000, 30, 500)), (5, 3, (300, 300, 300)), (40, 2, (1500, 200, 90)),
                                        (24, 1, (4000,) * 16), (9, 1, (4000, 3000) * 8), (5, 3, (2500,) * 24), (40, 2, (3000,) * 12)], ids=str)
def test_new_tokens_beside_large_queries(H, new, lens):
    """Heads fill up to 16, 32 or 64 columns; what fills the rest are the next sequence's.  Few sequences, a part of a context to a CTA; many, with several tiles
    one behind the other, between which the results may be rescaled."""
    t = tokens(list(lens), new, H, 64, torch.bfloat16, seed=H, junk=0.0)
    want = run_tokens(t, 0.05)
    for size in (0.0, 5.0, 100.0):
        for n in (0, 1, len(lens) // 2):
            s = dict(t, q=t["q"].clone())
            s["q"][:n] *= size
            s["q"][n + 1:] *= size
            got = run_tokens(s, 0.05)
            assert torch.equal(got[0][n], want[0][n]) and torch.equal(got[1][n], want[1][n]), (size, n)
