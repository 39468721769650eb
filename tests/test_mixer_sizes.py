"""The mixers' host-only answers at the largest sizes that the library takes: nothing wraps round.  No GPU."""
import pytest

import paper_2609_32114_b200 as ha
from paper_2609_32114_b200 import build, mixer

MOST = 2 ** 31 - 257                                         # tokens of a call


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return ha.load_library()


@pytest.mark.parametrize("channels", [1, 8])
@pytest.mark.parametrize("tokens", [2 ** 31 - 513, 2 ** 31 - 512, 2 ** 31 - 511, MOST])
def test_convolution_of_the_most_tokens(tokens, channels):
    """The gradients' runs are up to 512 tokens long, each with five sums a channel in 32 bits."""
    have = ha.ha_la_conv_workspace_bytes(mixer.ha_la_conv_args(dtype=0, batch=1, seqlen=tokens, channels=channels, taps=4, activation=0))
    assert have >= -(-tokens // 512) * 5 * channels * 4


@pytest.mark.parametrize("tokens,channels,groups", [(2_100_000_000, 4, 4), (2_132_000_000, 1, 1), (MOST, 1, 1), (MOST, 4, 4), (MOST, 18, 18)])
def test_scan_of_the_most_tokens(tokens, channels, groups):
    """Few channels are cut into segments, two and a half times as many as SMs at the most, each with a state of up to 16 and a sum of steps a channel."""
    args = mixer.ha_la_scan_args(dtype=0, batch=1, seqlen=tokens, channels=channels, states=1, groups=groups, softplus=1)
    have = ha.ha_la_scan_workspace_bytes(args)
    assert 2 * channels * 17 * 4 <= have <= 400 * channels * 17 * 4 + 1024
    assert ha.ha_la_scan_workspace_bytes(args, backward=True) >= tokens // 8 * channels * 16 * 4
