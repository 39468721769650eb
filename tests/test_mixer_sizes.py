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
