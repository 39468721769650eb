"""The norms' gradients where a row, or what takes a row's place, is far from ordinary; against the 64-bit plain form, with the bounds of
test_gpu_norm.py, which hold here as well: they are relative to the magnitude of a value's terms, and no step of the formulas needs a value
whose size is a higher power of the row's than the first."""
import pytest
import torch

from tests import layer_reference as ref
from tests import test_gpu_norm as norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 5, 37, 300])
@pytest.mark.parametrize("cols", [1, 8, 16, 17, 32])
@pytest.mark.parametrize("lift", [0, 1])
def test_places_without_a_row_without_eps(lift, cols, rows, dtype):
    """Several rows to a CTA, more places than rows, eps = 0: a place without a row has no norm, and adds nothing to the weights' gradients."""
    norm.gated(rows, cols, dtype, None, lift=lift, eps=0.0)
    norm.gated(rows, cols, dtype, "silu", lift=lift, eps=0.0)
    norm.added(rows, cols, dtype, True, lift=lift, eps=0.0)
    norm.added(rows, cols, dtype, False, lift=lift, eps=0.0)
