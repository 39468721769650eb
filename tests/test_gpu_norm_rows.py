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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("cols", [16, 128, 1000, 2048, 8200])
@pytest.mark.parametrize("lift", [0, 1])
@pytest.mark.parametrize("size", [1e-17, 1e-14, 1e13, 1e15, 1e17])
def test_rows_far_from_one(size, lift, cols, dtype):
    """Mean squares that fp32 holds, gradients too; only products of three norms would not be."""
    ha = norm._ha()
    (x, r, z, dy, dr_out), (w, wp) = norm.make(9, cols, dtype, 5, seed=cols, lift=lift)
    x.mul_(size)
    r.mul_(size)
    dr_out.mul_(1 / size)                                  # (as large as what the norm adds to it)
    for name in (None, "silu"):
        kw = dict(activation=name or "silu", eps=0.0)
        dx, dw, dz = ha.ha_la_gated_norm_backward(dy, x, w, z if name else None, **kw)
        grads = ref.gated_norm_backward(dy, x, w, z if name else None, name, 0.0)
        norm.close("dx", dx, *grads["dx"], dtype)
        norm.close("dw", dw, *grads["dw"], torch.float32)
        if name:
            norm.close("dz", dz, *grads["dz"], dtype)
    for post in (None, wp):
        for given in (None, dr_out):
            dx, dr, dw, dwp = ha.ha_la_add_norm_backward(dy, given, x, r, w, w_post=post, scale=0.7, eps=0.0)
            grads = ref.add_norm_backward(dy, given, x, r, w, post, 0.7, 0.0)
            norm.close("dr", dr, *grads["dr"], dtype)
            norm.close("dx", dx, *grads["dx"], dtype)
            norm.close("dw", dw, *grads["dw"], torch.float32)
            if post is not None:
                norm.close("dw_post", dwp, *grads["dw_post"], torch.float32)
