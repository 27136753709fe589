"""The gated block's activations at the ends of fp32."""
import pytest
import torch

import paper_1910_11971_gb300 as cci
from test_gated_tails_gpu import dev, forward_of, gradients_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", list(cci.ACTIVATIONS))
def test_far_out(dev, act):
    """Values whose squares and cubes leave fp32: act is g, 0 or 1 and act' 0 or 1 there, exactly."""
    far = torch.tensor([1e3, 1e10, 1.8e19, 1.9e19, 1e20, 1e30, 1e38, 3.4e38], device=dev)
    g = torch.cat([far, -far])
    up = (g > 0).double()
    want = up if act == "sigmoid" else up * g.double()
    slope, value = gradients_of(g, act, dev)
    assert torch.equal(slope, up * (0.0 if act == "sigmoid" else 1.0))
    # as operands of the gradients' products the values are three bf16: within 2^-23
    assert ((value - want).abs() <= 2.0 ** -23 * want.abs()).all()
    h = forward_of(g[g.abs() < 1e30], act, dev)
    want = want[g.abs() < 1e30]
    assert ((h - want).abs() <= 2.0 ** -23 * want.abs()).all()
