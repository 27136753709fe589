"""The gated block's GELU where it is small."""
import math

import pytest
import torch

import paper_1910_11971_gb300 as cci

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def forward_of(g, act, dev):
    """act(g): g itself is the product of one column with a weight of 1, u = 1.  g is whole in three bf16 planes."""
    n = g.numel()
    x = torch.zeros((n, 8), device=dev)
    x[:, 0], x[:, 1] = g, 1.0
    one, up = torch.zeros((8, 8), device=dev), torch.zeros((8, 8), device=dev)
    one[:, 0], up[:, 1] = 1.0, 1.0
    h = cci.gated_linear(x, one, up, act=act)
    assert (h == h[:, :1]).all()
    return h[:, 0].double()


def gradients_of(g, act, dev):
    """(act'(g), act(g)) as the backward pass takes them: dh = u = 1, one of the weights an identity, the other 0."""
    n = g.numel()
    gm = g.view(-1, 8).contiguous()
    rows = gm.shape[0]
    x = torch.zeros((rows, 8), device=dev)
    ones = torch.ones_like(gm)
    eye, zero = torch.eye(8, device=dev), torch.zeros((8, 8), device=dev)
    slope, _, _ = cci.gated_linear_backward(ones, x, eye, zero, gm, ones, act=act, need_dw=False)
    value, _, _ = cci.gated_linear_backward(ones, x, zero, eye, gm, ones, act=act, need_dw=False)
    return slope.double().reshape(n), value.double().reshape(n)


def test_gelu_keeps_its_relative_accuracy(dev):
    """gelu(g) = g Phi(g) for negative g, to where fp32 ends.  Phi(-a) = e^(-a^2 / 2) R(a): R by a polynomial, within
    2^-21; the exponential within 2 + 1.173 a^2 / 2 units of 2^-23 (CUDA's documented error of its fast form) and its
    argument within a^2 / 2 half units; four products around them.  So (4 + 2 + 0.84 a^2 + 4) 2^-23 of the value, with
    0.16 a^2 for the rest of the argument's roundings; below 2^-100 it may be 0."""
    g = torch.cat([-torch.linspace(0, 13, 8184), torch.tensor([-1e-6, -1e-3, -0.75, -1.0, -5.0, -6.0, -8.0, -11.5])]).to(dev)
    a = g.double()
    ref = a * torch.special.erfc(-a / math.sqrt(2.0)) * 0.5
    tol = (10 + a * a) * 2.0 ** -23 * ref.abs() + 2.0 ** -100
    h = forward_of(g, "gelu", dev)
    assert ((h - ref).abs() <= tol).all(), float(((h - ref).abs() / ref.abs().clamp(min=2.0 ** -100)).max())
    slope, value = gradients_of(g, "gelu", dev)
    assert ((value - ref).abs() <= tol).all()
    phi = torch.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi)
    cdf = torch.special.erfc(-a / math.sqrt(2.0)) * 0.5
    # Phi + g phi cancels near -0.75: the error is that of the two terms
    assert ((slope - (cdf + a * phi)).abs() <= (10 + a * a) * 2.0 ** -23 * (cdf + a.abs() * phi) + 2.0 ** -100).all()


def test_gelu_above_zero(dev):
    """Phi(g) = 1 - Phi(-g), half at least: the same 2^-21 and roundings, without the exponential's share."""
    g = torch.cat([torch.linspace(0, 13, 8184), torch.tensor([1e-6, 1e-3, 0.75, 1.0, 5.0, 20.0, 100.0, 1e4])]).to(dev)
    ref = g.double() * torch.special.ndtr(g.double())
    tol = 10 * 2.0 ** -23 * ref.abs() + 2.0 ** -100
    h = forward_of(g, "gelu", dev)
    assert ((h - ref).abs() <= tol).all(), float(((h - ref).abs() / tol).max())
    _, value = gradients_of(g, "gelu", dev)
    assert ((value - ref).abs() <= tol).all()
