"""Distillation where a student is sure of a token that its teacher does not list: the sum of its exponentials is a 1 and next to
nothing, which two roundings take to the other side of 1 for some maxima and not for others, and the sign of that sum's logarithm is
what tells the gradient how the maximum is held.  Hundreds of maxima, therefore, on both sides of 0 and of 64 temperatures, in each
of the kernels; formulas and tolerances are those of test_distillation_gpu."""
import pytest
import torch

import paper_1910_11971_gb300 as cci
from test_distillation_gpu import DTYPES, check_shifted, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def sure_rows(N, V, k, T, tail, dtype, seed):
    """Logits, lists, the gradient of the losses: the largest logit of a row lies 20 to 60 temperatures above all others and is not
    listed; every eighth row lists nothing."""
    g = torch.Generator().manual_seed(seed)
    top = (40.0 + 40.0 * torch.rand((N, 1), generator=g)) * T * torch.where(torch.arange(N)[:, None] % 2 > 0, -1.0, 1.0)
    gap = (20.0 + 40.0 * torch.rand((N, 1), generator=g)) * T
    x = top - gap - T * torch.rand((N, V), generator=g)
    order = torch.stack([torch.randperm(V, generator=g)[:k + 1] for _ in range(N)])
    x.scatter_(1, order[:, k:], top)
    idx = order[:, :k].to(torch.int32).contiguous()
    idx[3::8] = -1
    value = torch.log(torch.full((N, k), 0.7 / k)) if tail else torch.randn((N, k), generator=g)
    return x.to(DTYPES[dtype]), idx, value.contiguous(), torch.randn(N, generator=g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [0.5, 0.7, 1.0, 2.0, 3.0])
@pytest.mark.parametrize("N,V", [(600, 900), (57, 5000), (400, 5000)])
def test_sure_of_an_unlisted_token(dev, N, V, T, tail, dtype):
    k = 5
    for seed in range(1 if N > 57 else 8):
        x, idx, value, dloss = sure_rows(N, V, k, T, tail, dtype, V + seed)
        apart = (x.double() - x.double().max(1, keepdim=True).values) / T
        apart_value = value.double() if tail else value.double() / T
        f = reference(apart, idx, apart_value, 1.0, tail)
        logits, lists = x.to(dev), (idx.to(dev), value.to(dev))
        _, stats = cci.distillation_loss(logits, *lists, temperature=T, tail=tail)
        dx = cci.distillation_loss_backward(dloss.to(dev), logits, *lists, stats, temperature=T, tail=tail)
        assert (dx[3::8] == 0).all()
        check_shifted(logits, lists, dloss, T, tail, dtype, f)


def test_two_at_the_top(dev):
    """The largest logit twice, listed once: p is a half each, whatever the maximum."""
    N, V = 500, 700
    g = torch.Generator().manual_seed(2)
    for T in (0.7, 2.0):
        x = torch.zeros((N, V)) - 90.0 * T
        top = (torch.rand(N, generator=g) - 0.5) * 200.0 * T
        x += top[:, None]
        x[:, 5], x[:, 600] = top, top
        idx, value = torch.full((N, 1), 5, dtype=torch.int32), torch.zeros((N, 1))
        loss, stats = cci.distillation_loss(x.to(dev), idx.to(dev), value.to(dev), temperature=T)
        dx = cci.distillation_loss_backward(torch.full((N,), T, device=dev), x.to(dev), idx.to(dev), value.to(dev), stats, temperature=T).cpu()
        # log 2 and the half: the two exponentials by 2 units of 2 u each, and the same of the sum, its logarithm's, the quotient's
        assert ((loss.cpu() - 0.6931471805599453).abs() <= 32 * 2.0 ** -24).all()
        assert ((dx[:, 600] - 0.5).abs() <= 32 * 2.0 ** -24).all() and ((dx[:, 5] + 0.5).abs() <= 32 * 2.0 ** -24).all()
