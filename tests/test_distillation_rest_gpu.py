"""Distillation with the rest of the vocabulary as one more outcome, where all that is not listed lies far below the listed: its share of
the softmax is no number of 32 bits, and its logarithm is one all the same.  Against the formulas in 64 bits, from logarithms
throughout.

Tolerances, with u = 2^-24, z = x / T, a the listed, b the others, each group's exponentials relative to its own maximum (d below it):
  an exponential (8 + 4 d) u of itself, a sum of them those in their shares and V / 4096 + 60 units of u more (as in
      test_distillation_gpu); q (8 + 4 |t| + k) u of itself
  gap = log sum of all - log sum of b: 8 u of it (a difference, a quotient and two additions), and the sums' own
  loss: sum q |log p| (e_q + 8 u) + Q e_a + left (e_a + e_b + 8 u gap) + the error of left, sum q e_q, times gap
  gradient: dloss / T times, listed: p (Q e_p + e_left) + q (e_q + 8 u), e_p = its exponential's, the sum's and 4 u (4 + |z| + |m|);
      others: left r e_r + r e_left, e_r likewise with the gap up to 64, from where on it has no part in it; the output's rounding
"""
import pytest
import torch

import paper_1910_11971_gb300 as cci

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def check(dev, x, idx, value, dloss, T, dtype):
    N, V = x.shape
    k = idx.shape[1]
    z = x.double() / T
    valid = idx >= 0
    at = torch.where(valid, idx, V).long()
    on = torch.zeros((N, V + 1), dtype=torch.bool).scatter_(1, at, True)[:, :V]
    za, zb = torch.where(on, z, -INF), torch.where(on, -INF, z)
    la, lb = torch.logsumexp(za, 1), torch.logsumexp(zb, 1)
    ls = torch.logaddexp(la, lb)
    m = z.max(1).values
    q = torch.where(valid, torch.exp(value.double()), 0.0)
    left = (1.0 - q.sum(1)).clamp(min=0.0)
    Q = q.sum(1) + left
    wide = torch.cat([z, torch.zeros((N, 1), dtype=torch.float64)], 1)
    lp = torch.where(valid, wide.gather(1, at) - ls[:, None], 0.0)
    gap = ls - lb
    want = -(q * lp).sum(1) + left * gap

    def sums_error(zz):
        d = torch.where(zz == -INF, 0.0, zz.max(1, keepdim=True).values - zz)
        share = torch.softmax(zz, 1)  # from differences: 1e30 + log n is 1e30 in 64 bits, too
        return (8 + 4 * d) * U, (share * (8 + 4 * d) * U).sum(1) + (V / 4096 + 60) * U

    each_a, e_a = sums_error(za)
    each_b, e_b = sums_error(zb)
    e_q = (8 + 4 * torch.where(valid, value.double().abs(), 0.0) + k) * U
    e_left = (q * e_q).sum(1)
    tol = (q * lp.abs() * (e_q + 8 * U)).sum(1) + Q * (e_a + 8 * U) + left * (e_a + e_b + 8 * U * gap) + e_left * gap
    logits, lists = x.to(dev), (idx.to(dev), value.to(dev))
    loss, stats = cci.distillation_loss(logits, *lists, temperature=T, tail=True)
    diff = (loss.cpu().double() - want).abs()
    assert (diff <= tol).all(), float((diff / tol).max())
    dx = cci.distillation_loss_backward(dloss.to(dev), logits, *lists, stats, temperature=T, tail=True)
    w = (dloss.double() / T)[:, None]
    p, r = torch.softmax(z, 1), torch.softmax(zb, 1)
    target = torch.zeros((N, V + 1), dtype=torch.float64).scatter_add_(1, at, q)[:, :V]
    grad = w * (p * Q[:, None] - target - left[:, None] * r)
    e_p = torch.where(on, each_a, each_b) + e_a[:, None] + 4 * U * (4 + m.abs() + torch.where(on, z, 0.0).abs().amax(1))[:, None]
    e_r = each_b + e_b[:, None] + 4 * U * (4 + (m.abs() + gap).clamp(max=70.0))[:, None]
    bound = p * (Q[:, None] * e_p + e_left[:, None]) + r * (left[:, None] * e_r + e_left[:, None])
    bound += torch.zeros((N, V + 1), dtype=torch.float64).scatter_add_(1, at, q * (e_q + 8 * U))[:, :V]
    bound = w.abs() * bound + ((2.0 ** -8 if dtype == "bf16" else 0.0) + 4 * U) * grad.abs() + 1e-40
    diff = (dx.cpu().double() - grad).abs()
    assert (diff <= bound).all(), float((diff / bound).max())
    assert cci.distillation_loss_backward(dloss.to(dev), logits, *lists, stats, temperature=T, tail=True, out=logits) is logits
    assert torch.equal(logits, dx)


def inputs(N, V, k, below, T, dtype, seed):
    """Listed logits around 0, all others `below` temperatures lower, a spread of three; the teacher leaves 0.1 to 0.9 to them."""
    g = torch.Generator().manual_seed(seed)
    x = T * (3.0 * torch.rand((N, V), generator=g) - 3.0 - torch.as_tensor(below))
    idx = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(N)])
    x.scatter_(1, idx, T * torch.randn((N, k), generator=g))
    q = torch.rand((N, k), generator=g) + 0.1
    q = q / q.sum(1, keepdim=True) * (0.1 + 0.8 * torch.rand((N, 1), generator=g))
    return x.to(DTYPES[dtype]), idx.to(torch.int32), torch.log(q).contiguous(), torch.randn(N, generator=g)


SIZES = [(40, 900), (9, 20000), (300, 5000)]  # a warp, a cluster a row; rows that share blocks


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.1, 1.0, 2.0])
@pytest.mark.parametrize("below", [40.0, 63.0, 65.0, 80.0, 86.0, 100.0, 104.0, 1e3, 1e4, 1e6])
@pytest.mark.parametrize("N,V", SIZES)
def test_far_below(dev, N, V, below, T, dtype):
    check(dev, *inputs(N, V, 5, below, T, dtype, V + int(below)), T, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", SIZES)
def test_masks_that_are_numbers(dev, N, V, dtype):
    """All that is not listed masked, by the type's lowest value too; one of it left at -inf beside one that is not."""
    x, idx, value, dloss = inputs(N, V, 5, 10.0, 1.0, dtype, 7)
    free = torch.ones((N, V), dtype=torch.bool).scatter_(1, idx.long(), False)
    masks = torch.tensor([-1e4, -1e9, -1e30, torch.finfo(DTYPES[dtype]).min])
    some = torch.arange(N) % 5
    x = torch.where(free & (some < 4)[:, None], masks[some.clamp(max=3)][:, None].to(x.dtype), x)
    only = torch.where(free, -INF, x.float())
    last = (free * torch.arange(V)).argmax(1)
    only[torch.arange(N), last] = -500.0
    x = torch.where((some == 4)[:, None], only.to(x.dtype), x)
    loss, stats = cci.distillation_loss(x.to(dev), idx.to(dev), value.to(dev), tail=True)
    assert loss[some < 4].isfinite().all()
    check(dev, x, idx, value, dloss, 1.0, dtype)


@pytest.mark.parametrize("N,V", SIZES)
def test_a_full_teacher_leaves_nothing_to_them(dev, N, V):
    """q that add up to 1 or more: the rest has no part in the loss, however far it lies below."""
    x, idx, value, dloss = inputs(N, V, 2, 1e4, 1.0, "f32", 8)
    value = torch.log(torch.tensor([0.75, 0.5])).repeat(N, 1)
    check(dev, x, idx, value, dloss, 1.0, "f32")
