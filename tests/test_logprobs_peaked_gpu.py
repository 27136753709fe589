"""Confident rows: one logit 10 to 39 above all others, wherever it stands.  The sum of exp(x - max) is at least 1, so
its logarithm and the entropy are not negative and no log probability is positive; for such rows both are small, and
their errors have to be small beside them.

Tolerances, u = 2^-24, s = 1 + r the sum, n = V / 512 + 64 the most additions on a term's way.  Adding to a number
that is at least 1 errs by at most u of it and by no more than what is added, so s is off by at most
min(n u (1 + r), r), and by the terms' own errors: each exponential within 8 u and, from its argument y, 4 |y| u, both
again for each of at most 16 larger maxima before the last (more maxima leave nothing of what came first).
  log s     min(n u (1 + r), r) + (128 + 4 Y) u r,  Y the largest |x - max| that counts (100)
  entropy   that, and (n + 128 + 4 Y) u of itself
  logp      log s' error and 4 u |logp|
"""
import math

import pytest
import torch

import paper_1910_11971_gb300 as cci

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows(V, dtype, seed):
    """A row for each gap and place of the high logit: at a thread's end of the row, its middle and its start."""
    g = torch.Generator().manual_seed(seed)
    places = [0, 1, V // 3, V // 2 + 5, V - 40, V - 9, V - 1]
    gaps = [10.0, 14.5, 20.0, 27.0, 33.0, 39.0]
    x = (0.5 * torch.randn((len(places) * len(gaps), V), generator=g)).to(DTYPES[dtype])
    at = torch.tensor([p for p in places for _ in gaps])
    x[torch.arange(len(at)), at] = torch.tensor(gaps * len(places)).to(DTYPES[dtype])
    return x, at


def rising(V, dtype, seed):
    """Rows whose maximum is passed again and again, in steps of up to 39 in all, the high part late."""
    g = torch.Generator().manual_seed(seed)
    x = (0.3 * torch.randn((12, V), generator=g))
    for i in range(12):
        x[i] += torch.linspace(0, 10.0 + 2.6 * i, V).round()
    x = x.to(DTYPES[dtype])
    return x, x.argmax(1)


def check(dev, x, t):
    V = x.shape[1]
    logp, h, stats, _, _ = (a.cpu().double() if a is not None else None for a in cci.token_logprobs(x.to(dev), t.to(dev)))
    assert (h >= 0).all(), float(h.min())
    assert (stats[:, 1] >= 0).all(), float(stats[:, 1].min())
    assert (logp <= 0).all(), float(logp.max())
    x = x.double()
    m = x.max(1, keepdim=True).values
    assert torch.equal(stats[:, 0], m[:, 0])
    y = x - m
    e = torch.exp(y)
    # r = s - 1 without cancellation
    top = torch.zeros_like(e).scatter_(1, x.argmax(1, keepdim=True), 1.0)
    r = (e * (1.0 - top)).sum(1)
    log_s = torch.log1p(r)
    lp = y - log_s[:, None]
    ref = -(torch.exp(lp) * lp).sum(1)
    n, terms = V / 512 + 64, (128 + 4 * 100) * U
    tol_s = torch.minimum(n * U * (1 + r), r) + terms * r
    assert ((stats[:, 1] - log_s).abs() <= tol_s + 2 * U * log_s).all()
    tol_h = tol_s + (terms + n * U) * ref
    assert ((h - ref).abs() <= tol_h).all(), float(((h - ref).abs() / tol_h).max())
    want = lp.gather(1, t[:, None])[:, 0]
    assert ((logp - want).abs() <= tol_s + 4 * U * want.abs()).all()


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


# rows held by a warp, four warps, a block, and a cluster of blocks
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 1500, 2048, 6001, 20001, 50001, 131072])
def test_one_high_logit(dev, V, dtype):
    x, at = rows(V, dtype, V)
    check(dev, x, at)
    check(dev, x, (at + V // 2) % V)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2048, 20001, 131072])
def test_many_rows(dev, V, dtype):
    """More rows than the SMs hold at once: a warp, and four warps, a row."""
    x, at = rows(V, dtype, V)
    n = 2500 if V == 2048 else 640
    many = x.to(dev).repeat(-(-n // len(x)), 1)[:n].contiguous()
    tokens = at.to(dev).repeat(-(-n // len(x)))[:n].contiguous()
    logp, h, stats, _, _ = cci.token_logprobs(many, tokens)
    assert (h >= 0).all() and (stats[:, 1] >= 0).all() and (logp <= 0).all()
    few = [a[:len(x)].cpu() for a in (logp, h, stats)]
    y = x.double() - x.double().max(1, keepdim=True).values
    top = torch.zeros_like(y).scatter_(1, at[:, None], 1.0)
    r = (torch.exp(y) * (1.0 - top)).sum(1)
    tol = torch.minimum((V / 512 + 64) * U * (1 + r), r) + (128 + 4 * 100) * U * r + 2 * U * r
    assert ((few[2][:, 1].double() - torch.log1p(r)).abs() <= tol).all()
    assert ((few[0].double() + torch.log1p(r)).abs() <= tol + 4 * U * r).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1500, 6001, 20001, 131072])
def test_rising_rows(dev, V, dtype):
    x, at = rising(V, dtype, V)
    logp, h, stats, _, _ = (a.cpu().double() if a is not None else None for a in cci.token_logprobs(x.to(dev), at.to(dev)))
    assert (h >= 0).all() and (stats[:, 1] >= 0).all() and (logp <= 0).all()
    y = x.double() - x.double().max(1, keepdim=True).values
    s = torch.exp(y).sum(1)
    assert (s > 1).all() and math.isfinite(float(s.max()))
    E = (V / 512 + 64 + 128 + 4 * 40) * U
    ref = torch.log(s) - (torch.exp(y) * y).sum(1) / s
    assert ((stats[:, 1] - torch.log(s)).abs() <= E * (1 + torch.log(s))).all()
    assert ((h - ref).abs() <= E * (2 + ref)).all()
