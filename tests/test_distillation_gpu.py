"""Distillation from a teacher's top logits against the formulas in 64 bits, and its gradient against differences.

Tolerances, with u = 2^-24, z = x / T, d = max z - z:
  an exponential of z - max z: (8 + 4 d) u of it (2 units of 2 u for the function, the rest for its argument: the difference,
      the factor and their product round, and the maximum's division by T)
  the sums of exponentials: each one's error in its share, and V / 4096 + 60 units of u for the additions (8 in a step of
      8192 logits, one a step, 11 joins of 4 units)
  q: exp(t) or exp(t / T - its normaliser): (8 + 4 |t| / T + k) u of it
  loss: the sum's error (twice with a tail) and u (2 + |log sum|), times the weight it has; each term's own roundings
  gradient: the errors of p, q and r through the difference, where z and its maximum round too when multiplied
      out (4 u (|z| + |max z| + |log sum|)); bf16: 2^-8 of the result
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


def inputs(N, V, k, dtype, seed, T=1.0, tail=False, pad=0, off=0):
    g = torch.Generator().manual_seed(seed)
    wide = torch.randn((N, V + pad + off), generator=g) * (0.5 + 2.0 * torch.rand((N, 1), generator=g))
    wide = wide.to(DTYPES[dtype])
    x = wide[:, off:off + V]
    teacher = x.float() + 0.5 * torch.randn((N, V), generator=g)
    value, idx = torch.topk(torch.log_softmax(teacher / T if tail else teacher, 1), k, dim=1)
    idx = idx.to(torch.int32)
    if N > 3:
        idx[1, k // 2:] = -1  # fewer
        idx[2] = -1           # none
        value[1, k // 2:] = float("nan")
    return wide, x, idx, value.contiguous(), torch.randn(N, generator=g) / N


def reference(x, idx, value, T, tail):
    """Everything in 64 bits: a dict."""
    V = x.shape[1]
    z = torch.cat([x.double() / T, torch.full((x.shape[0], 1), -INF, dtype=torch.float64)], 1)
    valid = idx >= 0
    at = torch.where(valid, idx, V).long()
    m = z.max(1).values
    e = torch.exp(z - torch.where(m == -INF, 0.0, m)[:, None])
    on = torch.zeros_like(z, dtype=torch.bool).scatter_(1, at, True)
    S, R = e.sum(1), torch.where(on, 0.0, e).sum(1)
    t = torch.where(valid, value.double() / (1.0 if tail else T), -INF)
    if tail:
        q = torch.exp(t)
        given = q.sum(1)
        left = torch.where(R > 0, (1.0 - given).clamp(min=0.0), 0.0)
    else:
        norm = torch.logsumexp(t, 1)
        q = torch.exp(t - torch.where(norm == -INF, 0.0, norm)[:, None])
        given, left = norm, torch.zeros_like(m)
    log_p = z.gather(1, at) - m[:, None] - torch.log(S)[:, None]
    loss = -torch.where(q > 0, q * log_p, 0.0).sum(1) + torch.where(left > 0, left * (torch.log(S) - torch.log(R)), 0.0)
    Q = q.sum(1) + left
    p = e / S[:, None]
    r = torch.where(on, 0.0, e) / torch.where(R > 0, R, 1.0)[:, None]
    target = torch.zeros_like(z).scatter_add_(1, at, q) + left[:, None] * r
    target[:, V] = 0.0
    k = idx.shape[1]
    d = torch.where(e > 0, m[:, None] - z, 0.0)
    e_exp = (8 + 4 * d) * U
    add = (V / 4096 + 60) * U
    e_S = (p * e_exp).sum(1) + add
    e_R = (r * e_exp).sum(1) + add
    e_q = (8 + 4 * torch.where(q > 0, t.abs(), 0.0) + k) * U
    return dict(z=z, m=m, S=S, R=R, q=q, at=at, valid=valid, given=given, left=left, log_p=log_p, loss=loss, Q=Q, p=p, r=r, on=on,
                target=target, d=d, e_exp=e_exp, e_S=e_S, e_R=e_R, e_q=e_q)


def check_forward(loss, stats, f, tail):
    log_S, log_R = torch.log(f["S"]), torch.log(f["R"])
    lp = torch.where(f["q"] > 0, f["log_p"], 0.0)
    tol = (f["q"] * lp.abs() * (f["e_q"] + 8 * U)).sum(1) + f["Q"] * (f["e_S"] + 4 * U * (1 + log_S.abs()))
    tol += (f["q"] * torch.where(f["q"] > 0, f["d"].gather(1, f["at"]), 0.0)).sum(1) * 4 * U
    off = torch.where(f["R"] > 0, log_S - log_R, 0.0)
    tol += (f["q"] * f["e_q"]).sum(1) * off.abs() + f["left"] * (f["e_S"] + f["e_R"] + 4 * U * (1 + log_S.abs() + off.abs()))
    loss, stats = loss.cpu().double(), stats.cpu().double()
    assert ((loss - f["loss"]).abs() <= tol).all(), float(((loss - f["loss"]).abs() / tol).max())
    assert ((stats[:, 0] - f["m"]).abs() <= 2 * U * f["m"].abs()).all()
    assert ((stats[:, 1] - log_S).abs() <= f["e_S"] + 2 * U * (1 + log_S.abs())).all()
    some = f["R"] > 0
    assert (stats[~some, 2] == -INF).all()
    assert ((stats[:, 2] - log_R)[some].abs() <= (f["e_R"] + 2 * U * (1 + log_R.abs()))[some]).all()
    e = (f["q"] * f["e_q"]).sum(1) if tail else f["e_q"].max(1).values + 4 * U * torch.where(f["given"] == -INF, 0.0, f["given"]).abs()
    same = stats[:, 3] == f["given"]
    assert (same | ((stats[:, 3] - f["given"]).abs() <= e)).all()


def check_backward(dx, f, dloss, T, V, dtype):
    w = (dloss.double() / T)[:, None]
    want = (w * (f["p"] * f["Q"][:, None] - f["target"]))[:, :V]
    log_S = torch.log(f["S"])[:, None].abs()
    z = torch.where(f["z"] == -INF, 0.0, f["z"]).abs()
    e_p = f["e_exp"] + f["e_S"][:, None] + f["e_R"][:, None] + 4 * U * (4 + z + f["m"].abs()[:, None] + log_S)
    of_left = (f["q"] * f["e_q"]).sum(1)[:, None]
    e_target = torch.zeros_like(f["z"]).scatter_add_(1, f["at"], f["q"] * (f["e_q"] + 8 * U))
    tol = w.abs() * (f["p"] * (f["Q"][:, None] * e_p + of_left) + f["r"] * (f["left"][:, None] * e_p + of_left) + e_target)
    tol = tol[:, :V] + (2.0 ** -8 + 4 * U if dtype == "bf16" else 4 * U) * want.abs() + 1e-40
    diff = (dx.cpu().double() - want).abs()
    assert (diff <= tol).all(), float((diff / tol).max())


def both(dev, N, V, k, dtype, T, tail, pad=0, off=0, seed=None):
    wide, x, idx, value, dloss = inputs(N, V, k, dtype, V + k if seed is None else seed, T, tail, pad, off)
    f = reference(x, idx, value, T, tail)
    logits = wide.to(dev)[:, off:off + V]
    status = cci.new_status(dev)
    lists = idx.to(dev), value.to(dev)
    loss, stats = cci.distillation_loss(logits, *lists, temperature=T, tail=tail, status=status)
    check_forward(loss, stats, f, tail)
    assert int(status.item()) == 0
    dx = cci.distillation_loss_backward(dloss.to(dev), logits, *lists, stats, temperature=T, tail=tail)
    assert dx.dtype == x.dtype and dx.shape == x.shape
    check_backward(dx, f, dloss, T, V, dtype)
    return logits, lists, dloss, stats, dx


# vocabularies at both sides of a group, a warp's step, a block's, and of the two sizes of blocks; rows over clusters
SIZES = [(5, 1, 1), (4, 2, 2), (6, 7, 3), (9, 8, 8), (7, 9, 1), (5, 31, 20), (40, 129, 128), (33, 255, 5), (20, 1000, 64), (5, 2047, 1),
         (5, 2048, 128), (5, 2049, 20), (6, 8191, 5), (6, 8200, 128), (4, 40000, 32), (5, 70001, 20), (1100, 300, 7), (1, 5, 5)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,tail", [(1.0, False), (1.0, True), (2.0, False), (0.7, True)])
@pytest.mark.parametrize("N,V,k", SIZES)
def test_against_64_bits(dev, N, V, k, T, tail, dtype):
    both(dev, N, V, k, dtype, T, tail)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,off", [(3, 0), (0, 1), (5, 3), (7, 7), (24, 8)])
@pytest.mark.parametrize("V", [50, 3001, 20000])
def test_rows_from_any_place(dev, V, pad, off, dtype):
    logits, lists, dloss, stats, dx = both(dev, 6, V, 9, dtype, 1.0, True, pad, off)
    # and into rows that start elsewhere than theirs
    out = torch.full((6, V + 9), 7.0, dtype=logits.dtype, device=dev)
    got = cci.distillation_loss_backward(dloss.to(dev), logits, *lists, stats, tail=True, out=out[:, 5:5 + V])
    assert torch.equal(got, dx) and (out[:, :5] == 7).all() and (out[:, 5 + V:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 9000])
def test_in_place(dev, V, dtype):
    logits, lists, dloss, stats, dx = both(dev, 8, V, 20, dtype, 2.0, False)
    assert cci.distillation_loss_backward(dloss.to(dev), logits, *lists, stats, temperature=2.0, out=logits) is logits
    assert torch.equal(logits, dx)


def test_rows_longer_than_a_block_has_bits_for(dev):
    both(dev, 1, (1 << 22) + 5, 128, "bf16", 1.0, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,k", [(57, 5000, 20), (58, 5000, 20), (200, 9001, 5), (456, 3000, 64), (500, 4097, 20), (3648, 2100, 7), (3647, 2100, 7), (2, 300001, 128),
                                   (130, 40000, 9), (40, 140000, 20)])
def test_rows_that_share_blocks(dev, N, V, k, dtype):
    """On both sides of what takes a cluster a row, a warp a row, or blocks that cut the rows evenly."""
    both(dev, N, V, k, dtype, 1.0, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
def test_masked_logits(dev, tail, dtype):
    """-inf and the type's lowest value take no part; a listed token that is masked has no chance."""
    N, V, k = 6, 3000, 8
    _, x, idx, value, dloss = inputs(N, V, k, dtype, 3, 1.0, tail)
    x = x.clone()
    low = torch.finfo(DTYPES[dtype]).min
    free = torch.ones((N, V), dtype=torch.bool).scatter_(1, idx.clamp(min=0).long(), False)
    x[0] = torch.where(free[0], -INF, x[0])              # nothing but the listed
    x[1] = torch.where(free[1] & (torch.arange(V) % 3 > 0), low, x[1])
    x[3, idx[3, 2]] = -INF                               # a listed one
    x[4] = -INF                                          # nothing at all
    x[5] = low                                           # the same everywhere
    d = x.to(dev), idx.to(dev), value.to(dev)
    loss, stats = cci.distillation_loss(*d, tail=tail)
    dx = cci.distillation_loss_backward(dloss.to(dev), *d, stats, tail=tail).cpu()
    ok = [0, 1, 2]
    f = reference(x[ok], idx[ok], value[ok], 1.0, tail)
    check_forward(loss[ok], stats[ok], f, tail)
    check_backward(dx[ok], f, dloss[ok], 1.0, V, dtype)
    assert loss[3] == INF and dx[3].isfinite().all()
    assert loss[4] == INF and (dx[4] == 0).all() and (stats[4, 0] == -INF) and (stats[4, 1] == 0)
    # all logits alike: p = 1 / V
    f = reference(torch.zeros((1, V)), idx[5:], value[5:], 1.0, tail)
    assert abs(float(loss[5]) - float(f["loss"])) <= 1e-5 * float(f["loss"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [0.5, 2.0 ** -10, 2.0 ** -127])
@pytest.mark.parametrize("N,V", [(6, 900), (6, 20000), (300, 5000)])
def test_maxima_beyond_32_bits(dev, N, V, T, tail, dtype):
    """Rows whose maximum is the type's lowest value, or its largest, divided by a temperature below 1.  What is not at the maximum is
    at least 2^-24 of it below, more than any exponent: the formula's result is that of 0 at the maximum and -inf elsewhere.
    So it is of a teacher's values."""
    k, info = 8, torch.finfo(DTYPES[dtype])
    g = torch.Generator().manual_seed(V)
    at_most = torch.rand((N, V), generator=g) < 0.3
    at_most[:, :4] = True
    at_most[N - 1] = True                                # nothing but the maximum
    high = torch.full((N, 1), info.min)
    high[1] = info.max
    lower = torch.where(high < 0, -INF, torch.randn((N, V), generator=g))
    x = torch.where(at_most, high, lower).to(DTYPES[dtype])
    idx = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(N)]).to(torch.int32)
    idx[0, :3] = torch.tensor([0, 1, 2])
    idx[2] = -1
    value = torch.full((N, k), -2.0)
    if not tail:                                         # alike far down, but for one lower
        value[:] = torch.finfo(torch.float32).min * 0.9
        value[:, 1] = torch.finfo(torch.float32).min
    chance = at_most.gather(1, idx.clamp(min=0).long())  # the listed have to have one, or the loss is infinite
    idx = torch.where(chance, idx, -1)
    most = torch.where(idx >= 0, value, -INF).max(1, keepdim=True).values
    same = value if tail else torch.where(value == most, 0.0, -INF)
    dloss = torch.rand(N, generator=g) * min(T, 1.0)
    f = reference(torch.where(at_most, 0.0, -INF), idx, same, 1.0, tail)
    logits, lists = x.to(dev), (idx.to(dev), value.to(dev))
    check_shifted(logits, lists, dloss, T, tail, dtype, f)


def check_shifted(logits, lists, dloss, T, tail, dtype, f):
    """Against the formula of logits and a teacher's values less their rows' largest, which is the same."""
    N, V = logits.shape
    m = logits.cpu().double().max(1).values
    loss, stats = cci.distillation_loss(logits, *lists, temperature=T, tail=tail)
    shown = stats.cpu().double()
    as_is = torch.signbit(shown[:, 1])
    assert (shown[as_is, 0] == m[as_is]).all() and ((shown[:, 0] - m / T).abs() <= 2 * U * (m / T).abs())[~as_is].all()
    shown[:, 0], shown[:, 1] = 0.0, shown[:, 1].abs()
    if not tail:
        shown[:, 3] = f["given"]
    check_forward(loss, shown, f, tail)
    # the gradient takes maxima and normalisers of up to 64 from their quotients by T, whose roundings count as above
    t = (torch.where(f["valid"], lists[1].cpu().double(), 0.0) / T).abs().max(1, keepdim=True).values
    f = dict(f, m=torch.where(as_is | ((m / T).abs() >= 64), 0.0, m / T))
    if not tail:
        f["e_q"] = f["e_q"] + 4 * U * torch.where(t < 68, t, 0.0)
    dloss_on = dloss.to(logits.device)
    dx = cci.distillation_loss_backward(dloss_on, logits, *lists, stats, temperature=T, tail=tail)
    check_backward(dx, f, dloss, T, V, dtype)
    assert cci.distillation_loss_backward(dloss_on, logits, *lists, stats, temperature=T, tail=tail, out=logits) is logits
    assert torch.equal(logits, dx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [0.7, 1.0, 1.5, 3.0])
@pytest.mark.parametrize("mask", [-50.0, -1e4, -1e6, -1e9, -1e30, -1e38, 1e5])
@pytest.mark.parametrize("N,V", [(6, 900), (6, 20000), (300, 5000)])
def test_rows_that_lie_far_from_0(dev, N, V, mask, T, tail, dtype):
    """Every logit of a row, and the teacher's values, with the same number added: as a mask that covers all of a row does.  The
    type keeps what it has room for of their differences."""
    k, t = 8, DTYPES[dtype]
    g = torch.Generator().manual_seed(V)
    x = (torch.randn((N, V), generator=g) * 3 + mask).to(t)
    idx = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(N)]).to(torch.int32)
    value = torch.log(torch.full((N, k), 0.08)) if tail else torch.randn((N, k), generator=g) + mask
    value = value.contiguous()
    apart = (x.double() - x.double().max(1, keepdim=True).values) / T
    value_apart = value.double() if tail else (value.double() - value.double().max(1, keepdim=True).values) / T
    dloss = torch.randn(N, generator=g)
    check_shifted(x.to(dev), (idx.to(dev), value.to(dev)), dloss, T, tail, dtype, reference(apart, idx, value_apart, 1.0, tail))


def test_nan_and_inf_keep_to_their_rows(dev):
    N, V, k = 5, 5000, 6
    _, x, idx, value, dloss = inputs(N, V, k, "f32", 4, 1.0, True)
    good = cci.distillation_loss(x.to(dev), idx.to(dev), value.to(dev), tail=True)[0]
    x = x.clone()
    x[0, 17], x[3, 4000] = float("nan"), INF
    value[4, 1] = float("nan")
    d = x.to(dev), idx.to(dev), value.to(dev)
    loss, stats = cci.distillation_loss(*d, tail=True)
    assert loss[[0, 3, 4]].isnan().all() and torch.equal(loss[1:3], good[1:3])
    dx = cci.distillation_loss_backward(dloss.to(dev), *d, stats, tail=True)
    assert dx[0].isnan().all() and dx[3].isnan().all() and dx[1:3].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V", [(9, 1000), (9, 20000), (300, 5000), (4000, 3000)])
def test_pad_rows_may_hold_anything(dev, N, V, tail, dtype):
    """Rows that list nothing, and rows without a gradient."""
    _, x, idx, value, dloss = inputs(N, V, 6, dtype, 14, 1.0, tail)
    pad, off = torch.arange(N) % 4 == 1, torch.arange(N) % 4 == 2
    idx[pad], dloss[off] = -1, 0.0
    clean = torch.where((pad | off)[:, None], 0.0, x.float()).to(x.dtype)
    dirty = clean.clone()
    dirty[pad | off] = torch.tensor([1.0, float("nan"), INF, -INF, 2.0]).repeat(V // 5).to(x.dtype)
    dirty[5] = INF
    got = []
    for logits in (clean, dirty):
        d = logits.to(dev), idx.to(dev), value.to(dev)
        status = cci.new_status(dev)
        loss, stats = cci.distillation_loss(*d, tail=tail, status=status)
        assert int(status.item()) == 0
        got.append((loss[~off.to(dev)], cci.distillation_loss_backward(dloss.to(dev), *d, stats, tail=tail)))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and got[0][1].isfinite().all()
    assert (got[1][1].cpu()[pad | off] == 0).all()


def test_teacher_values_of_minus_inf(dev):
    """They are listed, with q = 0: with a tail their logits are not among the rest."""
    N, V, k = 4, 700, 6
    for tail in (False, True):
        _, x, idx, value, dloss = inputs(N, V, k, "f32", 8, 1.0, tail)
        value[0, 3:] = -INF
        value[3] = -INF
        f = reference(x, idx, value, 1.0, tail)
        d = x.to(dev), idx.to(dev), value.to(dev)
        loss, stats = cci.distillation_loss(*d, tail=tail)
        check_forward(loss, stats, f, tail)
        check_backward(cci.distillation_loss_backward(dloss.to(dev), *d, stats, tail=tail), f, dloss, 1.0, V, "f32")


@pytest.mark.parametrize("V", [900, 60000])
def test_bad_indices_are_reported(dev, V):
    N, k = 7, 5
    _, x, idx, value, dloss = inputs(N, V, k, "bf16", 9, 1.0, True)
    idx[0, 4] = V
    idx[3, 0] = -2
    idx[4, 3] = idx[4, 1]       # listed twice
    idx[6, 2] = 2 ** 31 - 1
    d = x.to(dev), idx.to(dev), value.to(dev)
    status = cci.new_status(dev)
    loss, stats = cci.distillation_loss(*d, tail=True, status=status)
    assert cci.read_status(status) == 10  # CCI_ERR_INDEX
    bad = torch.tensor([True, False, False, True, True, False, True])
    assert (loss.cpu().isnan() == bad).all()
    dx = cci.distillation_loss_backward(dloss.to(dev), *d, stats, tail=True).cpu()
    assert dx[bad].isnan().all() and dx[~bad].isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(6, 300), (6, 20000), (300, 5000)])
def test_small_losses(dev, N, V, dtype):
    """Relative to themselves: a student's that is sure of what its teacher says, and what a few tokens of a small chance
    take from the rest.  An exponential is off by (8 + 4 * 33) u, the sums by V / 4096 + 60 units of u, q by (8 + 4 * 9) u, the
    rest's share of the teacher, 0.99 at least, by as much of 0.01, three logarithms and products by 4 u each: 300 u."""
    g = torch.Generator().manual_seed(V)
    x = torch.rand((N, V), generator=g).to(DTYPES[dtype])
    idx = torch.stack([torch.randperm(V, generator=g)[:3] for _ in range(N)]).to(torch.int32)
    sure = x.clone()
    sure[torch.arange(N), idx[:, 0].long()] = 32.0
    value = torch.tensor([0.0, -INF, -INF]).repeat(N, 1)
    loss, _ = cci.distillation_loss(sure.to(dev), idx.to(dev), value.to(dev))
    # 1 + 6e-12 is off by 2^-53 in 64 bits too, 1.8e-5 of the loss: what is added to the 1 by itself
    want = torch.log1p(torch.exp(sure.double() - 32.0).scatter(1, idx[:, :1].long(), 0.0).sum(1))
    assert want.max() < 1e-8 and ((loss.cpu().double() - want).abs() <= 300 * U * want).all()
    value = torch.tensor([-9.0, -7.0, -INF]).repeat(N, 1)
    loss, _ = cci.distillation_loss(x.to(dev), idx.to(dev), value.to(dev), tail=True)
    want = reference(x, idx, value, 1.0, True)["loss"]
    assert want.max() < 0.1 and ((loss.cpu().double() - want).abs() <= 300 * U * want).all()


def test_gradient_against_differences(dev):
    N, V, k = 2, 30, 4
    for T, tail in ((1.5, False), (1.0, True)):
        _, x, idx, value, dloss = inputs(N, V, k, "f32", 12, T, tail)
        d = x.to(dev), idx.to(dev), value.to(dev)
        loss, stats = cci.distillation_loss(*d, temperature=T, tail=tail)
        dx = cci.distillation_loss_backward(dloss.to(dev), *d, stats, temperature=T, tail=tail)
        step = 1e-4
        for n, v in ((0, int(idx[0, 0])), (0, 3), (1, int(idx[1, 2])), (1, 29)):
            ends = []
            for sign in (1, -1):
                moved = x.double()
                moved[n, v] += sign * step
                ends.append(float((reference(moved, idx, value, T, tail)["loss"] * dloss.double()).sum()))
            # third derivatives of the loss are below 1
            assert abs((ends[0] - ends[1]) / (2 * step) - float(dx[n, v])) <= 1e-6


def test_no_rows(dev):
    e, i, v = torch.empty((0, 100), device=dev), torch.empty((0, 5), dtype=torch.int32, device=dev), torch.empty((0, 5), device=dev)
    loss, stats = cci.distillation_loss(e, i, v)
    assert loss.shape == (0,) and stats.shape == (0, 4)
    assert cci.distillation_loss_backward(loss, e, i, v, stats).shape == (0, 100)
