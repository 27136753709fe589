"""Rows of distillation whose list is wrong, or whose logits are no numbers, where the teacher gives nothing any weight: their loss
is NaN all the same, in each of the kernels, and the rows beside them are as they were."""
import pytest
import torch

import paper_1910_11971_gb300 as cci

INF, NAN = float("inf"), float("nan")
INDEX = 10  # CCI_ERR_INDEX

pytestmark = pytest.mark.gpu

SIZES = [(40, 900), (9, 20000), (300, 5000)]  # a warp, a cluster a row; rows that share blocks


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def lists(N, V, kind):
    """idx, value, the wrong rows: every third."""
    g = torch.Generator().manual_seed(V)
    k = 1 if kind == "one" else 4
    idx = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(N)]).to(torch.int32)
    value = torch.log(torch.full((N, k), 0.2))
    bad = torch.arange(N) % 3 == 1
    if kind == "one":
        idx[bad, 0] = -2
    elif kind == "pads":          # another number than -1 for what is not there
        idx[bad] = -100
    elif kind == "past":
        idx[bad, 2] = V
        idx[bad, :2], idx[bad, 3] = -1, -1
    else:                         # listed twice, of no weight
        idx[bad, 3] = idx[bad, 1]
        value[bad] = -INF
    return idx, value, bad


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("kind", ["one", "pads", "past", "twice"])
@pytest.mark.parametrize("N,V", SIZES)
def test_wrong_lists(dev, N, V, kind, tail):
    x = torch.randn((N, V), generator=torch.Generator().manual_seed(1)).to(dev)
    idx, value, bad = lists(N, V, kind)
    status = cci.new_status(dev)
    loss, _ = cci.distillation_loss(x, idx.to(dev), value.to(dev), tail=tail, status=status)
    assert cci.read_status(status) == INDEX
    assert (loss.cpu().isnan() == bad).all()
    good = torch.where(bad[:, None], -1, idx).to(torch.int32)
    same, _ = cci.distillation_loss(x, good.to(dev), value.to(dev), tail=tail)
    assert torch.equal(loss.cpu()[~bad], same.cpu()[~bad])


@pytest.mark.parametrize("what", [NAN, INF])
@pytest.mark.parametrize("N,V", SIZES)
def test_no_numbers_where_nothing_has_weight(dev, N, V, what):
    x = torch.randn((N, V), generator=torch.Generator().manual_seed(2))
    idx = torch.arange(3, dtype=torch.int32).repeat(N, 1)
    value = torch.full((N, 3), -INF)
    bad = torch.arange(N) % 3 == 1
    x[bad, V // 2] = what
    loss, _ = cci.distillation_loss(x.to(dev), idx.to(dev), value.to(dev))
    assert (loss.cpu().isnan() == bad).all() and (loss.cpu()[~bad] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("kind", ["one", "pads", "past", "twice"])
@pytest.mark.parametrize("N,V", SIZES)
def test_gradients_of_wrong_lists(dev, N, V, kind, tail, dtype):
    """NaN all along the row, unless its loss has no gradient; the other rows' as without."""
    x = torch.randn((N, V), generator=torch.Generator().manual_seed(1)).to(dtype)
    idx, value, bad = lists(N, V, kind)
    x[1], x = -INF, x.to(dev)  # nothing but a wrong list
    dloss = torch.where(torch.arange(N) % 6 == 4, 0.0, 1.0)
    got = []
    for at in (idx, torch.where(bad[:, None], -1, idx).to(torch.int32)):
        args = x, at.to(dev), value.to(dev)
        _, stats = cci.distillation_loss(*args, tail=tail)
        got.append(cci.distillation_loss_backward(dloss.to(dev), *args, stats, tail=tail).cpu())
    lost = bad & (dloss != 0)
    assert got[0][lost].isnan().all() and (got[0][bad & ~lost] == 0).all()
    assert torch.equal(got[0][~bad], got[1][~bad]) and got[1].isfinite().all()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V", SIZES)
def test_pad_rows_have_no_gradient_whatever_their_loss_has(dev, N, V, tail):
    """Rows that list nothing, beside an incoming gradient of NaN or inf for them."""
    x = torch.randn((N, V), generator=torch.Generator().manual_seed(3)).to(dev)
    idx = torch.arange(4, dtype=torch.int32).repeat(N, 1)
    pad = torch.arange(N) % 3 == 1
    idx[pad] = -1
    value = torch.log(torch.full((N, 4), 0.2))
    args = x, idx.to(dev), value.to(dev)
    _, stats = cci.distillation_loss(*args, tail=tail)
    for what in (NAN, INF, 1.0):
        dx = cci.distillation_loss_backward(torch.where(pad, what, 1.0).to(dev), *args, stats, tail=tail).cpu()
        assert (dx[pad] == 0).all() and dx[~pad].isfinite().all()
