"""Layer norm of many wide rows, whose weight and bias lie in shared memory, against the formulas in 64 bits: blocks
that take several rows and unequal numbers of them, on both sides of that choice.  Tolerances as derived for the
narrower rows."""
import pytest
import torch

import paper_1910_11971_gb300 as cci
from test_norm_gpu import backward_inputs, check_backward, check_forward, params, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


# one row short of five a block of 152, and one more; widths just over a layout's end, odd words, and a layout's end
SHAPES = [(607, 4104), (609, 4104), (1300, 2056), (1300, 8192), (700, 8200), (700, 9784), (620, 16376), (620, 16384), (608, 16384)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D", SHAPES)
def test_forward(dev, N, D, dtype):
    x, (w, b) = rows(N, D, dtype, N + D, 2.0, 0.3), params(D, D)
    xd, wd, bd = x.to(dev), w.to(dev), b.to(dev)
    first = cci.layer_norm(xd, wd, bd)
    check_forward(*first, x, w, b, dtype)
    check_forward(*cci.layer_norm(xd, None, bd), x, None, b, dtype)
    check_forward(*cci.layer_norm(xd, wd), x, w, None, dtype)
    # a row's bits are the same in a call of few rows, and at every call
    few = cci.layer_norm(xd[:9], wd, bd)
    assert all(torch.equal(a, c[:9]) for a, c in zip(few, first))
    assert all(torch.equal(a, c) for a, c in zip(cci.layer_norm(xd, wd, bd), first))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D", SHAPES)
def test_backward(dev, N, D, dtype):
    x, dy, w, mean, rstd = backward_inputs(N, D, dtype, N + D)
    args = [t.to(dev) for t in (dy, x, mean, rstd)]
    first = cci.layer_norm_backward(*args, w.to(dev))
    check_backward(*first, dy, x, mean, rstd, w, dtype)
    check_backward(*cci.layer_norm_backward(*args), dy, x, mean, rstd, None, dtype)
    assert all(torch.equal(a, c) for a, c in zip(cci.layer_norm_backward(*args, w.to(dev)), first))
