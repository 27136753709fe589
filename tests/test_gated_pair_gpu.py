"""CTA pairs of the gated block end in order: launches back to back, with reductions of fewer stages than the ring
has, as many, and more, in each of the products.  Whole numbers, so that every launch has to give the same bits as
64 bits do; every wait at the end of a launch is for something that arrives, so the status stays 0 and no launch
takes the time of an expired wait."""
import time

import pytest
import torch

import paper_1910_11971_gb300 as cci

pytestmark = pytest.mark.gpu
LAUNCHES = 20


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def whole(shape, seed, dev):
    g = torch.Generator(device=dev).manual_seed(seed)
    return torch.randint(-1, 2, shape, generator=g, device=dev).bfloat16()


# the forward pass reduces over D, dX over twice F, dW over N, 64 to a stage: one stage to many, ragged
@pytest.mark.parametrize("N,D,F", [(4096, 8, 4096), (4096, 64, 4096), (4100, 136, 4096), (4096, 320, 4104), (4096, 384, 4096),
                                   (4096, 448, 4096), (4000, 1000, 4096), (64, 4096, 8192), (136, 4096, 8192), (320, 4104, 8192),
                                   (384, 4096, 8192), (448, 4096, 8192), (4096, 4096, 64), (4096, 4096, 200)])
def test_launches_back_to_back(dev, N, D, F):
    x, wg, wu, dh = (whole(s, k, dev) for k, s in enumerate(((N, D), (F, D), (F, D), (N, F))))
    st = cci.new_status(dev)
    h, g, u = cci.gated_linear(x, wg, wu, act="relu", save=True, status=st)
    grads = cci.gated_linear_backward(dh, x, wg, wu, g, u, act="relu", status=st)
    torch.cuda.synchronize()
    start = time.perf_counter()
    runs = [(cci.gated_linear(x, wg, wu, act="relu", status=st), *cci.gated_linear_backward(dh, x, wg, wu, g, u, act="relu", status=st))
            for _ in range(LAUNCHES)]
    assert cci.read_status(st) == 0
    assert time.perf_counter() - start < 0.9  # a wait expires after about a second
    for run in runs:
        assert all(torch.equal(a, b) for a, b in zip(run, (h, *grads)))
    del runs
    gr, ur = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    assert torch.equal(g.double(), gr) and torch.equal(u.double(), ur)
    dg = (dh.double() * ur * (gr > 0)).bfloat16().double()  # rounded to bf16 as operands, where they pass 256
    du = (dh.double() * gr.clamp(min=0)).bfloat16().double()
    for got, ref in ((grads[0], dg @ wg.double() + du @ wu.double()), (grads[1], dg.t() @ x.double()), (grads[2], du.t() @ x.double())):
        assert ref.abs().max() < 2 ** 24
        assert torch.equal(got, ref.float().bfloat16())
