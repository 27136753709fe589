"""fp32 products of the gated block whose tiles are too few for the SMs: their reductions are cut over all of them, or
over as many as have eight stages each, and the forward pass' parts are joined with its activation.

Whole numbers below 2^24 are exact in every product of planes and in fp32 sums of any order, so every result is
compared bit for bit with 64 bits."""
import pytest
import torch

import paper_1910_11971_gb300 as cci
from paper_1910_11971_gb300 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def whole(shape, seed, dev):
    return wl.integer_valued(shape, -1, 1, seed).float().to(dev)


# tiles of 128 and 64 columns, ragged edges in each; one tile and many; shares that end inside a tile and at its end;
# fewer shares than SMs; one more row or channel than a tile
SHAPES = [(427, 4088, 648), (194, 1608, 112), (583, 1832, 72), (55, 2704, 712), (17, 4096, 264), (128, 1024, 64), (129, 1024, 72),
          (24, 376, 728), (52, 200, 120), (300, 2048, 1032), (1300, 4096, 8), (1000, 512, 2048), (17, 8192, 8), (641, 1000, 640)]


@pytest.mark.parametrize("N,D,F", SHAPES)
def test_forward_and_backward_are_exact(dev, N, D, F):
    x, wg, wu, dh = (whole(s, k, dev) for k, s in enumerate(((N, D), (F, D), (F, D), (N, F))))
    st = cci.new_status(dev)
    h, g, u = cci.gated_linear(x, wg, wu, act="relu", save=True, status=st)
    gr, ur = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    hr = gr.clamp(min=0) * ur
    assert hr.abs().max() < 2 ** 24
    assert torch.equal(g.double(), gr) and torch.equal(u.double(), ur) and torch.equal(h.double(), hr)
    assert torch.equal(cci.gated_linear(x, wg, wu, act="relu", status=st), h)  # not saved: the same
    dg, du = dh.double() * ur * (gr > 0), dh.double() * gr.clamp(min=0)
    dx, dwg, dwu = cci.gated_linear_backward(dh, x, wg, wu, g, u, act="relu", status=st)
    for got, ref in ((dx, dg @ wg.double() + du @ wu.double()), (dwg, dg.t() @ x.double()), (dwu, du.t() @ x.double())):
        assert ref.abs().max() < 2 ** 24
        assert torch.equal(got.double(), ref)
    assert cci.read_status(st) == 0


@pytest.mark.parametrize("N,D,F,G,K", [(194, 1608, 112, 8, 2), (55, 2704, 704, 32, 8), (427, 1000, 640, 64, 8), (20, 4096, 256, 4, 1)])
def test_packed_gives_the_bits_of_dense(dev, N, D, F, G, K):
    x = whole((N, D), 1, dev)
    pairs = [cci.pack(torch.randn(F, D, device=dev), G, K) for _ in range(2)]
    full = []
    for values, idx in pairs:
        w = torch.zeros((F // G, D, G), device=dev)
        full.append(w.scatter_(2, idx.long(), values).permute(0, 2, 1).reshape(F, D).contiguous())
    st = cci.new_status(dev)
    packed = cci.gated_linear_packed(x, pairs[0], pairs[1], F, G, K, act="gelu", status=st)
    assert torch.equal(packed, cci.gated_linear(x, full[0], full[1], act="gelu", status=st))
    assert cci.read_status(st) == 0


# what lies past the outputs and the stated workspace stays as it is
def test_nothing_else_is_written(dev):
    N, D, F = 130, 2056, 72
    x, wg, wu = (whole(s, k, dev) for k, s in enumerate(((N, D), (F, D), (F, D))))
    need = cci.gated_workspace(cci.GATED_FORWARD, torch.float32, N, D, F, dev).nbytes
    ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device=dev)
    out = torch.full((N + 2, F), 7.0, device=dev)
    st = cci.new_status(dev)
    cci.gated_linear(x, wg, wu, act="relu", out=out[1:-1], workspace=ws[:need], status=st)
    assert cci.read_status(st) == 0
    assert bool((ws[need:] == 0x5A).all()) and bool((out[0] == 7).all()) and bool((out[-1] == 7).all())
    assert torch.equal(out[1:-1], cci.gated_linear(x, wg, wu, act="relu"))
