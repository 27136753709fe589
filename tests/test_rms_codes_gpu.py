"""Codes and scales of the root-mean-square norm in 8 bits, bit for bit: y = x rstd weight, both products rounded to fp32, is
known from the call's own rstd, scale = max(max |y| / 448, 2^-126) and q = e4m3(y / scale) with the quotients that fp32 rounds
to the nearest.  Whole numbers under a row's 448 lie on the middle of two codes by the dozen (17 between 16 and 18): a quotient that
is one unit off takes the other code."""
import pytest
import torch

import paper_1910_11971_gb300 as cci

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def check(x, w, group, dev):
    N, D = x.shape
    q, scales, _, rstd = (t.cpu() for t in cci.rms_norm_fp8(x.to(dev), w.to(dev), group=group))
    y = x.float() * rstd[:, None] * w
    for i in range(scales.shape[1]):
        at = slice(i * (group or D), (i + 1) * (group or D))
        scale = (y[:, at].abs().amax(1, keepdim=True) / 448.0).clamp(min=2.0 ** -126)
        assert torch.equal(scales[:, i:i + 1], scale)
        want = (y[:, at] / scale).to(torch.float8_e4m3fn).float()
        assert torch.equal(q[:, at].float().nan_to_num(nan=1e9), want.nan_to_num(nan=1e9))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("D", [8, 128, 512, 1000, 4096, 8192, 16384, 16392])
@pytest.mark.parametrize("factor", [1.0, 0.7, 1e-12, 1e-30, 1e-33, 3e-37, 1e30, 1e37])
def test_middles_of_codes(dev, D, group, factor, dtype):
    """Weights that leave the scales tiny, down to the least one, and large among them."""
    N = 200 if D < 4096 else 20
    g = torch.Generator().manual_seed(D)
    x = torch.randint(-448, 449, (N, D), generator=g).float()
    x[:, ::8] = 448.0
    check(x.to(DTYPES[dtype]), torch.full((D,), factor), group, dev)


@pytest.mark.parametrize("group", [0, 128])
def test_infinite_scales(dev, group):
    """y beyond fp32: what is finite is 0 of such a scale, and the infinite has no code."""
    x = torch.randn((20, 512), generator=torch.Generator().manual_seed(1))
    w = torch.full((512,), 3e38)
    w[128:] = 1.0
    assert (x[:, :128].abs().amax(1) > 2).all()
    check(x, w, group, dev)
