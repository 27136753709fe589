"""Layer norm's bounded waits say when they expire: the backward pass takes a status word, no kernel waits without one,
and a word given to a call that succeeds stays 0.  The forward pass waits for nothing."""
import glob
import os
import re

import pytest
import torch

import paper_1910_11971_gb300 as cci
from paper_1910_11971_gb300 import build as cci_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # never dereferenced: refused before any launch
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 4, 5, 11


def test_every_bounded_wait_has_a_status_word():
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_1910_11971_gb300", "csrc", "*.cu*"))):
        for call in re.findall(r"mbar_wait(?:<[^>]*>)?\([^;]*;", open(path).read()):
            assert "nullptr" not in call and "NULL" not in call, (os.path.basename(path), call)


def test_refusals_with_a_status_word():
    cci_build.build()
    b = cci.lib().cci_layer_norm_backward_ex

    def bwd(dy=FAKE, dt=0, N=4, D=8, ws=FAKE, n=0):
        return b(dy, 8, FAKE, 8, dt, N, D, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, ws, n, None)

    assert bwd(dt=3) == DTYPE and bwd(dy=FAKE + 2) == ALIGN and bwd(dy=None) == NULL and bwd(D=0) == SHAPE
    assert bwd() == WORKSPACE and bwd(ws=None, n=1 << 20) == WORKSPACE


# groups of a warp to a whole block, one row a group, as many as the ring holds and more, unequal numbers of them; a
# layout without a ring (odd rows), and rows past the widest that a block holds
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,D", [(1, 8), (9, 64), (4100, 64), (30011, 256), (5000, 1024), (3001, 4096), (700, 8192), (400, 16384),
                                 (500, 1001), (40, 20000)])
def test_status_stays_clear(N, D, dtype):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(N + D)
    x, dy = (torch.randn((N, D), generator=g, device=dev).to(dtype) for _ in range(2))
    w, b = (torch.randn(D, generator=g, device=dev) for _ in range(2))
    st = cci.new_status(dev)
    y, mean, rstd = cci.layer_norm(x, w, b)
    got = cci.layer_norm_backward(dy, x, mean, rstd, w, status=st)
    assert cci.read_status(st) == 0
    assert all(t.isfinite().all() for t in (y, mean, rstd, *got))
    # again, and without a word: the same bits
    assert all(torch.equal(p, q) for p, q in zip((y, mean, rstd), cci.layer_norm(x, w, b)))
    assert all(torch.equal(p, q) for p, q in zip(got, cci.layer_norm_backward(dy, x, mean, rstd, w)))
