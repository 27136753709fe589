"""What the calls of the root-mean-square norm, a head's cross entropy and distillation refuse, before anything is
enqueued: checked at the C entries with addresses that are never read, without a GPU."""
import pytest

import paper_1910_11971_gb300 as cci
from paper_1910_11971_gb300 import build as cci_build

OK, NULL, SHAPE, GROUP, DTYPE, ALIGN, VALUE, CUDA, TIMEOUT, UNSUP, INDEX, WORKSPACE = range(12)
P = 0x100000  # aligned and not null; never read on these paths
NAN = float("nan")
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    cci_build.build()
    return cci.lib()


def rms(lib, x=P, dt=1, N=4, D=64, ldx=64, r=P, ldr=64, w=P, eps=1e-5, y=P, h=P, rstd=P):
    return lib.cci_rms_norm(x, dt, N, D, ldx, r, ldr, w, eps, y, h, rstd, None)


def rms8(lib, x=P, dt=1, N=4, D=64, ldx=64, r=P, ldr=64, w=P, eps=1e-5, group=0, q=P, scales=P, h=P, rstd=P):
    return lib.cci_rms_norm_fp8(x, dt, N, D, ldx, r, ldr, w, eps, group, q, scales, h, rstd, None)


def rms_back(lib, dy=P, lddy=64, h=P, ldh=64, dh=P, lddh=64, dt=1, N=4, D=64, rstd=P, w=P, dx=P, dw=P, ws=P, wb=1 << 20):
    return lib.cci_rms_norm_backward(dy, lddy, h, ldh, dh, lddh, dt, N, D, rstd, w, dx, dw, ws, wb, None)


def ce(lib, x=P, dt=1, N=4, D=64, w=P, V=100, t=P, loss=P, stats=P, ws=P, wb=1 << 30):
    return lib.cci_linear_cross_entropy(x, dt, N, D, w, V, t, -100, loss, stats, None, ws, wb, None)


def ce_back(lib, dl=P, x=P, dt=1, N=4, D=64, w=P, V=100, t=P, stats=P, dx=P, dw=P, ws=P, wb=1 << 40):
    return lib.cci_linear_cross_entropy_backward(dl, x, dt, N, D, w, V, t, -100, stats, dx, dw, None, ws, wb, None)


def kd(lib, x=P, dt=1, N=4, V=100, ld=100, i=P, v=P, k=5, T=1.0, tail=0, loss=P, stats=P, ws=P, wb=1 << 30):
    return lib.cci_distillation_loss(x, dt, N, V, ld, i, v, k, T, tail, loss, stats, None, ws, wb, None)


def kd_back(lib, dl=P, x=P, dt=1, N=4, V=100, ld=100, i=P, v=P, k=5, T=1.0, tail=0, stats=P, dx=P, ldd=100):
    return lib.cci_distillation_loss_backward(dl, x, dt, N, V, ld, i, v, k, T, tail, stats, dx, ldd, None)


COMMON_RMS = [(dict(x=0), NULL), (dict(dt=2), DTYPE), (dict(N=-1), SHAPE), (dict(D=0), SHAPE), (dict(ldx=63), SHAPE), (dict(ldr=63), SHAPE),
              (dict(N=1 << 31), SHAPE), (dict(D=1 << 30, ldx=1 << 30, ldr=1 << 30), SHAPE), (dict(N=BIG, ldx=BIG), SHAPE),
              (dict(eps=-1.0), VALUE), (dict(eps=NAN), VALUE), (dict(x=P + 1), ALIGN), (dict(w=P + 2), ALIGN), (dict(rstd=P + 2), ALIGN)]


@pytest.mark.parametrize("change,want", COMMON_RMS + [(dict(y=0), NULL), (dict(y=P + 1), ALIGN), (dict(h=P + 1), ALIGN), (dict(r=P + 1), ALIGN)])
def test_rms_norm(lib, change, want):
    assert rms(lib, **change) == want


@pytest.mark.parametrize("change,want", COMMON_RMS + [
    (dict(q=0), NULL), (dict(scales=0), NULL), (dict(group=64), GROUP), (dict(group=-128), GROUP), (dict(D=60, ldx=64, ldr=64), UNSUP),
    (dict(x=P + 8), ALIGN), (dict(ldx=68), ALIGN), (dict(ldr=65), ALIGN), (dict(r=P + 2), ALIGN), (dict(h=P + 8), ALIGN), (dict(q=P + 8), ALIGN),
    (dict(w=P + 8), ALIGN), (dict(scales=P + 1), ALIGN)])
def test_rms_norm_fp8(lib, change, want):
    assert rms8(lib, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(dy=0), NULL), (dict(h=0), NULL), (dict(rstd=0), NULL), (dict(dx=0), NULL), (dict(dt=-1), DTYPE), (dict(N=-1), SHAPE), (dict(D=0), SHAPE),
    (dict(lddy=63), SHAPE), (dict(ldh=63), SHAPE), (dict(lddh=63), SHAPE), (dict(N=1 << 31), SHAPE), (dict(dy=P + 1), ALIGN), (dict(dh=P + 1), ALIGN),
    (dict(dw=P + 2), ALIGN), (dict(dx=P + 1), ALIGN), (dict(ws=0), WORKSPACE), (dict(ws=P + 8), WORKSPACE), (dict(wb=4 * 64 - 1), WORKSPACE)])
def test_rms_norm_backward(lib, change, want):
    assert rms_back(lib, **change) == want


HEAD = [(dict(x=0), NULL), (dict(w=0), NULL), (dict(t=0), NULL), (dict(stats=0), NULL), (dict(dt=3), DTYPE), (dict(N=-1), SHAPE), (dict(D=0), SHAPE),
        (dict(V=0), SHAPE), (dict(N=1 << 30), SHAPE), (dict(V=1 << 30), SHAPE), (dict(D=1 << 30), SHAPE), (dict(D=60), UNSUP), (dict(x=P + 8), ALIGN),
        (dict(w=P + 8), ALIGN), (dict(t=P + 4), ALIGN), (dict(stats=P + 2), ALIGN), (dict(ws=0), WORKSPACE), (dict(ws=P + 8), WORKSPACE), (dict(wb=8), WORKSPACE)]


@pytest.mark.parametrize("change,want", HEAD + [(dict(loss=0), NULL), (dict(loss=P + 2), ALIGN)])
def test_cross_entropy(lib, change, want):
    assert ce(lib, **change) == want


@pytest.mark.parametrize("change,want", HEAD + [(dict(dl=0), NULL), (dict(dl=P + 2), ALIGN), (dict(dx=P + 8), ALIGN), (dict(dw=P + 8), ALIGN)])
def test_cross_entropy_backward(lib, change, want):
    assert ce_back(lib, **change) == want


KD = [(dict(x=0), NULL), (dict(i=0), NULL), (dict(v=0), NULL), (dict(stats=0), NULL), (dict(dt=2), DTYPE), (dict(N=-1), SHAPE), (dict(V=0, k=1), SHAPE),
      (dict(ld=99), SHAPE), (dict(V=(1 << 24) + 1, ld=1 << 25), SHAPE), (dict(N=1 << 28), SHAPE), (dict(N=1 << 27, V=1 << 24, ld=1 << 24), SHAPE),
      (dict(k=0), SHAPE), (dict(k=129, V=200, ld=200), SHAPE), (dict(k=101), SHAPE), (dict(T=0.0), VALUE), (dict(T=-1.0), VALUE), (dict(T=NAN), VALUE),
      (dict(T=float("inf")), VALUE), (dict(x=P + 1), ALIGN), (dict(i=P + 2), ALIGN), (dict(v=P + 2), ALIGN), (dict(stats=P + 8), ALIGN)]


KD += [(dict(T=4e-39), VALUE), (dict(T=1e-45), VALUE)]  # log2(e) / T is infinite


@pytest.mark.parametrize("call", [rms, rms8])
def test_sums_go_over_no_other_row(lib, call):
    """In place of rows that are not packed."""
    assert call(lib, ldx=128) == SHAPE and call(lib, ldr=72) == SHAPE
    assert call(lib, x=0, N=0, ldx=128, h=0) == OK


def test_gradients_go_over_no_other_row(lib):
    assert kd_back(lib, ldd=101) == SHAPE and kd_back(lib, ld=101) == SHAPE


LONG = dict(N=1, V=1 << 24, ld=1 << 24)  # one row for many blocks, too long for a cluster


@pytest.mark.parametrize("change,want", KD + [(dict(loss=0), NULL), (dict(loss=P + 2), ALIGN), (dict(ws=0, **LONG), WORKSPACE),
                                              (dict(ws=P + 8, **LONG), WORKSPACE), (dict(wb=8, **LONG), WORKSPACE)])
def test_distillation(lib, change, want):
    assert kd(lib, **change) == want


@pytest.mark.parametrize("change,want", KD + [(dict(dl=0), NULL), (dict(dx=0), NULL), (dict(ldd=99), SHAPE), (dict(dl=P + 2), ALIGN), (dict(dx=P + 1), ALIGN)])
def test_distillation_backward(lib, change, want):
    assert kd_back(lib, **change) == want


def test_nothing_to_do_needs_no_device(lib):
    assert rms(lib, N=0, x=0, y=0, h=0, r=0) == OK
    assert rms8(lib, N=0, x=0, q=0, scales=0, h=0, r=0) == OK
    assert ce(lib, N=0, x=0, t=0, loss=0, stats=0, ws=0, wb=0) == OK
    assert kd(lib, N=0, x=0, i=0, v=0, loss=0, stats=0, ws=0, wb=0) == OK
    assert kd_back(lib, N=0, x=0, i=0, v=0, stats=0, dx=0, dl=0) == OK
    assert rms_back(lib, N=0, dy=0, h=0, dh=0, rstd=0, dx=0, dw=0, ws=0, wb=0) == OK
    assert ce_back(lib, N=0, x=0, t=0, dl=0, stats=0, dx=0, dw=0, ws=0, wb=0) == OK


def test_workspace_sizes(lib):
    assert lib.cci_rms_norm_workspace_size(0, 64) == 0 and lib.cci_rms_norm_workspace_size(4, 0) == 0
    assert lib.cci_rms_norm_workspace_size(1, 64) == 256
    for N, V in ((0, 100000), (1, 0), (1, (1 << 24) + 1), (5, 2048), (100000, 50000)):
        assert lib.cci_distillation_workspace_size(N, V) == 0
    assert lib.cci_distillation_workspace_size(1, 1 << 24) >= 8
    for call in (cci.HEAD_FORWARD, cci.HEAD_BACKWARD):
        for bad in ((2, 4, 64, 100), (1, 0, 64, 100), (1, 4, 0, 100), (1, 4, 64, 0), (1, 1 << 30, 64, 100)):
            assert lib.cci_head_workspace_size(call, *bad) == 0
        assert lib.cci_head_workspace_size(call, 1, 4, 64, 100) > 0
    assert lib.cci_head_workspace_size(2, 1, 4, 64, 100) == 0
    # pieces of the vocabulary: far below the logits' own bytes
    logits = 2 * 16384 * 131072
    assert lib.cci_head_workspace_size(cci.HEAD_FORWARD, 1, 16384, 4096, 131072) < logits // 8
    assert lib.cci_head_workspace_size(cci.HEAD_BACKWARD, 1, 16384, 4096, 131072) < logits // 4
