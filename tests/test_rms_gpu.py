"""Root-mean-square norm with the residual's addition, its 8-bit form and its backward pass against the formulas in 64
bits, and the gradient against differences.

Tolerances, with u = 2^-24 and n = 64 + D / 1024 roundings on the way of any sum over a row (as in a row's sums of
layer norm):
  h     u |s| for the addition and the output's rounding: 2^-8 of it in bf16, none in fp32
  rstd  (n / 2 + 4) u of it: the sum's error counts half
  y     (n + 8) u |y| and the output's rounding, 2^-8 in bf16, u in fp32
  scale (n + 10) u of it;  q: half a step of e4m3, 2^-4 of the value, or of a subnormal step, 2^-10, and (2 n + 20) u of
        the value for y's and the scale's errors
  dx    n u rstd (|g| + |xh| mean |g xh|) + 2 u |dh| + 2 u |dx|, and 2^-8 |dx| in bf16
  dweight  (64 + N / 64) u times the sum of the terms' magnitudes
"""
import pytest
import torch

import paper_1910_11971_gb300 as cci

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
LEAST = 2.0 ** -126

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def rows(N, D, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((N, D), generator=g) * scale * (0.5 + torch.rand((N, 1), generator=g))).to(DTYPES[dtype])


def weight(D, seed):
    return 1.0 + 0.3 * torch.randn(D, generator=torch.Generator().manual_seed(seed + 99))


def half(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


def reference(x, r, w, eps=EPS):
    s = x.double() + (0.0 if r is None else r.double())
    rstd = 1.0 / torch.sqrt((s * s).mean(1) + eps)
    return s, rstd, s * rstd[:, None] * (1.0 if w is None else w.double())


def check(got, x, r, w, dtype, eps=EPS):
    y, h, rstd = (t.cpu() for t in got)
    s, rs, want = reference(x, r, w, eps)
    n = 64 + x.shape[1] / 1024
    assert y.dtype == x.dtype and h.dtype == x.dtype and rstd.dtype == torch.float32
    assert ((h.double() - s).abs() <= (half(dtype) + 2 * U) * s.abs()).all()
    assert ((rstd.double() - rs).abs() <= (n / 2 + 4) * U * rs).all()
    assert ((y.double() - want).abs() <= ((n + 8) * U + half(dtype)) * want.abs() + 1e-40).all()


def check_fp8(got, x, r, w, group, dtype):
    q, scales, h, rstd = (t.cpu() for t in got)
    s, rs, want = reference(x, r, w)
    N, D = x.shape
    n = 64 + D / 1024
    width = group or D
    assert q.dtype == torch.float8_e4m3fn and scales.shape == (N, -(-D // width))
    assert ((h.double() - s).abs() <= (half(dtype) + 2 * U) * s.abs()).all()
    assert ((rstd.double() - rs).abs() <= (n / 2 + 4) * U * rs).all()
    for i in range(scales.shape[1]):
        y, v, sc = want[:, i * width:(i + 1) * width], q[:, i * width:(i + 1) * width].double(), scales[:, i].double()
        least = (y.abs().max(1).values / 448).clamp(min=LEAST)
        assert ((sc - least).abs() <= (n + 10) * U * least).all()
        e = y / sc[:, None]
        assert ((v - e).abs() <= torch.maximum(2.0 ** -4 * e.abs(), torch.tensor(2.0 ** -10, dtype=torch.float64)) + (2 * n + 20) * U * e.abs()).all()


# widths at both sides of every row layout, of whole vectors and odd
WIDTHS = [1, 2, 7, 8, 33, 120, 128, 136, 255, 256, 257, 264, 512, 520, 1000, 1001, 1024, 1032, 2047, 2048, 2056, 4096, 4100, 4104,
          8192, 8200, 9999, 16384, 16385, 20000]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(dev, D, dtype):
    N = 37 if D < 4096 else 5
    x, r, w = rows(N, D, dtype, D, 0.5), rows(N, D, dtype, D + 1, 2.0), weight(D, D)
    check(cci.rms_norm(x.to(dev), w.to(dev), residual=r.to(dev)), x, r, w, dtype)
    check(cci.rms_norm(x.to(dev), w.to(dev)), x, None, w, dtype)
    if D % 8 == 0:
        for group in (0, 128):
            check_fp8(cci.rms_norm_fp8(x.to(dev), w.to(dev), residual=r.to(dev), group=group), x, r, w, group, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D", [(1, 4096), (1, 1), (3000, 40), (1500, 1024), (1300, 264), (700, 2048)])
def test_forward_rows(dev, N, D, dtype):
    x, r = rows(N, D, dtype, N, 0.5), rows(N, D, dtype, N + 1)
    check(cci.rms_norm(x.to(dev), residual=r.to(dev)), x, r, None, dtype)
    check(cci.rms_norm(x.to(dev), eps=0.25), x, None, None, dtype, eps=0.25)
    if D % 8 == 0:
        check_fp8(cci.rms_norm_fp8(x.to(dev), group=128), x, None, None, 128, dtype)
        check_fp8(cci.rms_norm_fp8(x.to(dev), residual=r.to(dev)), x, r, None, 0, dtype)


def test_without_residual_h_is_x(dev):
    x = rows(3, 64, "bf16", 1).to(dev)
    assert cci.rms_norm(x)[1] is x and cci.rms_norm_fp8(x)[2] is x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 1000, 1001, 4096])
@pytest.mark.parametrize("pad,off", [(8, 0), (3, 0), (16, 8), (5, 1)])
def test_strides(dev, D, pad, off, dtype):
    """Rows inside wider ones, from any place on, x and residual with strides of their own."""
    N = 50
    x, r, w = rows(N, D + pad, dtype, D, 0.5), rows(N, D + 2 * pad, dtype, D + 1), weight(D, 0)
    xs, rs = x[:, off:off + D], r[:, off:off + D]
    xd, rd = x.to(dev)[:, off:off + D], r.to(dev)[:, off:off + D]
    check(cci.rms_norm(xd, w.to(dev), residual=rd), xs, rs, w, dtype)
    wide = torch.zeros(D + 1, device=dev)
    wide[1:] = w.to(dev)
    check(cci.rms_norm(xd, wide[1:], residual=rd), xs, rs, w, dtype)  # a weight off 16 bytes


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D", [(2000, 512), (1000, 4096), (5, 20000), (900, 77)])
def test_the_residual_stream_in_place(dev, N, D, dtype):
    x, r, w = rows(N, D, dtype, 5, 0.5), rows(N, D, dtype, 6), weight(D, 7)
    stream = r.to(dev)
    y, h, rstd = cci.rms_norm(x.to(dev), w.to(dev), residual=stream, h=stream)
    assert h is stream
    check((y, h, rstd), x, r, w, dtype)
    if D % 8 == 0:
        stream = r.to(dev)
        got = cci.rms_norm_fp8(x.to(dev), w.to(dev), residual=stream, h=stream, group=128)
        check_fp8(got, x, r, w, 128, dtype)


def test_rows_of_zeros_nan_and_inf_keep_to_themselves(dev):
    x = rows(40, 512, "f32", 9)
    x[3] = 0.0
    x[5, 7] = float("nan")
    x[9, 400] = float("inf")
    q, scales, h, rstd = cci.rms_norm_fp8(x.to(dev), group=128)
    y, _, _ = cci.rms_norm(x.to(dev))
    q, scales, y = q.cpu().float(), scales.cpu(), y.cpu()
    assert (y[3] == 0).all() and (q[3] == 0).all() and (scales[3] == LEAST).all()
    assert y[5].isnan().all() and q[5].isnan().all() and scales[5].isnan().all()
    assert y[9, 400].isnan() and (y[9, :400] == 0).all() and q[9, 400].isnan()
    good = [i for i in range(40) if i not in (3, 5, 9)]
    check_fp8((q[good].to(torch.float8_e4m3fn), scales[good], h.cpu()[good], rstd.cpu()[good]), x[good], None, None, 128, "f32")


def test_tiny_rows_have_finite_scales(dev):
    x = rows(4, 256, "f32", 10) * 1e-30
    q, scales, _, _ = cci.rms_norm_fp8(x.to(dev), torch.full((256,), 1e-12, device=dev), eps=1e-5, group=0)
    assert (scales == LEAST).all() and q.float().isfinite().all()


def test_the_same_call_gives_the_same_bits(dev):
    x, dy = rows(3000, 1001, "bf16", 1).to(dev), rows(3000, 1001, "bf16", 2).to(dev)
    y, h, rstd = cci.rms_norm(x)
    a, b = cci.rms_norm_backward(dy, h, rstd), cci.rms_norm_backward(dy, h, rstd)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- backward ----

def backward64(dy, h, rstd, w, dh):
    dy, h, r = dy.double(), h.double(), rstd.double()[:, None]
    xh, g = h * r, dy * (1.0 if w is None else w.double())
    dx = r * (g - xh * (g * xh).mean(1, keepdim=True)) + (0.0 if dh is None else dh.double())
    return dx, (dy * xh).sum(0), xh, g, r


def check_backward(got, dy, h, rstd, w, dh, dtype):
    dx, dw = (t.cpu() for t in got)
    want, dwant, xh, g, r = backward64(dy, h, rstd, w, dh)
    N, D = h.shape
    n = 64 + D / 1024
    tol = n * U * r * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True)) + 2 * U * want.abs()
    if dh is not None:
        tol = tol + 2 * U * dh.double().abs()
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * want.abs()
    assert dx.dtype == h.dtype and ((dx.double() - want).abs() <= tol).all()
    assert ((dw.double() - dwant).abs() <= (64 + N / 64) * U * (dy.double() * xh).abs().sum(0)).all()


def backward_inputs(N, D, dtype, seed):
    h, dy, dh = rows(N, D, dtype, seed, 2.0), rows(N, D, dtype, seed + 1, 0.1), rows(N, D, dtype, seed + 2, 0.1)
    return h, dy, dh, weight(D, seed), reference(h, None, None)[1].float()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(dev, D, dtype):
    h, dy, dh, w, rstd = backward_inputs(37 if D < 4096 else 5, D, dtype, D)
    d = [t.to(dev) for t in (dy, h, rstd, w)]
    check_backward(cci.rms_norm_backward(*d, dh=dh.to(dev)), dy, h, rstd, w, dh, dtype)
    check_backward(cci.rms_norm_backward(*d), dy, h, rstd, w, None, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D", [(1, 4096), (1, 1), (5000, 40), (2500, 1024), (3000, 264), (1000, 2056), (700, 4096), (400, 8192), (200, 16384), (40, 17000), (1003, 1001)])
def test_backward_rows(dev, N, D, dtype):
    h, dy, dh, w, rstd = backward_inputs(N, D, dtype, N)
    check_backward(cci.rms_norm_backward(dy.to(dev), h.to(dev), rstd.to(dev), dh=dh.to(dev)), dy, h, rstd, None, dh, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 1001, 4096])
@pytest.mark.parametrize("pad,off", [(8, 0), (3, 0), (5, 1)])
def test_backward_strides(dev, D, pad, off, dtype):
    N = 60
    big = [rows(N, D + k * pad, dtype, D + k, 0.5) for k in (1, 2, 3)]
    dy, h, dh = (b[:, off:off + D] for b in big)
    w, rstd = weight(D, 1), reference(h, None, None)[1].float()
    out = torch.empty((N, D), dtype=DTYPES[dtype], device=dev)
    got = cci.rms_norm_backward(*(b.to(dev)[:, off:off + D] for b in big[:2]), rstd.to(dev), w.to(dev), dh=big[2].to(dev)[:, off:off + D], out=out)
    assert got[0] is out
    check_backward(got, dy, h, rstd, w, dh, dtype)


def test_no_rows(dev):
    e, w = torch.empty((0, 64), device=dev), torch.ones(64, device=dev)
    y, h, rstd = cci.rms_norm(e, w, residual=e)
    assert y.shape == (0, 64) and h.shape == (0, 64) and rstd.shape == (0,)
    q, scales, _, _ = cci.rms_norm_fp8(e, w, group=128)
    assert q.shape == (0, 64) and scales.shape == (0, 1)
    dx, dw = cci.rms_norm_backward(e, e, rstd, w)
    assert dx.shape == (0, 64) and (dw == 0).all()


def test_gradient_against_differences(dev):
    """d/dx and d/dw of sum(y * a + h * b), by central differences of the formula in 64 bits."""
    N, D = 3, 40
    x, r, w = rows(N, D, "f32", 1), rows(N, D, "f32", 2), weight(D, 3)
    a, b = rows(N, D, "f32", 4), rows(N, D, "f32", 5)
    y, h, rstd = cci.rms_norm(x.to(dev), w.to(dev), residual=r.to(dev))
    dx, dw = cci.rms_norm_backward(a.to(dev), h, rstd, w.to(dev), dh=b.to(dev))

    def value(x64, w64):
        s, _, out = reference(x64, r, w64)
        return float((out * a.double()).sum() + (s * b.double()).sum())

    # the third derivative of a row's norm is of the order of 10; h is rounded to fp32
    step = 1e-4
    x64, w64 = x.double(), w.double()
    for n, c in ((0, 0), (1, 7), (2, 39)):
        hi, lo = x64.clone(), x64.clone()
        hi[n, c] += step
        lo[n, c] -= step
        assert abs((value(hi, w64) - value(lo, w64)) / (2 * step) - float(dx[n, c])) <= 1e-5
        hi, lo = w64.clone(), w64.clone()
        hi[c] += step
        lo[c] -= step
        assert abs((value(x64, hi) - value(x64, lo)) / (2 * step) - float(dw[c])) <= 1e-5
