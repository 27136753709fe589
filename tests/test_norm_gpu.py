"""Layer norm and its backward pass against the formulas in 64 bits, and the gradient against differences.

Tolerances, with u = 2^-24 (fp32) and at most 64 roundings on the way of any sum over a row (16 in a thread,
10 in the trees, the rest in the few operations around them; rows over 16384 long: one more per 1024):
  y   64 u (kappa + |xh|) |w| + 2 u |b|, kappa = max|x| rstd (what the mean's error becomes in units of y)
  dx  64 u rstd (|g| + mean|g| + |xh| mean|g xh|)
  dweight, dbias  (64 + N / 64) u times the sum of the terms' magnitudes (a column's rows are added one by one
      in each block and the blocks' sums in turn)
plus half a unit in the last place of a bf16 output (2^-8 of its magnitude).
"""
import pytest
import torch

import paper_1910_11971_gb300 as cci

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def rows(N, D, dtype, seed, scale=1.0, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    return ((torch.randn((N, D), generator=g) + offset) * scale).to(DTYPES[dtype])


def params(D, seed):
    g = torch.Generator().manual_seed(seed + 99)
    return 1.0 + 0.3 * torch.randn(D, generator=g), 0.5 * torch.randn(D, generator=g)


def forward64(x, w, b, eps=EPS):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    xh = (x - mean) * rstd
    return xh * w + b, mean, rstd, xh


def check_forward(y, mean, rstd, x, w, b, dtype, eps=EPS):
    w = torch.ones(x.shape[1]).double() if w is None else w.double()
    b = torch.zeros(x.shape[1]).double() if b is None else b.double()
    yr, mr, rr, xh = forward64(x, w, b, eps)
    n = 64 + x.shape[1] / 1024
    top = x.double().abs().max(1, keepdim=True).values
    kappa = top * rr
    tol = n * U * (kappa + xh.abs()) * w.abs() + 2 * U * b.abs() + (2.0 ** -8 * yr.abs() if dtype == "bf16" else 2 * U * yr.abs())
    assert ((y.cpu().double() - yr).abs() <= tol).all()
    assert ((mean.cpu().double()[:, None] - mr).abs() <= n * U * top).all()
    # a mean off by d changes the variance by d^2 alone
    assert ((rstd.cpu().double()[:, None] - rr).abs() <= n * U * rr * (1 + (n * U * kappa) ** 2 / U)).all()


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


# widths at both sides of every row layout (256, 512, 1024, 2048, 4096, 8192, 16384), of whole vectors and odd
WIDTHS = [1, 2, 7, 8, 33, 255, 256, 257, 264, 511, 512, 520, 1000, 1001, 1024, 1032, 2047, 2048, 2056, 4096, 4100,
          5000, 8192, 8200, 9999, 16384, 16385, 20000]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_forward(dev, D, dtype):
    N = 37 if D < 4096 else 5
    x, (w, b) = rows(N, D, dtype, D, 2.0, 0.3), params(D, D)
    y, mean, rstd = cci.layer_norm(x.to(dev), w.to(dev), b.to(dev))
    assert y.dtype == x.dtype and y.shape == x.shape
    check_forward(y, mean, rstd, x, w, b, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D", [(1, 4096), (1, 1), (3000, 40), (700, 1024), (2500, 2048), (1300, 264)])
def test_forward_rows(dev, N, D, dtype):
    x, (w, b) = rows(N, D, dtype, N), params(D, N)
    check_forward(*cci.layer_norm(x.to(dev), w.to(dev), b.to(dev)), x, w, b, dtype)
    check_forward(*cci.layer_norm(x.to(dev), w.to(dev)), x, w, None, dtype)
    check_forward(*cci.layer_norm(x.to(dev), None, b.to(dev)), x, None, b, dtype)
    check_forward(*cci.layer_norm(x.to(dev), eps=0.25), x, None, None, dtype, eps=0.25)


@pytest.mark.gpu
def test_forward_far_offset(dev):
    """The variance is that of the differences: a row a thousand spreads from zero keeps it."""
    x = rows(16, 4096, "f32", 3, 1.0, 1000.0)
    check_forward(*cci.layer_norm(x.to(dev)), x, None, None, "f32")
    c = torch.full((4, 1000), 3.25)  # no spread at all
    y, mean, rstd = cci.layer_norm(c.to(dev))
    assert (y == 0).all() and (mean == 3.25).all()
    assert (rstd.double().cpu() - EPS ** -0.5).abs().max() <= 4 * U * EPS ** -0.5


def backward64(dy, x, mean, rstd, w):
    dy, x = dy.double(), x.double()
    xh = (x - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy * w.double()
    r = rstd.double()[:, None]
    dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), xh, g, r


def check_backward(dx, dw, db, dy, x, mean, rstd, w, dtype):
    w = torch.ones(x.shape[1]) if w is None else w
    dxr, dwr, dbr, xh, g, r = backward64(dy, x, mean, rstd, w)
    N, D = x.shape
    n = 64 + D / 1024
    tol = n * U * r * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    tol = tol + (2.0 ** -8 * dxr.abs() if dtype == "bf16" else 0.0)
    assert ((dx.cpu().double() - dxr).abs() <= tol).all()
    m = 64 + N / 64
    assert ((dw.cpu().double() - dwr).abs() <= m * U * (dy.double() * xh).abs().sum(0)).all()
    assert ((db.cpu().double() - dbr).abs() <= m * U * dy.double().abs().sum(0)).all()


def backward_inputs(N, D, dtype, seed):
    x, dy, (w, b) = rows(N, D, dtype, seed, 2.0, 0.3), rows(N, D, dtype, seed + 1, 0.1), params(D, seed)
    _, mean, rstd, _ = forward64(x, torch.ones(D).double(), torch.zeros(D).double())
    return x, dy, w, mean[:, 0].float(), rstd[:, 0].float()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_backward(dev, D, dtype):
    x, dy, w, mean, rstd = backward_inputs(37 if D < 4096 else 5, D, dtype, D)
    got = cci.layer_norm_backward(dy.to(dev), x.to(dev), mean.to(dev), rstd.to(dev), w.to(dev))
    assert got[0].dtype == x.dtype
    check_backward(*got, dy, x, mean, rstd, w, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D", [(1, 4096), (1, 8), (5000, 40), (3001, 264), (2000, 1024), (1500, 2048), (900, 4096), (400, 8192)])
def test_backward_rows(dev, N, D, dtype):
    x, dy, w, mean, rstd = backward_inputs(N, D, dtype, N)
    args = [t.to(dev) for t in (dy, x, mean, rstd)]
    check_backward(*cci.layer_norm_backward(*args, w.to(dev)), dy, x, mean, rstd, w, dtype)
    first = cci.layer_norm_backward(*args)
    check_backward(*first, dy, x, mean, rstd, None, dtype)
    for again in (cci.layer_norm_backward(*args), cci.layer_norm_backward(*args)):
        assert all(torch.equal(a, b) for a, b in zip(first, again))  # the same bits


@pytest.mark.gpu
@pytest.mark.parametrize("D", [24, 1001])
def test_gradient_against_differences(dev, D):
    """The directional derivative of L = sum(c * y) by central differences of the 64-bit forward pass.
    Step h: truncation h^2 / 6 of a third derivative of order one per spread, rounding 2^-52 / h: 1e-4 leaves
    both under 1e-6 of the sum of the terms' magnitudes; the kernel's own error is under 64 u of it."""
    N, h = 6, 1e-4
    x, dy, w, _, _ = backward_inputs(N, D, "f32", 5 * D)
    b = torch.zeros(D)
    _, mean, rstd = cci.layer_norm(x.to(dev), w.to(dev), b.to(dev))
    dx, dw, db = cci.layer_norm_backward(dy.to(dev), x.to(dev), mean, rstd, w.to(dev))
    g = torch.Generator().manual_seed(1)
    vx, vw, vb = (torch.randn(s, generator=g).double() for s in ((N, D), (D,), (D,)))

    def loss(s):
        return (dy.double() * forward64(x.double() + s * vx, w.double() + s * vw, b.double() + s * vb)[0]).sum()

    numeric = (loss(h) - loss(-h)) / (2 * h)
    terms = [(dx.cpu().double() * vx), (dw.cpu().double() * vw), (db.cpu().double() * vb)]
    size = sum(t.abs().sum() for t in terms)
    assert abs(sum(t.sum() for t in terms) - numeric) <= (1e-6 + 64 * U) * size


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,pad,shift", [(1024, 8, 0), (1000, 7, 0), (512, 0, 1), (2048, 3, 1)])
def test_strides_and_alignment(dev, D, pad, shift, dtype):
    """Rows with a stride, and views that start off a 16-byte boundary."""
    N = 19
    x, dy, w, mean, rstd = backward_inputs(N, D, dtype, D + pad)

    def view(t):
        flat = torch.full((shift + N * (D + pad),), float("nan"), dtype=t.dtype, device=dev)
        v = flat[shift:].view(N, D + pad)[:, :D]
        v.copy_(t)
        return v

    wv = torch.empty(D + 1, device=dev)[1:]
    wv.copy_(w)
    check_forward(*cci.layer_norm(view(x), wv), x, w, None, dtype)
    check_backward(*cci.layer_norm_backward(view(dy), view(x), mean.to(dev), rstd.to(dev), wv), dy, x, mean, rstd, w, dtype)


@pytest.mark.gpu
def test_empty_and_streams(dev):
    z = torch.empty((0, 64), device=dev)
    y, mean, rstd = cci.layer_norm(z)
    assert y.shape == (0, 64) and mean.numel() == 0
    dx, dw, db = cci.layer_norm_backward(z, z, mean, rstd)
    assert dx.shape == (0, 64) and (dw == 0).all() and (db == 0).all()
    # the current stream is used: the call runs behind a long product there
    s = torch.cuda.Stream(dev)
    x = rows(64, 4096, "f32", 1)
    with torch.cuda.stream(s):
        a = torch.randn((4096, 4096), device=dev)
        xd = (a @ a)[:64] * 0 + x.to(dev)
        y, mean, rstd = cci.layer_norm(xd)
    s.synchronize()
    check_forward(y, mean, rstd, x, None, None, "f32")


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_row(dev):
    x = rows(9, 1024, "f32", 4)
    x[2, 5], x[7, 1000] = float("inf"), float("nan")
    y, _, _ = cci.layer_norm(x.to(dev))
    y = y.cpu()
    assert y[[2, 7]].isnan().any(1).all()
    keep = [0, 1, 3, 4, 5, 6, 8]
    assert torch.equal(y[keep], cci.layer_norm(x[keep].to(dev))[0].cpu())


FAKE = 0x10000  # never dereferenced: refused before any launch
OK, NULL, SHAPE, DTYPE, ALIGN, VALUE, WORKSPACE = 0, 1, 2, 4, 5, 6, 11


def test_refusals():
    f, b = cci.lib().cci_layer_norm, cci.lib().cci_layer_norm_backward

    def fwd(x=FAKE, dt=0, N=4, D=8, ld=8, w=FAKE, bias=FAKE, eps=1e-5, y=FAKE, m=FAKE, r=FAKE):
        return f(x, dt, N, D, ld, w, bias, eps, y, m, r, None)

    assert fwd(dt=3) == DTYPE
    assert fwd(x=None) == NULL and fwd(y=None) == NULL and fwd(m=None) == NULL and fwd(r=None) == NULL
    assert fwd(N=-1) == SHAPE and fwd(D=0) == SHAPE and fwd(ld=7) == SHAPE and fwd(N=1 << 40, ld=1 << 30) == SHAPE
    assert fwd(eps=-1.0) == VALUE and fwd(eps=float("nan")) == VALUE
    assert fwd(x=FAKE + 2) == ALIGN and fwd(dt=1, y=FAKE + 1) == ALIGN and fwd(w=FAKE + 2) == ALIGN
    assert fwd(N=0, x=None, y=None, m=None, r=None) == OK

    def bwd(dy=FAKE, lddy=8, x=FAKE, ldx=8, dt=0, N=4, D=8, m=FAKE, r=FAKE, w=FAKE, dx=FAKE, dw=FAKE, db=FAKE, ws=FAKE, n=0):
        return b(dy, lddy, x, ldx, dt, N, D, m, r, w, dx, dw, db, ws, n, None)

    assert bwd(dt=3) == DTYPE and bwd(dy=None) == NULL and bwd(dx=None) == NULL and bwd(m=None) == NULL
    assert bwd(lddy=7) == SHAPE and bwd(ldx=7) == SHAPE and bwd(D=0) == SHAPE
    assert bwd(dw=FAKE + 2) == ALIGN and bwd(dt=1, dy=FAKE + 1) == ALIGN
    assert bwd() == WORKSPACE and bwd(ws=None, n=1 << 20) == WORKSPACE and bwd(ws=FAKE + 4, n=1 << 30) == WORKSPACE
    assert cci.lib().cci_layer_norm_workspace_size(0, 8) == 0
    host = torch.zeros((4, 8))
    with pytest.raises(ValueError):
        cci.layer_norm(host)
    with pytest.raises(ValueError):
        cci.layer_norm_backward(host, host, host[0], host[0])
