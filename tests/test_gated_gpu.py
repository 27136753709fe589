"""The gated feed-forward block and its gradients against the formulas in 64 bits.

Tolerances, u = 2^-24, S the sum of the magnitudes |x||w| of a product's terms.  The tensor core adds a product's
terms in fp32 in groups; every addition may cut (not round) at the running sum: K / 16 groups of at most four
alignments each, so a pre-activation is off by at most E = (K / 4 + 32) 2 u S (fp32 the same, six products deep:
its planes drop below 2^-25 of a term, and six times the additions: 6 K / 4).
  h      |act'| Eg |u| + |act| Eu + 16 u |h|, |act'| at most 1.2
  dg, du the same through the product with dh, and half a bf16 unit (2^-8 of the magnitude, bf16 only)
  dX, dW the terms' errors in dg and du times the other operand, summed, plus E of the product itself
plus 2^-8 of a bf16 output's magnitude.
"""
import math

import pytest
import torch

import paper_1910_11971_gb300 as cci
from paper_1910_11971_gb300 import workloads as wl

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = list(cci.ACTIVATIONS)


def act64(g, act):
    if act == "silu":
        return g * torch.sigmoid(g)
    if act == "gelu":
        return g * torch.special.ndtr(g)
    if act == "gelu_tanh":
        return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)))
    if act == "relu":
        return g * (g > 0)
    return torch.sigmoid(g)


def slope64(g, act):
    g = g.detach().requires_grad_(True)
    return torch.autograd.grad(act64(g, act).sum(), g)[0]


def inputs(N, D, F, dtype, seed, dev):
    g = torch.Generator().manual_seed(seed)
    dt = DTYPES[dtype]
    x = torch.randn((N, D), generator=g).to(dt)
    wg = (torch.randn((F, D), generator=g) * math.sqrt(2.0 / D)).to(dt)
    wu = (torch.randn((F, D), generator=g) * math.sqrt(1.0 / D)).to(dt)
    dh = (torch.randn((N, F), generator=g) * 0.1).to(dt)
    return [t.to(dev) for t in (x, wg, wu, dh)]


def sum_error(K, dtype):
    return ((6 if dtype == "f32" else 1) * K / 4 + 32) * 2 * U


class Reference:
    """Values and error bounds in 64 bits (on the GPU, by elementary products)."""

    def __init__(self, x, wg, wu, act, dtype, dh=None):
        x, wg, wu = x.double(), wg.double(), wu.double()
        D, K = x.shape[1], x.shape[1]
        self.g, self.u = x @ wg.t(), x @ wu.t()
        e = sum_error(K, dtype)
        eg, eu = e * (x.abs() @ wg.abs().t()), e * (x.abs() @ wu.abs().t())
        self.eg, self.eu = eg, eu
        a, s = act64(self.g, act), slope64(self.g, act)
        half = 2.0 ** -8 if dtype == "bf16" else 2 * U
        self.h = a * self.u
        # act has slopes of at most 1.2; the error moves u's factor too
        da = 1.2 * eg + 16 * U * a.abs()
        self.h_tol = da * (self.u.abs() + eu) + a.abs() * eu + (16 * U + half) * self.h.abs() + 1e-30
        if dh is None:
            return
        dh = dh.double()
        self.dg, self.du = dh * self.u * s, dh * a
        # act' moves by at most 1.2 |dg| (its own slope; ReLU: checked apart from the kink)
        ds = 1.2 * eg + 16 * U * (1 + s.abs())
        if act == "relu":
            ds = torch.where(self.g.abs() <= eg, torch.ones_like(ds), torch.zeros_like(ds))
        part = 2.0 ** -8 if dtype == "bf16" else 2 * U
        tg = dh.abs() * (ds * (self.u.abs() + eu) + s.abs() * eu) + part * self.dg.abs() * (1 + 2.0 ** -8)
        tu = dh.abs() * da + part * self.du.abs() * (1 + 2.0 ** -8)
        ex, ew = sum_error(2 * wg.shape[0], dtype), sum_error(x.shape[0], dtype)
        self.dx = self.dg @ wg + self.du @ wu
        self.dx_tol = ((tg + ex * self.dg.abs()) @ wg.abs() + (tu + ex * self.du.abs()) @ wu.abs()) * 1.01 + half * self.dx.abs() + 1e-30
        self.dwg, self.dwu = self.dg.t() @ x, self.du.t() @ x
        self.dwg_tol = (tg + ew * self.dg.abs()).t() @ x.abs() * 1.01 + half * self.dwg.abs() + 1e-30
        self.dwu_tol = (tu + ew * self.du.abs()).t() @ x.abs() * 1.01 + half * self.dwu.abs() + 1e-30


def near(a, r, tol, what):
    assert a.shape == r.shape and torch.isfinite(a).all(), what
    err = (a.double() - r).abs()
    assert (err <= tol).all(), f"{what}: off by up to {float((err / tol).max())} of the tolerance"
    return float(err.norm() / r.norm().clamp(min=1e-300))


def whole(dtype):
    """Norm of the error over the norm of the result: one bf16 rounding of the result and one of dg or du
    (2^-8 / sqrt(3) of a magnitude each at most), or fp32 sums."""
    return 2 * 2.0 ** -8 / math.sqrt(3.0) if dtype == "bf16" else 4e-6


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def run_all(dev, N, D, F, dtype, act, seed=None):
    x, wg, wu, dh = inputs(N, D, F, dtype, seed or N + D + F, dev)
    ref = Reference(x, wg, wu, act, dtype, dh)
    st = cci.new_status(dev)
    h = cci.gated_linear(x, wg, wu, act=act, status=st)
    h2, g, u = cci.gated_linear(x, wg, wu, act=act, save=True, status=st)
    assert torch.equal(h, h2) and h.dtype == x.dtype
    assert near(h, ref.h, ref.h_tol, "h") <= whole(dtype)
    # bf16: one running sum, cut by half a unit in the mean at each of its D / 16 additions
    cut = 4e-6 if dtype == "f32" else 1e-6 + D / 16 * U
    assert near(g, ref.g, ref.eg, "g") <= cut and near(u, ref.u, ref.eu, "u") <= cut
    dx, dwg, dwu = cci.gated_linear_backward(dh, x, wg, wu, g, u, act=act, status=st)
    assert cci.read_status(st) == 0
    for got, name in ((dx, "dx"), (dwg, "dwg"), (dwu, "dwu")):
        assert got.dtype == x.dtype
        assert near(got, getattr(ref, name), getattr(ref, name + "_tol"), name) <= whole(dtype), name


# one token to more tokens than a pair tile, widths below, at and past the tiles' (32, 64, 128, 256) and the
# stage's 64, none a multiple of them but some
SIZES = [(1, 8, 8), (1, 64, 32), (2, 72, 40), (7, 136, 200), (8, 256, 128), (31, 1000, 264), (65, 512, 1000), (127, 328, 136),
         (128, 128, 128), (129, 200, 72), (200, 1024, 504), (255, 64, 512), (257, 264, 264), (300, 72, 1032), (513, 512, 256)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,F", SIZES)
def test_block_and_gradients(dev, N, D, F, dtype):
    run_all(dev, N, D, F, dtype, ACTS[(N + D + F) // 8 % len(ACTS)])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activations(dev, act, dtype):
    run_all(dev, 70, 128, 96, dtype, act, seed=3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,D,F", [("bf16", 3000, 1024, 2048), ("bf16", 1111, 2048, 5000), ("bf16", 4096, 520, 4096), ("bf16", 1, 4096, 4096),
                                         ("bf16", 40, 4096, 2048), ("f32", 700, 512, 1032), ("f32", 2100, 264, 2048), ("f32", 1, 2048, 1024)])
def test_large(dev, N, D, F, dtype):
    run_all(dev, N, D, F, dtype, "silu")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_integers_are_exact(dev, dtype):
    """Small whole numbers: products and sums are exact, so every place of the tiles is checked bit for bit
    (g, u, and with ReLU and dh of whole numbers the gradients, as long as they fit the type)."""
    N, D, F = 300, 200, 328
    x = wl.integer_valued((N, D), -2, 2, 1).to(DTYPES[dtype]).to(dev)
    wg = wl.integer_valued((F, D), -1, 1, 2).to(DTYPES[dtype]).to(dev)
    wu = wl.integer_valued((F, D), -1, 1, 3).to(DTYPES[dtype]).to(dev)
    dh = wl.integer_valued((N, F), -1, 1, 4).to(DTYPES[dtype]).to(dev)
    _, g, u = cci.gated_linear(x, wg, wu, act="relu", save=True)
    gr, ur = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    assert torch.equal(g.double(), gr) and torch.equal(u.double(), ur)
    dx, dwg, dwu = cci.gated_linear_backward(dh, x, wg, wu, g, u, act="relu")
    dg, du = dh.double() * ur * (gr > 0), dh.double() * gr.clamp(min=0)
    for got, ref in ((dx, dg @ wg.double() + du @ wu.double()), (dwg, dg.t() @ x.double()), (dwu, du.t() @ x.double())):
        assert torch.equal(got.double(), ref.float().to(DTYPES[dtype]).double())  # |g|, |u| < 256: exact as bf16


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(dev, act):
    """The directional derivative of sum(dh h) by central differences of the 64-bit block, step 1e-4: error of
    order h^2 and 2^-52 / h, both under 1e-6 of the terms' magnitudes; fp32 gradients add 4e-6."""
    N, D, F, s = 9, 40, 48, 1e-4
    x, wg, wu, dh = inputs(N, D, F, "f32", 11, dev)
    gen = torch.Generator().manual_seed(5)
    vx, vg, vu = (torch.randn(t.shape, generator=gen).double().to(dev) for t in (x, wg, wu))
    _, g, u = cci.gated_linear(x, wg, wu, act=act, save=True)
    dx, dwg, dwu = cci.gated_linear_backward(dh, x, wg, wu, g, u, act=act)

    def loss(t):
        a, b, c = x.double() + t * vx, wg.double() + t * vg, wu.double() + t * vu
        gg = a @ b.t()
        if act == "relu":  # the side of the kink that the forward pass took
            return (dh.double() * torch.where(g > 0, gg, 0.0) * (a @ c.t())).sum()
        return (dh.double() * act64(gg, act) * (a @ c.t())).sum()

    numeric = (loss(s) - loss(-s)) / (2 * s)
    terms = [dx.double() * vx, dwg.double() * vg, dwu.double() * vu]
    assert abs(sum(t.sum() for t in terms) - numeric) <= 5e-6 * sum(t.abs().sum() for t in terms)


PACKED = [(1, 64, 64, 4, 2), (16, 1024, 512, 8, 2), (33, 72, 96, 32, 8), (200, 264, 320, 16, 3), (5, 40, 512, 256, 9), (130, 520, 192, 64, 64),
          (7, 136, 128, 128, 1), (300, 512, 1024, 8, 4), (3, 8, 24, 3, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,F,G,K", PACKED)
def test_packed(dev, N, D, F, G, K, dtype):
    """Packed weights give the bits of their dense form."""
    x, wg, wu, _ = inputs(N, D, F, dtype, N + F, dev)
    gate, up = cci.pack(wg, G, K), cci.pack(wu, G, K)
    st = cci.new_status(dev)

    def dense(v, i):
        w = torch.zeros((F // G, D, G), dtype=v.dtype, device=dev)
        return w.scatter_(2, i.long(), v).permute(0, 2, 1).reshape(F, D).contiguous()

    h = cci.gated_linear_packed(x, gate, up, F, G, K, act="gelu", status=st)
    assert cci.read_status(st) == 0
    wgd, wud = dense(*gate), dense(*up)
    ref = Reference(x, wgd, wud, "gelu", dtype)
    assert near(h, ref.h, ref.h_tol, "h") <= whole(dtype)
    assert torch.equal(h, cci.gated_linear(x, wgd, wud, act="gelu"))


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1])
def test_packed_reports_bad_index_sets(dev, which):
    N, D, F, G, K = 4, 64, 64, 8, 4
    x, wg, wu, _ = inputs(N, D, F, "bf16", 1, dev)
    for bad in ([0, 1, 2, G], [0, 1, 1, 2], [0, 2, 1, 3], [255, 1, 2, 3]):
        pairs = [cci.pack(wg, G, K), cci.pack(wu, G, K)]
        pairs[which][1][-1, -1] = torch.tensor(bad, dtype=torch.uint8)
        st = cci.new_status(dev)
        cci.gated_linear_packed(x, pairs[0], pairs[1], F, G, K, status=st)
        assert cci.read_status(st) == 10, bad


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_and_nan_inputs_stay_in_their_rows(dev, dtype):
    N, D, F = 150, 200, 136
    x, wg, wu, _ = inputs(N, D, F, dtype, 2, dev)
    clean = cci.gated_linear(x, wg, wu)
    y = x.clone()
    y[3, 100], y[140, 0] = float("inf"), float("nan")
    h = cci.gated_linear(y, wg, wu)
    assert (~torch.isfinite(h[[3, 140]])).all()
    keep = [i for i in range(N) if i not in (3, 140)]
    assert torch.equal(h[keep], clean[keep])


@pytest.mark.gpu
def test_large_finite_values_split(dev):
    """fp32 values next to the type's largest, and tiny ones, keep their planes finite."""
    N, D, F = 8, 16, 16
    x = torch.full((N, D), 0.0, device=dev)
    x[0, 0], x[1, 0], x[2, 0] = 3.4028234e38, 1e-30, -3.4e38
    w = torch.zeros((F, D), device=dev)
    w[:, 0] = 0.5
    _, g, u = cci.gated_linear(x, w, w, act="relu", save=True)
    assert torch.isfinite(g).all()
    r = x.double()[:, :1] * 0.5
    assert ((g.double() - r).abs() <= 2.0 ** -23 * r.abs()).all()


@pytest.mark.gpu
def test_parts_empty_and_streams(dev):
    N, D, F = 40, 128, 64
    x, wg, wu, dh = inputs(N, D, F, "bf16", 4, dev)
    _, g, u = cci.gated_linear(x, wg, wu, save=True)
    dx, dwg, dwu = cci.gated_linear_backward(dh, x, wg, wu, g, u)
    only_x = cci.gated_linear_backward(dh, x, wg, wu, g, u, need_dw=False)
    only_w = cci.gated_linear_backward(dh, x, wg, wu, g, u, need_dx=False)
    assert torch.equal(only_x[0], dx) and only_x[1] is None and only_x[2] is None
    assert only_w[0] is None and torch.equal(only_w[1], dwg) and torch.equal(only_w[2], dwu)
    e = torch.empty((0, D), dtype=torch.bfloat16, device=dev)
    h, g0, u0 = cci.gated_linear(e, wg, wu, save=True)
    assert h.shape == (0, F)
    dx0, dw0, du0 = cci.gated_linear_backward(h, e, wg, wu, g0, u0)
    assert dx0.shape == (0, D) and (dw0 == 0).all() and (du0 == 0).all()
    s = torch.cuda.Stream(dev)
    with torch.cuda.stream(s):
        a = torch.randn((4096, 4096), device=dev)
        late = x + ((a @ a)[:N, :D] * 0).to(x.dtype)
        h1 = cci.gated_linear(late, wg, wu)
    s.synchronize()
    assert torch.equal(h1, cci.gated_linear(x, wg, wu))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_of_other_sizes_leave_nothing_behind(dev, dtype):
    """A pass, passes of other sizes, the pass again: the same bits."""
    sizes = [(5, 64, 64), (300, 512, 264), (64, 1000, 40)]
    first = []
    for n in range(2):
        for k, (N, D, F) in enumerate(sizes):
            x, wg, wu, dh = inputs(N, D, F, dtype, k, dev)
            h, g, u = cci.gated_linear(x, wg, wu, save=True)
            got = (h, *cci.gated_linear_backward(dh, x, wg, wu, g, u))
            if n:
                assert all(torch.equal(a, b) for a, b in zip(first[k], got))
            else:
                first.append(got)


FAKE = 0x10000
OK, NULL, SHAPE, GROUP, DTYPE, ALIGN, VALUE, UNSUP, WORKSPACE = 0, 1, 2, 3, 4, 5, 6, 9, 11


def test_refusals():
    lib = cci.lib()

    def fwd(X=FAKE, dt=1, N=4, D=16, Wg=FAKE, Wu=FAKE, F=16, act=0, H=FAKE, g=None, u=None, ws=None, n=0):
        return lib.cci_gated_linear(X, dt, N, D, Wg, Wu, F, act, H, g, u, None, ws, n, None)

    assert fwd(dt=2) == DTYPE
    assert fwd(X=None) == NULL and fwd(Wg=None) == NULL and fwd(Wu=None) == NULL and fwd(H=None) == NULL
    assert fwd(g=FAKE) == NULL and fwd(u=FAKE) == NULL
    assert fwd(N=-1) == SHAPE and fwd(D=0) == SHAPE and fwd(F=0) == SHAPE and fwd(N=1 << 30) == SHAPE
    assert fwd(act=5) == VALUE and fwd(act=-1) == VALUE
    assert fwd(D=12) == UNSUP and fwd(F=20) == UNSUP
    assert fwd(X=FAKE + 8) == ALIGN and fwd(Wu=FAKE + 8) == ALIGN and fwd(H=FAKE + 8) == ALIGN and fwd(g=FAKE + 4, u=FAKE) == ALIGN
    assert fwd(dt=0) == WORKSPACE and fwd(dt=0, ws=FAKE + 8, n=1 << 20) == WORKSPACE
    assert fwd(N=0, X=None, H=None) == OK and fwd(N=0, dt=0, X=None, H=None) == OK

    def packed(X=FAKE, dt=1, N=4, D=16, gv=FAKE, gi=FAKE, uv=FAKE, ui=FAKE, F=16, G=8, K=2, act=0, H=FAKE, ws=FAKE, n=1 << 20):
        return lib.cci_gated_linear_packed(X, dt, N, D, gv, gi, uv, ui, F, G, K, act, H, None, ws, n, None)

    assert packed(gi=None) == NULL and packed(uv=None) == NULL and packed(H=None) == NULL
    assert packed(G=3) == GROUP and packed(K=9) == GROUP and packed(G=0) == GROUP
    assert packed(ws=None) == WORKSPACE and packed(n=16) == WORKSPACE and packed(dt=5) == DTYPE

    def bwd(dH=FAKE, X=FAKE, dt=1, N=4, D=16, Wg=FAKE, Wu=FAKE, F=16, act=0, g=FAKE, u=FAKE, dX=FAKE, dWg=FAKE, dWu=FAKE, ws=FAKE, n=1 << 20):
        return lib.cci_gated_linear_backward(dH, X, dt, N, D, Wg, Wu, F, act, g, u, dX, dWg, dWu, None, ws, n, None)

    assert bwd(dH=None) == NULL and bwd(g=None) == NULL and bwd(dWg=None) == NULL and bwd(dWu=None) == NULL
    assert bwd(dX=FAKE + 8) == ALIGN and bwd(dH=FAKE + 8) == ALIGN and bwd(n=0) == WORKSPACE and bwd(act=7) == VALUE
    size = cci.lib().cci_gated_workspace_size
    assert size(0, 1, 4, 16, 16) == 0 and size(0, 0, 4, 16, 16) > 0 and size(2, 1, 4, 16, 16) > 0 and size(3, 1, 4, 16, 16) == 0
    host = torch.zeros((4, 16))
    with pytest.raises(ValueError):
        cci.gated_linear(host, host, host)
    with pytest.raises(ValueError):
        cci._act_code("swish")
