"""The gated block on both sides of the rules that choose its kernels: few tokens and more, reductions cut over
all SMs, packed weights read as they are or expanded, the activations over their whole range.

Whole numbers are exact in every one of them, so places are compared bit for bit; a value below 2^24 is exact in
fp32 sums whatever their order."""
import math

import pytest
import torch

import paper_1910_11971_gb300 as cci
from paper_1910_11971_gb300 import workloads as wl

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def whole(shape, lo, hi, seed, dtype, dev):
    return wl.integer_valued(shape, lo, hi, seed).to(DTYPES[dtype]).to(dev)


def rounded(t, dtype):
    return t.float().to(DTYPES[dtype]).double()


def check_block(dev, N, D, F, dtype, act="relu"):
    x, wg, wu = (whole(s, -1, 1, k, dtype, dev) for k, s in enumerate(((N, D), (F, D), (F, D))))
    dh = whole((N, F), -1, 1, 9, dtype, dev)
    st = cci.new_status(dev)
    h, g, u = cci.gated_linear(x, wg, wu, act=act, save=True, status=st)
    gr, ur = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    assert torch.equal(g.double(), gr) and torch.equal(u.double(), ur)
    assert torch.equal(h.double(), rounded(gr.clamp(min=0) * ur, dtype))
    dg, du = dh.double() * ur * (gr > 0), dh.double() * gr.clamp(min=0)
    assert dg.abs().max() < 256 and du.abs().max() < 256  # exact as bf16
    dx, dwg, dwu = cci.gated_linear_backward(dh, x, wg, wu, g, u, act=act, status=st)
    assert cci.read_status(st) == 0
    for got, ref in ((dx, dg @ wg.double() + du @ wu.double()), (dwg, dg.t() @ x.double()), (dwu, du.t() @ x.double())):
        assert ref.abs().max() < 2 ** 24
        assert torch.equal(got.double(), rounded(ref, dtype))


# long reductions over few tiles (their stages are cut evenly over the SMs): into dX (2 F) and into dW (N), a last
# round nearly empty and nearly full, shares that meet one tile and two, every tile shape
@pytest.mark.parametrize("dtype,N,D,F", [
    ("bf16", 300, 512, 8192), ("bf16", 40, 1000, 8192), ("bf16", 1, 256, 16384), ("bf16", 8192, 136, 264), ("bf16", 6000, 512, 72),
    ("bf16", 1300, 2048, 4096), ("bf16", 520, 4096, 8200), ("bf16", 129, 4096, 2048), ("f32", 130, 256, 4096), ("f32", 4100, 72, 264),
    ("f32", 20, 520, 8192), ("f32", 700, 1032, 2048)])
def test_cut_reductions_are_exact(dev, dtype, N, D, F):
    check_block(dev, N, D, F, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16, 17, 24])
def test_few_tokens_are_exact(dev, N, dtype):
    for D, F in ((8, 8), (264, 24), (1000, 136), (2056, 72)):
        check_block(dev, N, D, F, dtype)


def dense(values, idx, F, G):
    w = torch.zeros((F // G, values.shape[1], G), dtype=values.dtype, device=values.device)
    return w.scatter_(2, idx.long(), values).permute(0, 2, 1).reshape(F, -1).contiguous()


# every (G, K) that few tokens read packed, one that they do not, widths off the rounds of 1024, 16-byte index runs and not
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,K", [(4, 1), (4, 2), (8, 1), (8, 2), (8, 4), (16, 1), (16, 2), (16, 4), (16, 8), (32, 1), (32, 2), (32, 4),
                                 (32, 8), (16, 16), (64, 8), (256, 4)])
def test_packed_forms_are_exact(dev, G, K, dtype):
    for N, D, F in ((1, 1024, 256), (8, 2056, 256), (9, 1000, 512), (16, 4104, 256), (17, 136, 256), (130, 264, 512)):
        x = whole((N, D), -2, 2, N, dtype, dev)
        packs = []
        for k in range(2):
            w = whole((F, D), -3, 3, 10 + k, dtype, dev)
            packs.append(cci.pack(w, G, K))
        st = cci.new_status(dev)
        h = cci.gated_linear_packed(x, packs[0], packs[1], F, G, K, act="relu", status=st)
        assert cci.read_status(st) == 0
        g, u = (x.double() @ dense(*q, F, G).double().t() for q in packs)
        assert torch.equal(h.double(), rounded(g.clamp(min=0) * u, dtype))


@pytest.mark.parametrize("shift", [1, 4, 8])
def test_packed_indices_off_their_words(dev, shift):
    """Index arrays may start at any byte."""
    N, D, F, G, K = 5, 1024, 64, 8, 2
    x = whole((N, D), -2, 2, 1, "bf16", dev)
    packs = []
    for k in range(2):
        v, i = cci.pack(whole((F, D), -3, 3, 10 + k, "bf16", dev), G, K)
        flat = torch.zeros(i.numel() + 16, dtype=torch.uint8, device=dev)
        j = flat[shift:shift + i.numel()].view(i.shape)
        j.copy_(i)
        packs.append((v, j))
    g, u = (x.double() @ dense(*q, F, G).double().t() for q in packs)
    for n in (N, 40):
        y = x.repeat(8, 1)[:n].contiguous()
        h = cci.gated_linear_packed(y, packs[0], packs[1], F, G, K, act="relu")
        assert torch.equal(h[:N].double(), rounded(g.clamp(min=0) * u, "bf16"))


@pytest.mark.parametrize("K,G", [(1, 8), (2, 8), (4, 16), (8, 16)])
@pytest.mark.parametrize("N", [3, 40])
def test_every_bad_index_set_is_reported(dev, N, K, G):
    """A fault in any slot of a set, in the first and last group and index, of either matrix; few tokens and more."""
    D, F = 1024, 64
    x = whole((N, D), -1, 1, 1, "bf16", dev)
    good = [cci.pack(whole((F, D), -3, 3, k, "bf16", dev), G, K) for k in (1, 2)]
    faults = [list(range(K - 1)) + [G]]
    for s in range(K - 1):
        same, swapped = list(range(K)), list(range(K))
        same[s + 1] = same[s]
        swapped[s], swapped[s + 1] = swapped[s + 1], swapped[s]
        faults += [same, swapped]
    for which in range(2):
        for at in ((0, 0), (-1, -1), (0, 5), (-1, 700)):
            for f in faults:
                packs = [(v, i.clone()) for v, i in good]
                packs[which][1][at] = torch.tensor(f, dtype=torch.uint8, device=dev)
                st = cci.new_status(dev)
                cci.gated_linear_packed(x, packs[0], packs[1], F, G, K, status=st)
                assert cci.read_status(st) == 10, (which, at, f)


@pytest.mark.parametrize("N", [4, 200])
@pytest.mark.parametrize("act", list(cci.ACTIVATIONS))
def test_activations_over_their_range(dev, act, N):
    """act and act' at g from -30 to 30 and far out, u = 1 (a single weight of 1 each).

    Bounds: the fast exponential is within 2 + 1.173 |z| units of 2^-23 (CUDA's documented error), its argument z
    (g, or gelu_tanh's 1.6 (g + 0.045 g^3)) within 3 |z| units of 2^-24, sum and quotient within 4 more; gelu's Phi
    within 3.1e-7; what is below 2^-100 may be 0."""
    F, D = 512, 16
    near = torch.linspace(-30, 30, N * F - 8)
    far = torch.tensor([-1e4, -200.0, -88.5, -87.0, 87.0, 88.5, 200.0, 1e4])
    g = torch.cat([near, far]).view(N, F).to(dev)
    x = torch.zeros((N, D), device=dev)
    x[:, 0] = 1.0
    # one product per row: feed g through the saved tensors of the backward pass, and h through equal rows of x
    u = torch.ones_like(g)
    dh = torch.ones_like(g)
    wg = torch.zeros((F, D), device=dev)
    wg[:, 0] = 1.0
    gd = g.double().requires_grad_(True)
    a = {"silu": lambda t: t * torch.sigmoid(t), "gelu": lambda t: t * torch.special.ndtr(t),
         # 0.5 (1 + tanh(z)) = sigmoid(2 z), which does not cancel for large negative z
         "gelu_tanh": lambda t: t * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3)),
         "relu": lambda t: t.clamp(min=0), "sigmoid": torch.sigmoid}[act](gd)
    s, = torch.autograd.grad(a.sum(), gd)
    phi = 3.1e-7 if act == "gelu" else 0.0
    # dX[:, 0] = sum over f of (act'(g) u + act(g)) with Wg = Wu = that column: taken apart by zero weights
    zero = torch.zeros_like(wg)
    ds, _, _ = cci.gated_linear_backward(dh, x, wg, zero, g, u, act=act, need_dw=False)
    da, _, _ = cci.gated_linear_backward(dh, x, zero, wg, g, u, act=act, need_dw=False)
    tol_s = (2.0 ** -19 * (1 + s.abs()) + phi * (1 + g.double().abs())).sum(1)
    tol_a = (2.0 ** -19 * (a.abs() + s.abs()) + phi * g.double().abs() + 2.0 ** -100).sum(1).detach()
    assert ((ds[:, 0].double() - s.sum(1)).abs() <= tol_s).all()
    assert ((da[:, 0].double() - a.sum(1).detach()).abs() <= tol_a).all()
    # forward: g itself as the product of x = g with a weight of 1
    y = torch.zeros((F, 8), device=dev)
    y[:, 0] = g[0]
    y[:, 1] = 1.0
    one, up = torch.zeros((8, 8), device=dev), torch.zeros((8, 8), device=dev)
    one[:, 0], up[:, 1] = 1.0, 1.0
    h = cci.gated_linear(y, one, up, act=act)
    z = 1.6 * (g[0] + 0.045 * g[0] ** 3) if act == "gelu_tanh" else g[0]
    rel = (6 + 2.7 * z.double().abs().clamp(max=100)) * 2.0 ** -23
    ref, tol = a[0].detach()[:, None], (rel * a[0].abs() + phi * g[0].double().abs() + 2.0 ** -100).detach()[:, None]
    assert ((h.double() - ref).abs() <= tol).all()
