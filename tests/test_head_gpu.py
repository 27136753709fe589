"""Cross entropy from a head's inputs and its gradients against the formulas in 64 bits, and against differences.

Tolerances, with u = 2^-24.
  Logits: the tensor core adds blocks of 16 products to a running sum and cuts what it aligns, at most 17 cuts of 2 u of
      the magnitudes' sum A = sum |x w| a block; forward, and in fp32, no more than 512 indices at a time (32 blocks), whose sums are
      added with one rounding each.  So ez = (34 * min(32, D / 16) + D * terms / 512 + 2) u A, and for the bf16 gradient's
      logits 34 * D / 16 + 2.  fp32 operands leave out 2^-25 of A, within the 2.
  Loss: twice the logits' ez (of the target, of the others), and for log s of s = sum exp(z - m): each exponential within
      2 + 1.17 |z - m| units of 2 u and the rounding of its argument, u |z - m|; 32 additions in a thread, 4 joins in it,
      V / 4096 + 6 joins of parts, each with an exponential of at most 3 units: 50 + V / 500 units of u in all.
  P: those of the softmax, times its own value; bf16: rounded, 2^-8 of itself, and its target's entry also by the
      cancellation in p - 1, which the softmax's tolerance covers with p = 1.
  dX, dW: P's tolerance through the product; the running sum's cuts, 34 / 16 u a term of the magnitudes' sum (fp32: 34 * 32 u
      and one rounding per 512); bf16: the output's rounding, 2^-8 of it.
"""
import pytest
import torch

import paper_1910_11971_gb300 as cci

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IGNORE = -100

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def inputs(N, D, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn((V, D), generator=g) * spread / D ** 0.5).to(DTYPES[dtype])
    targets = torch.randint(0, V, (N,), generator=g)
    x = torch.randn((N, D), generator=g) + 2.0 * torch.rand((N, 1), generator=g) * W[targets].float()
    dloss = torch.randn(N, generator=g) / N
    if N > 2:
        targets[N // 2] = IGNORE
    return x.to(DTYPES[dtype]), W, targets, dloss


def reference(X, W, targets):
    z = X.double() @ W.double().t()
    m = z.max(1).values
    lse = torch.logsumexp(z, 1)
    kept = targets != IGNORE
    zt = z.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    return z, m, lse, kept, torch.where(kept, lse - zt, 0.0)


def logit_error(X, W, dtype, chunked):
    D, terms = X.shape[1], 6 if dtype == "f32" else 1
    A = X.double().abs() @ W.double().abs().t()
    blocks = (D + 15) // 16
    return (34 * (min(32, blocks) if chunked else blocks) + D * terms / 512 + 2) * U * A


def softmax_error(z, m, ez, p, V):
    """(relative error of the sum of exponentials, of each softmax entry) a row."""
    far = (m[:, None] - z)
    each = ez + (4 + 3.4 * far) * U
    of_sum = (p * each).sum(1) + (50 + V / 500) * U
    return of_sum, each


def check_forward(X, W, targets, loss, stats, dtype):
    V = W.shape[0]
    z, m, lse, kept, want = reference(X, W, targets)
    ez = logit_error(X, W, dtype, True)
    p = torch.softmax(z, 1)
    of_sum, _ = softmax_error(z, m, ez, p, V)
    at = ez.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    tol = of_sum + at + ez.max(1).values + 4 * U * (lse.abs() + m.abs() + 1)
    assert ((loss.cpu().double() - want).abs() <= tol).all()
    assert (loss.cpu()[~kept] == 0).all()
    got = stats.cpu().double()
    assert ((got[:, 0] - m).abs() <= ez.max(1).values + 2 * U * m.abs()).all()
    assert ((got.sum(1) - lse).abs() <= tol).all()


def check_backward(X, W, targets, stats, dloss, dX, dW, dtype):
    N, D = X.shape
    V = W.shape[0]
    z, m, lse, kept, _ = reference(X, W, targets)
    ez = logit_error(X, W, dtype, dtype == "f32")
    p = torch.softmax(z, 1)
    of_sum, each = softmax_error(z, m, ez, p, V)
    d = torch.where(kept, dloss.double(), 0.0)[:, None]
    hit = torch.zeros_like(p)
    hit[torch.arange(N)[kept], targets[kept]] = 1.0
    P = d * (p - hit)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    # the forward pass' stats carry its own errors, within the same bound
    eP = d.abs() * (p * (each + 2 * of_sum[:, None] + ez.max(1, keepdim=True).values + 8 * U) + 4 * U * hit) + (half + 2 * U) * P.abs()

    def sums(n):  # of n terms
        return ((34 * 32 + n * 6 / 512) if dtype == "f32" else 34 * ((n + 15) // 16) + 200) * U + 4 * U

    Xd, Wd = X.double(), W.double()
    for got, want, tol, n in ((dX, P @ Wd, eP @ Wd.abs() + sums(V) * (P.abs() @ Wd.abs()), V),
                              (dW, P.t() @ Xd, eP.t() @ Xd.abs() + sums(N) * (P.abs().t() @ Xd.abs()), N)):
        assert got.dtype == X.dtype
        diff = (got.cpu().double() - want).abs()
        assert (diff <= tol + (half + 2 * U) * want.abs() + 1e-38).all(), float((diff / (tol + half * want.abs() + 1e-38)).max())


# tokens and vocabularies at both sides of a tile's rows and columns, one of each, widths of one and several stages
SIZES = [(1, 8, 1), (1, 64, 2), (2, 72, 7), (3, 64, 64), (7, 128, 65), (16, 200, 127), (33, 256, 128), (64, 264, 129),
         (100, 64, 255), (127, 512, 256), (128, 520, 257), (129, 64, 511), (130, 1024, 513), (255, 72, 1000),
         (256, 328, 1024), (257, 64, 2049), (300, 2048, 3001), (513, 136, 5003), (1, 1024, 40000), (5, 264, 70001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", SIZES)
def test_against_64_bits(dev, N, D, V, dtype):
    X, W, targets, dloss = inputs(N, D, V, dtype, N + D + V)
    status = cci.new_status(dev)
    args = X.to(dev), W.to(dev), targets.to(dev)
    loss, stats = cci.linear_cross_entropy(*args, status=status)
    check_forward(X, W, targets, loss, stats, dtype)
    dX, dW = cci.linear_cross_entropy_backward(dloss.to(dev), *args, stats, status=status)
    check_backward(X, W, targets, stats, dloss, dX, dW, dtype)
    assert int(status.item()) == 0
