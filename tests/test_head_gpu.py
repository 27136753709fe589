"""Cross entropy from a head's inputs and its gradients against the formulas in 64 bits, and against differences.

Tolerances, with u = 2^-24.
  Logits: the tensor core adds blocks of 16 products to a running sum and cuts what it aligns, at most 17 cuts of 2 u of
      the magnitudes' sum A = sum |x w| a block; forward, and in fp32, no more than 704 indices at a time (44 blocks), whose sums are
      added with one rounding each.  So ez = (34 * min(44, D / 16) + D * terms / 320 + 2) u A, and for the bf16 gradient's
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
    return (34 * (min(44, blocks) if chunked else blocks) + D * terms / 320 + 2) * U * A


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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V", [(20000, 16, 10000), (5000, 8, 60001)])
def test_several_pieces(dev, N, D, V, dtype):
    """Workspaces of a few pieces of the vocabulary: P's rows of 10000 entries are 400 MB, of 60001 600."""
    X, W, targets, dloss = inputs(N, D, V, dtype, N)
    args = X.to(dev), W.to(dev), targets.to(dev)
    loss, stats = cci.linear_cross_entropy(*args)
    dX, dW = cci.linear_cross_entropy_backward(dloss.to(dev), *args, stats)
    some = torch.arange(0, N, 97)  # rows of dX and of the loss, all of dW by the formula on the GPU in 64 bits
    z = args[0].double() @ args[1].double().t()
    lse = torch.logsumexp(z, 1)
    kept = args[2] != IGNORE
    check_forward(X[some], W, targets[some], loss[some], stats[some], dtype)
    P = torch.exp(z - lse[:, None]) * torch.where(kept, dloss.to(dev).double(), 0.0)[:, None]
    P[torch.arange(N, device=dev)[kept], args[2][kept]] -= dloss.to(dev).double()[kept]
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    # A probability p is off by at most 512 u p: 36 u of sum |x w|, up to 10 here, for its logit and as much for the sum's;
    # (4 + 3.4 * 20) u for its exponential, 70 u for the sum's additions.  The target's entry p - 1 is off by p's error, whatever
    # is left of it: at p = 0.999 that is 1000 times as much of the entry itself, so the error goes with d (p + 1[v = t]), not
    # with |P|.  The rounding of P and the products' sums go with |P|, as above
    off = dloss.to(dev).double().abs()[:, None] * torch.exp(z - lse[:, None]) * kept[:, None]
    rel = half + ((34 * 32 if dtype == "f32" else 34 * (max(N, V) // 16)) + 8) * U
    for got, want, tol in ((dX, P @ args[1].double(), (512 * U * off + rel * P.abs()) @ args[1].double().abs()),
                           (dW, P.t() @ args[0].double(), (512 * U * off + rel * P.abs()).t() @ args[0].double().abs())):
        assert ((got.double() - want).abs() <= tol + half * want.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_only_what_is_asked_for(dev, dtype):
    X, W, targets, dloss = (t.to(dev) for t in inputs(200, 64, 777, dtype, 1))
    loss, stats = cci.linear_cross_entropy(X, W, targets)
    dX, dW = cci.linear_cross_entropy_backward(dloss, X, W, targets, stats)
    a, none = cci.linear_cross_entropy_backward(dloss, X, W, targets, stats, need_dw=False)
    none2, b = cci.linear_cross_entropy_backward(dloss, X, W, targets, stats, need_dx=False)
    assert none is None and none2 is None and torch.equal(a, dX) and torch.equal(b, dW)
    assert cci.linear_cross_entropy_backward(dloss, X, W, targets, stats, need_dx=False, need_dw=False) == (None, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_call_gives_the_same_bits(dev, dtype):
    X, W, targets, dloss = (t.to(dev) for t in inputs(300, 520, 3001, dtype, 2))
    ref = None
    for _ in range(3):
        loss, stats = cci.linear_cross_entropy(X, W, targets)
        got = (loss, stats, *cci.linear_cross_entropy_backward(dloss, X, W, targets, stats))
        assert ref is None or all(torch.equal(a, b) for a, b in zip(got, ref))
        ref = got


def test_all_left_out(dev):
    X, W, _, dloss = (t.to(dev) for t in inputs(40, 64, 300, "bf16", 3))
    targets = torch.full((40,), IGNORE, device=dev)
    loss, stats = cci.linear_cross_entropy(X, W, targets)
    assert (loss == 0).all() and stats.isfinite().all()
    dX, dW = cci.linear_cross_entropy_backward(dloss * float("nan"), X, W, targets, stats)
    assert (dX == 0).all() and (dW == 0).all()
    # another value to leave out by, a valid entry's too
    loss, _ = cci.linear_cross_entropy(X, W, torch.full((40,), 7, device=dev), ignore_index=7)
    assert (loss == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [5, 20, 40, 300])
def test_left_out_rows_may_hold_anything(dev, N, dtype):
    """Pad rows of NaN and inf: to be ignored, with a bad target, without a gradient."""
    X, W, targets, dloss = inputs(N, 72, 700, dtype, 11)
    out = torch.arange(N) % 5 < 3
    targets[0::5], targets[1::5], dloss[2::5] = IGNORE, 700, 0.0
    clean = torch.where(out[:, None], 0.0, X.float()).to(X.dtype)
    dirty = torch.where(out[:, None], torch.tensor([float("nan"), float("inf"), -float("inf")]).repeat(24), X.float()).to(X.dtype)
    got = []
    for x in (clean, dirty):
        args = x.to(dev), W.to(dev), targets.to(dev)
        loss, stats = cci.linear_cross_entropy(*args)
        got.append((loss[~out.to(dev)], *cci.linear_cross_entropy_backward(dloss.to(dev), *args, stats)))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][2].isfinite().all()
    assert (got[1][1].cpu()[out] == 0).all()


def test_no_rows(dev):
    W = torch.ones((30, 16), device=dev)
    X, t = torch.empty((0, 16), device=dev), torch.empty(0, dtype=torch.int64, device=dev)
    loss, stats = cci.linear_cross_entropy(X, W, t)
    dX, dW = cci.linear_cross_entropy_backward(loss, X, W, t, stats)
    assert loss.shape == (0,) and stats.shape == (0, 2) and dX.shape == (0, 16) and (dW == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bad_targets_are_reported(dev, dtype):
    X, W, targets, dloss = inputs(300, 64, 500, dtype, 4)
    bad = torch.zeros(300, dtype=torch.bool)
    for n, t in ((0, 500), (7, -1), (131, 2 ** 40), (299, -(2 ** 63))):
        targets[n], bad[n] = t, True
    args = X.to(dev), W.to(dev), targets.to(dev)
    status = cci.new_status(dev)
    loss, stats = cci.linear_cross_entropy(*args, status=status)
    assert cci.read_status(status) == 10  # CCI_ERR_INDEX
    assert (loss.cpu().isnan() == bad).all()
    status = cci.new_status(dev)
    dX, dW = cci.linear_cross_entropy_backward(dloss.to(dev), *args, stats, status=status)
    assert cci.read_status(status) == 10
    # as if they were left out
    targets[bad] = IGNORE
    check_backward(X, W, targets, stats, dloss, dX, dW, dtype)
    assert (dX.cpu()[bad] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_and_inf_keep_to_their_rows(dev, dtype):
    X, W, targets, _ = inputs(300, 64, 500, dtype, 5)
    good = cci.linear_cross_entropy(X.to(dev), W.to(dev), targets.to(dev))[0].cpu()
    X[3, 5], X[200, 63] = float("nan"), float("inf")
    loss = cci.linear_cross_entropy(X.to(dev), W.to(dev), targets.to(dev))[0].cpu()
    bad = torch.zeros(300, dtype=torch.bool)
    bad[3] = bad[200] = True
    assert loss[bad].isnan().all() and torch.equal(loss[~bad], good[~bad])


def test_confident_tokens_keep_their_loss(dev):
    """Logits of 30 over thousands of indices whose sum grows all along: the loss is a difference of such sums."""
    D, V = 4096, 300
    g = torch.Generator().manual_seed(6)
    W = torch.randn((V, D), generator=g).to(torch.bfloat16)
    targets = torch.arange(0, V, 3)
    X = ((30.0 / D) * W[targets].float() + 0.1 / D ** 0.5 * torch.randn((100, D), generator=g)).to(torch.bfloat16)
    loss, stats = cci.linear_cross_entropy(X.to(dev), W.to(dev), targets.to(dev))
    check_forward(X, W, targets, loss, stats, "bf16")
    _, _, _, _, want = reference(X, W, targets)
    # eight chunks of 512 indices, a logit of 3.75 each at most, 32 cuts of half a unit (2^-23 of up to 4) in the mean while
    # the sum grows: 8 * 32 * 2^-23 / 2 * 4 / 2 = 3.1e-5 of the logit's difference, and as much of each token's chance to miss
    assert ((loss.cpu().double() - want).abs() <= 6.2e-5 * (1 - torch.exp(-want)) + 1e-6 * want + 2 ** -24).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 30, 100])
def test_sure_tokens_keep_their_gradient(dev, N, dtype):
    """Chances of 1 - 3e-4 or so: what is left of p - 1 is as right as that of the others.  A difference of logits is off by 2 ez of
    the chunks, which goes with p (1 - p); log s and the difference from it round to 8 u, whatever is left; the exponentials' and
    the sum's errors and the rounding of P as above."""
    D, V = 4096, 300
    g = torch.Generator().manual_seed(6)
    W = torch.randn((V, D), generator=g).to(DTYPES[dtype])
    targets = torch.randperm(V, generator=g)[:N]
    X = ((14.0 / D) * W[targets].float() + 0.1 / D ** 0.5 * torch.randn((N, D), generator=g)).to(DTYPES[dtype])
    dloss = torch.randn(N, generator=g)
    args = X.to(dev), W.to(dev), targets.to(dev)
    loss, stats = cci.linear_cross_entropy(*args)
    dX, dW = cci.linear_cross_entropy_backward(dloss.to(dev), *args, stats)
    z = X.double() @ W.double().t()
    m = z.max(1, keepdim=True).values
    p = torch.softmax(z, 1)
    assert 2e-5 < float((1 - p.max(1).values).min()) and float((1 - p.max(1).values).max()) < 1e-3
    P = p.scatter(1, targets[:, None], 0.0)
    P.scatter_(1, targets[:, None], -P.sum(1, keepdim=True))  # not by p - 1
    P = dloss.double()[:, None] * P
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    ez = logit_error(X, W, dtype, True).max(1, keepdim=True).values
    eP = P.abs() * (half + 2 * ez + (60 + V / 500 + 3.4 * (m - z)) * U) + 8 * U * dloss.double().abs()[:, None] * torch.maximum(p, p > 0.5)
    for got, want, mags in ((dX, P @ W.double(), W.double().abs()), (dW, P.t() @ X.double(), X.double().abs())):
        a, e = (P.abs(), eP) if got is dX else (P.abs().t(), eP.t())
        assert ((got.cpu().double() - want).abs() <= (e + 34 * 32 * U * a) @ mags + (half + 2 * U) * want.abs()).all()


def test_large_offsets(dev):
    """Logits that all lie far from 0."""
    N, D, V = 50, 64, 400
    X, W, targets, dloss = inputs(N, D, V, "f32", 7)
    X[:, 0], W[:, 0] = 100.0, 50.0
    args = X.to(dev), W.to(dev), targets.to(dev)
    loss, stats = cci.linear_cross_entropy(*args)
    check_forward(X, W, targets, loss, stats, "f32")
    dX, dW = cci.linear_cross_entropy_backward(dloss.to(dev), *args, stats)
    check_backward(X, W, targets, stats, dloss, dX, dW, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [10, 12, 16, 50])
@pytest.mark.parametrize("N", [5, 40, 200])
def test_logits_of_any_size(dev, N, scale, dtype):
    """Two values of logits, 2^20 to 2^100 and further apart than any exponent: p is 1 / c at the larger, c of them.  Sums as above:
    100 units of u for s (V / 500 and what its exponentials, all 1, leave), P's rounding, and the products' cuts."""
    D, V = 64, 301
    g = torch.Generator().manual_seed(N)
    X, W = torch.zeros((N, D)), torch.zeros((V, D))
    X[:, 3] = 1.5859375 * 2.0 ** scale * torch.where(torch.arange(N) % 2 > 0, -1.0, 1.0)
    W[:, 3] = 1.5703125 * 2.0 ** scale * torch.where(torch.rand(V, generator=g) < 0.4, 0.5, 1.0)
    z = X.double() @ W.double().t()
    top = z == z.max(1, keepdim=True).values
    c = top.sum(1).double()
    targets = torch.multinomial(top.double(), 1, generator=g)[:, 0]
    dloss = torch.randn(N, generator=g) / N
    args = X.to(DTYPES[dtype]).to(dev), W.to(DTYPES[dtype]).to(dev), targets.to(dev)
    loss, stats = cci.linear_cross_entropy(*args)
    assert ((loss.cpu().double() - torch.log(c)).abs() <= 100 * U * (1 + torch.log(c))).all()
    d = dloss.double()[:, None]
    p = top / c[:, None]
    P = d * p
    P[torch.arange(N), targets] -= dloss.double()
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    eP = 200 * U * d.abs() * p + (half + 4 * U) * P.abs()
    sums = 34 * 32 * U
    dX, dW = cci.linear_cross_entropy_backward(dloss.to(dev), *args, stats)
    for got, want, tol in ((dX, P @ W.double(), (eP + sums * P.abs()) @ W.double().abs()),
                           (dW, P.t() @ X.double(), (eP + sums * P.abs()).t() @ X.double().abs())):
        assert ((got.cpu().double() - want).abs() <= tol + (half + 2 * U) * want.abs()).all()


def test_gradient_against_differences(dev):
    N, D, V = 3, 16, 20
    X, W, targets, dloss = inputs(N, D, V, "f32", 8)
    args = X.to(dev), W.to(dev), targets.to(dev)
    loss, stats = cci.linear_cross_entropy(*args)
    dX, dW = (t.cpu() for t in cci.linear_cross_entropy_backward(dloss.to(dev), *args, stats))
    step = 1e-4
    for which, grad in ((0, dX), (1, dW)):
        for a, b in ((0, 3), (2, 15), (int(targets[0]) if which else 1, 7)):
            ends = []
            for sign in (1, -1):
                t = [X.double(), W.double()]
                t[which][a, b] += sign * step
                ends.append(float((reference(t[0], t[1], targets)[4] * dloss.double()).sum()))
            # third derivatives are below 10: |x|^3 and |w|^3 of a few
            assert abs((ends[0] - ends[1]) / (2 * step) - float(grad[a, b])) <= 1e-6


@pytest.mark.parametrize("call", [cci.HEAD_FORWARD, cci.HEAD_BACKWARD])
def test_a_given_workspace_is_enough(dev, call):
    N, D, V = 300, 64, 3001
    X, W, targets, dloss = (t.to(dev) for t in inputs(N, D, V, "f32", 9))
    ws = cci.head_workspace(call, torch.float32, N, D, V, dev)
    room = torch.full((ws.numel() + 512,), 7, dtype=torch.uint8, device=dev)
    at = room[256:256 + ws.numel()]
    loss, stats = cci.linear_cross_entropy(X, W, targets)
    if call == cci.HEAD_FORWARD:
        got = cci.linear_cross_entropy(X, W, targets, workspace=at)
        assert torch.equal(got[0], loss) and torch.equal(got[1], stats)
    else:
        want = cci.linear_cross_entropy_backward(dloss, X, W, targets, stats)
        got = cci.linear_cross_entropy_backward(dloss, X, W, targets, stats, workspace=at)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert (room[:256] == 7).all() and (room[256 + ws.numel():] == 7).all()
    with pytest.raises(cci.CCIError):
        cci.linear_cross_entropy(X, W, targets, workspace=at[:-256]) if call == cci.HEAD_FORWARD else \
            cci.linear_cross_entropy_backward(dloss, X, W, targets, stats, workspace=at[:-256])
