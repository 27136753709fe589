"""The end of a language model as it is trained and served: residual addition and norm, head, cross entropy, distillation
against a teacher and all gradients, in one run; captured into graphs, on streams of their own, over rows whose offsets pass
32 bits."""
import pytest
import torch

import paper_1910_11971_gb300 as cci

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def model(dev, dtype, seed=0, N=200, D=256, V=3001):
    g = torch.Generator(device=dev).manual_seed(seed)
    def rnd(*shape, std=1.0):
        return torch.randn(shape, generator=g, device=dev) * std
    t = DTYPES[dtype]
    return dict(x=rnd(N, D, std=0.3).to(t), stream=rnd(N, D).to(t), w=1.0 + 0.1 * rnd(D), head=rnd(V, D, std=2 / D ** 0.5).to(t),
                targets=torch.randint(0, V, (N,), generator=g, device=dev), teacher=rnd(N, V, std=2.0).to(t))


def step(m, k=20):
    """A training step's end: loss, distillation and the gradients of the residual stream, the norm's weight and the head."""
    N = m["x"].shape[0]
    y, h, rstd = cci.rms_norm(m["x"], m["w"], residual=m["stream"])
    loss, stats = cci.linear_cross_entropy(y, m["head"], m["targets"])
    logits = (y @ m["head"].t()).contiguous()
    _, _, _, top_logp, top_idx = cci.token_logprobs(m["teacher"], m["targets"], top=k)
    kd, kd_stats = cci.distillation_loss(logits, top_idx, top_logp, tail=True)
    each = torch.full((N,), 1.0 / N, device=y.device)
    dlogits = cci.distillation_loss_backward(each, logits, top_idx, top_logp, kd_stats, tail=True)
    dy, dhead = cci.linear_cross_entropy_backward(each, y, m["head"], m["targets"], stats)
    dh = (dlogits @ m["head"]).contiguous()  # here: the distillation's gradient enters where the stream goes on
    dx, dw = cci.rms_norm_backward(dy, h, rstd, m["w"], dh=dh)
    return loss, kd, dx, dw, dhead, y, h


def step64(m, k=20):
    """The same in 64 bits by differentiating the formulas."""
    x, stream, w, head = (m[n].double().detach() for n in ("x", "stream", "w", "head"))
    h = (x + stream).requires_grad_(True)
    w, head = w.requires_grad_(True), head.requires_grad_(True)
    N = h.shape[0]
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-5) * w
    logits = y @ head.t()
    loss = torch.logsumexp(logits, 1) - logits.gather(1, m["targets"][:, None])[:, 0]
    logp = torch.log_softmax(logits.detach(), 1)
    value, idx = torch.sort(torch.log_softmax(m["teacher"].double(), 1), dim=1, descending=True, stable=True)
    q, idx = value[:, :k].exp(), idx[:, :k]
    rest = torch.log1p(-logp.gather(1, idx).exp().sum(1))
    left = 1 - q.sum(1)
    kd = -(q * logp.gather(1, idx)).sum(1) - left * rest
    p = logp.exp()
    r = p / rest.exp()[:, None]
    r.scatter_(1, idx, 0.0)
    target = left[:, None] * r
    target.scatter_add_(1, idx, q)
    dlogits = (p - target) / N
    dx, dw, dhead = torch.autograd.grad(loss.mean(), (h, w, head))
    return loss.detach(), kd, dx + dlogits @ head.detach(), dw, dhead, y.detach(), h.detach()


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-5), ("bf16", 3e-2)])
def test_a_training_steps_end(dev, dtype, tol):
    """Relative to each result's norm.  bf16: y, logits and dlogits are rounded, 2^-9 of each value in the mean and of what
    they go into, where logits of a spread of 2 to 8 move probabilities by up to 8 * 2^-9 = 1.6e-2, twice."""
    m = model(dev, dtype)
    for got, want in zip(step(m), step64(m)):
        assert got.shape == want.shape
        assert float((got.double() - want).norm() / want.norm()) <= tol


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(dev, dtype):
    """New values in the same buffers: nothing is kept from the call that was captured."""
    m, other = model(dev, dtype, 1), model(dev, dtype, 2)
    want, want_other = [t.clone() for t in step(m)], [t.clone() for t in step(other)]
    stream = torch.cuda.Stream(dev)
    with torch.cuda.stream(stream):
        step(m)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = step(m)
    for values, ref in ((m, want), (other, want_other), (None, want_other)):
        if values is not None and values is not m:
            for name in m:
                m[name].copy_(values[name])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_graphs_share_a_workspace(dev, dtype):
    """One after the other on one stream, as a server's graphs of two batch sizes do."""
    ms = [model(dev, dtype, 3, N=130), model(dev, dtype, 4, N=37)]
    size = max(cci.head_workspace(cci.HEAD_BACKWARD, DTYPES[dtype], m["x"].shape[0], 256, 3001, dev).numel() for m in ms)
    size = max(size, *(cci.head_workspace(cci.HEAD_FORWARD, DTYPES[dtype], m["x"].shape[0], 256, 3001, dev).numel() for m in ms))
    ws = torch.empty(size, dtype=torch.uint8, device=dev)

    def run(m):
        loss, stats = cci.linear_cross_entropy(m["x"], m["head"], m["targets"], workspace=ws)
        return (loss, *cci.linear_cross_entropy_backward(loss, m["x"], m["head"], m["targets"], stats, workspace=ws))

    want = [[t.clone() for t in run(m)] for m in ms]
    torch.cuda.synchronize()
    graphs, got = [], []
    for m in ms:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(run(m))
        graphs.append(graph)
    for i in (0, 1, 0, 0, 1):
        graphs[i].replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_two_streams_at_once(dev):
    ms = [model(dev, "bf16", 5), model(dev, "bf16", 6)]
    want = [[t.clone() for t in step(m)] for m in ms]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(dev) for _ in ms]
    got = [[], []]
    for _ in range(5):
        for i, (m, s) in enumerate(zip(ms, streams)):
            with torch.cuda.stream(s):
                got[i].append(step(m))
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(run, want[i]))


def test_rows_past_32_bits(dev):
    """More than 2^31 elements a matrix: the last rows come out as they do by themselves."""
    N, D = 600000, 4096
    x = torch.empty((N, D), dtype=torch.bfloat16, device=dev).normal_(0, 1)
    assert x.numel() > 2 ** 31
    few = x[-5:].clone()
    y, h, rstd = cci.rms_norm(x, residual=x)
    y1, h1, rstd1 = cci.rms_norm(few, residual=few)
    assert torch.equal(y[-5:], y1) and torch.equal(h[-5:], h1) and torch.equal(rstd[-5:], rstd1)
    dx, _ = cci.rms_norm_backward(y, h, rstd, dh=x)
    dx1, _ = cci.rms_norm_backward(y1, h1, rstd1, dh=few)
    assert torch.equal(dx[-5:], dx1)
    q, scales, _, _ = cci.rms_norm_fp8(x, group=128)
    q1, scales1, _, _ = cci.rms_norm_fp8(few, group=128)
    assert torch.equal(q[-5:].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(scales[-5:], scales1)


def test_logits_past_32_bits(dev):
    N, V, k = 20000, 131072, 9
    x = torch.empty((N, V), dtype=torch.bfloat16, device=dev).normal_(0, 2)
    assert x.numel() > 2 ** 31
    idx = (torch.arange(N * k, device=dev).view(N, k) * 13 % V).to(torch.int32)
    value = torch.full((N, k), -3.0, device=dev)
    few = [t[-4:].clone() for t in (x, idx, value)]
    loss, stats = cci.distillation_loss(x, idx, value, tail=True)
    loss1, stats1 = cci.distillation_loss(*few, tail=True)
    # a few rows are cut into parts, whose sums are added in another order: 60 roundings
    assert ((loss[-4:] - loss1).abs() <= 60 * 2.0 ** -24 * loss1.abs().clamp(min=12.0)).all()
    each = torch.ones(N, device=dev)
    dx = cci.distillation_loss_backward(each, x, idx, value, stats, tail=True)
    dx1 = cci.distillation_loss_backward(each[-4:], *few, stats[-4:].contiguous(), tail=True)
    assert torch.equal(dx[-4:], dx1)


def test_a_head_past_32_bits(dev):
    """2.4 G weights: the last entries' gradients are those of their targets' rows."""
    V, D, N = 300000, 8192, 3
    W = torch.empty((V, D), dtype=torch.bfloat16, device=dev).normal_(0, 0.01)
    assert W.numel() > 2 ** 31
    X = torch.empty((N, D), dtype=torch.bfloat16, device=dev).normal_(0, 1)
    targets = torch.tensor([V - 1, 5, V - 2], device=dev)
    loss, stats = cci.linear_cross_entropy(X, W, targets)
    z = torch.cat([X.float() @ w.float().t() for w in W.split(50000)], 1).double()
    lse = torch.logsumexp(z, 1)
    want = lse - z.gather(1, targets[:, None])[:, 0]
    # logits of spread 0.9, 8192 products each: below 1e-4 of 13 in fp32 here and there
    assert ((loss.double() - want).abs() <= 1e-4).all()
    d = torch.tensor([1.0, -2.0, 0.5], device=dev)
    dX, dW = cci.linear_cross_entropy_backward(d, X, W, targets, stats)
    at = [0, 5, 4097, V - 3, V - 2, V - 1]
    P = d.double()[:, None] * torch.exp(z[:, at] - lse[:, None])
    for n in range(N):
        if int(targets[n]) in at:
            P[n, at.index(int(targets[n]))] -= d[n].double()
    ref = P.t() @ X.double()
    # P and dW rounded to bf16, 2^-8 each, and P's softmax within 1e-3 of itself
    assert ((dW[at].double() - ref).abs() <= (2.0 ** -7 + 1e-3) * (P.abs().t() @ X.double().abs())).all()
