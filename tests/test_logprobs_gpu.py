"""Log probabilities of tokens, entropy, top alternatives and their gradient against 64 bits.

Tolerances, u = 2^-24.  A row's sum of exponentials is added one by one in each thread (V / 512 terms at least,
at most 64 in the short forms) and then in trees: with the exponential's own error (2 u and, from its argument,
2 u |y|) the logarithm of the sum is off by at most E = (V / 512 + 64) u + 4 u H, H the entropy.
  logp     E + 4 u |logp|
  entropy  E (2 + log V)
  dlogits  p (|dlogp| + |dentropy| (|log p| + H)) 8 u (4 + |log p|) + 4 u |dlogits|, and 2^-8 of a bf16 result
Whole numbers are equal.
"""
import math

import pytest
import torch

import paper_1910_11971_gb300 as cci

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")
IGNORE = -100


def logits_of(N, V, dtype, seed, spread=2.0, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((N, V), generator=g) * spread
    if masked:
        x.masked_fill_(torch.rand((N, V), generator=g) < masked, -INF)
    t = torch.randint(0, V, (N,), generator=g)
    return x.to(DTYPES[dtype]), t


def forward64(x, t, top):
    """(logp, entropy, m, log_s, top_logp, top_idx), all from the definitions."""
    x = x.double()
    m = x.max(1, keepdim=True).values
    ref = torch.where(m == -INF, 0.0, m)
    y = x - ref
    e = torch.exp(y)
    s = e.sum(1, keepdim=True)
    log_s = torch.where(s == 0, 0.0, torch.log(s))
    lp = y - log_s
    p = torch.exp(lp)
    h = -torch.where(p > 0, p * lp, 0.0).sum(1)
    order = torch.argsort(-x, dim=1, stable=True)[:, :top]
    kept = t != IGNORE
    logp = torch.where(kept, lp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    return logp, h, m[:, 0], log_s[:, 0], lp.gather(1, order), order, lp, p


def near(a, r, tol):
    a = a.cpu().double()
    fine = torch.isfinite(r)
    assert torch.equal(a[~fine], r[~fine])
    assert ((a[fine] - r[fine]).abs() <= tol[fine]).all(), float((a[fine] - r[fine]).abs().max())


def check(x, t, top, got, V=None):
    V = V or x.shape[1]
    logp, h, stats, top_logp, top_idx = got
    rl, rh, rm, rs, rt, ri, _, _ = forward64(x, t, top)
    E = (V / 512 + 64) * U + 4 * U * rh
    near(logp, rl, E + 4 * U * rl.abs())
    near(h, rh, E * (2 + math.log(V)))
    assert torch.equal(stats[:, 0].cpu().double(), rm)
    near(stats[:, 1], rs, E + 2 * U * rs)
    if top:
        assert torch.equal(top_idx.cpu().long(), ri)
        near(top_logp, rt, E[:, None] + 4 * U * rt.abs())
    else:
        assert top_logp is None and top_idx is None


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


# both sides of every form: a warp a row (128, 512, 1024), 128 threads (8192), a block, clusters
SIZES = [1, 2, 3, 31, 32, 33, 127, 128, 129, 500, 512, 513, 1000, 1024, 1025, 1031, 2048, 4099, 8191, 8192, 8193, 16383,
         16384, 20001, 50001, 65536, 131072]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_forward(dev, V, dtype):
    N = 11 if V <= 8192 else 3
    for top in sorted({0, 1, min(V, 5), min(V, 20), min(V, 32)}):
        x, t = logits_of(N, V, dtype, V + top)
        check(x, t, top, cci.token_logprobs(x.to(dev), t.to(dev), top=top))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(1, 131072), (40, 65536), (90, 33000), (310, 17000), (1000, 1500), (2100, 77), (700, 8200)])
def test_forward_rows(dev, N, V, dtype):
    x, t = logits_of(N, V, dtype, N, masked=0.3)
    t[::7] = IGNORE
    check(x, t, 10, cci.token_logprobs(x.to(dev), t.to(dev), top=10))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 700, 5000, 30000, 100003])
def test_masks_ties_and_orders(dev, V, dtype):
    """Rows that are all masked, masked but for one logit, masked by the type's lowest value, all equal, of few
    distinct values, sorted both ways, far from zero: each with 20 alternatives."""
    dt = DTYPES[dtype]
    lowest = torch.finfo(dt).min
    g = torch.Generator().manual_seed(V)
    x = torch.randn((13, V), generator=g).to(dt)
    x[0] = -INF
    x[1] = -INF
    x[1, V // 2] = 3.0
    x[2, : V // 2] = lowest
    x[3] = lowest
    x[4] = 1.5
    x[5] = torch.randint(-2, 3, (V,), generator=g).to(dt)
    x[6] = torch.sort(x[6].float()).values.to(dt)
    x[7] = torch.sort(x[7].float(), descending=True).values.to(dt)
    x[8] += 1000.0
    x[9] -= 1000.0
    x[10, 1:] = -INF
    x[11, :-1] = -INF
    x[12] = torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0).to(dt)
    t = torch.randint(0, V, (13,), generator=g)
    check(x, t, 20, cci.token_logprobs(x.to(dev), t.to(dev), top=20))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 3000, 40000])
def test_infinite_and_nan_logits_stay_in_their_row(dev, V, dtype):
    x, t = logits_of(6, V, dtype, V)
    x[1, 3], x[3, V - 1], x[4] = INF, float("nan"), float("nan")
    logp, h, _, top_logp, top_idx = cci.token_logprobs(x.to(dev), t.to(dev), top=4)
    assert logp[[1, 3, 4]].isnan().all() and h[[1, 3, 4]].isnan().all()
    assert (top_idx[4] == -1).all() and top_logp[4].isnan().all()
    order = torch.argsort(torch.where(x.isnan(), -INF, x.double()), dim=1, descending=True, stable=True)[:, :4]
    assert torch.equal(top_idx[[1, 3]].cpu().long(), order[[1, 3]])
    keep = [0, 2, 5]
    check(x[keep], t[keep], 4, [a[keep] for a in (logp, h, _, top_logp, top_idx)])


@pytest.mark.gpu
@pytest.mark.parametrize("V", [100, 3000, 40000])
def test_tokens_outside_are_reported(dev, V):
    x, t = logits_of(5, V, "f32", 1)
    st = cci.new_status(dev)
    t[2] = -7
    got = cci.token_logprobs(x.to(dev), t.to(dev), ignore_index=-7, status=st)
    assert cci.read_status(st) == 0 and got[0][2] == 0
    for bad in (V, -1, 1 << 40):
        t[3] = bad
        st = cci.new_status(dev)
        logp, h, stats, _, _ = cci.token_logprobs(x.to(dev), t.to(dev), ignore_index=-7, status=st)
        assert cci.read_status(st) == 10 and logp[3].isnan() and logp[[0, 1, 2, 4]].isfinite().all()
        st = cci.new_status(dev)
        d = cci.token_logprobs_backward(x.to(dev), t.to(dev), stats, dlogp=torch.ones(5, device=dev), ignore_index=-7, status=st)
        assert cci.read_status(st) == 10 and (d[[2, 3]] == 0).all()


def backward64(x, t, g, ge):
    _, h, _, _, _, _, lp, p = forward64(x, t, 0)
    empty = (x == -INF).all(1)
    g = torch.where(t == IGNORE, 0.0, g.double())[:, None]
    ge = ge.double()[:, None]
    d = -g * p - ge * torch.where(p > 0, p * (lp + h[:, None]), 0.0)
    d.scatter_add_(1, t.clamp(min=0)[:, None], g)
    d[empty] = 0.0
    size = p * (g.abs() + ge.abs() * (torch.where(p > 0, lp.abs(), 0.0) + h[:, None]))
    return d, size * 8 * U * (4 + torch.where(p > 0, lp.abs(), 0.0))


def check_backward(d, x, t, g, ge, dtype):
    r, tol = backward64(x, t, g, ge)
    tol = tol + 4 * U * r.abs() + (2.0 ** -8 * r.abs() if dtype == "bf16" else 0.0) + 1e-36
    assert ((d.cpu().double() - r).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(1, 1), (5, 2), (7, 31), (300, 40), (9, 1000), (5, 8191), (5, 8192), (4, 8193), (3, 50001), (2, 131072)])
def test_backward(dev, N, V, dtype):
    x, t = logits_of(N, V, dtype, N + V, masked=0.2)
    x[-1] = -INF
    if N > 2:
        t[1] = IGNORE
        x[0] = torch.randn(V, generator=torch.Generator().manual_seed(1)).to(x.dtype)
    gen = torch.Generator().manual_seed(3)
    g, ge = torch.randn(N, generator=gen), torch.randn(N, generator=gen)
    xd, td = x.to(dev), t.to(dev)
    logp, h, stats, _, _ = cci.token_logprobs(xd, td)
    zero = torch.zeros(N)
    d = cci.token_logprobs_backward(xd, td, stats, dlogp=g.to(dev), entropy=h, dentropy=ge.to(dev))
    assert d.dtype == x.dtype and d.shape == x.shape
    # the entropy and the statistics that come in carry the forward pass' errors: E of the sum's logarithm is a
    # relative error of every p, and of the entropy times p dentropy
    r, tol = backward64(x, t, g, ge)
    _, rh, _, _, _, _, lp, p = forward64(x, t, 0)
    E = ((V / 512 + 64) * U + 4 * U * rh)[:, None]
    size = p * (torch.where(t == IGNORE, 0.0, g.double()).abs()[:, None] + ge.double().abs()[:, None] *
                (torch.where(p > 0, lp.abs(), 0.0) + rh[:, None] + 4 + math.log(V)))
    tol = tol + E * size + 4 * U * r.abs() + (2.0 ** -8 * r.abs() if dtype == "bf16" else 0.0) + 1e-36
    assert ((d.cpu().double() - r).abs() <= tol).all()
    one = cci.token_logprobs_backward(xd, td, stats, dlogp=g.to(dev))
    r1, tol1 = backward64(x, t, g, zero)
    tol1 = tol1 + E * size + 4 * U * r1.abs() + (2.0 ** -8 * r1.abs() if dtype == "bf16" else 0.0) + 1e-36
    assert ((one.cpu().double() - r1).abs() <= tol1).all()
    two = cci.token_logprobs_backward(xd, None, stats, entropy=h, dentropy=ge.to(dev))
    assert two.isfinite().all()
    # in place, over the logits
    assert torch.equal(cci.token_logprobs_backward(xd, td, stats, dlogp=g.to(dev), out=xd), one)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [50, 1001, 9000])
def test_gradient_against_differences(dev, V):
    """The directional derivative of sum(a logp + b entropy) by central differences in 64 bits: step 1e-4, error
    of order h^2 and 2^-52 / h, both under 1e-6 of the terms' magnitudes."""
    N, h = 4, 1e-4
    x, t = logits_of(N, V, "f32", V)
    gen = torch.Generator().manual_seed(3)
    a, b = torch.randn(N, generator=gen), torch.randn(N, generator=gen)
    v = torch.randn((N, V), generator=gen).double()
    _, ent, stats, _, _ = cci.token_logprobs(x.to(dev), t.to(dev))
    d = cci.token_logprobs_backward(x.to(dev), t.to(dev), stats, dlogp=a.to(dev), entropy=ent, dentropy=b.to(dev))

    def loss(s):
        lp, e = forward64(x.double() + s * v, t, 0)[:2]
        return (a.double() * lp + b.double() * e).sum()

    numeric = (loss(h) - loss(-h)) / (2 * h)
    terms = d.cpu().double() * v
    assert abs(terms.sum() - numeric) <= (1e-6 + (V / 512 + 200) * U) * terms.abs().sum()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,pad,shift", [(1000, 24, 0), (5001, 7, 0), (20000, 0, 1), (33333, 3, 3), (64, 1, 1)])
def test_strides_and_alignment(dev, V, pad, shift, dtype):
    N = 4
    x, t = logits_of(N, V, dtype, V)
    flat = torch.full((shift + N * (V + pad),), float("nan"), dtype=x.dtype, device=dev)
    view = flat[shift:].view(N, V + pad)[:, :V]
    view.copy_(x)
    got = cci.token_logprobs(view, t.to(dev), top=7)
    check(x, t, 7, got)
    g = torch.ones(N)
    d = cci.token_logprobs_backward(view, t.to(dev), got[2], dlogp=g.to(dev))
    assert d.stride(0) == V + pad
    out = torch.empty((N, V), dtype=x.dtype, device=dev)  # rows at other offsets than the logits'
    assert torch.equal(cci.token_logprobs_backward(view, t.to(dev), got[2], dlogp=g.to(dev), out=out), d)
    r, tol = backward64(x, t, g, torch.zeros(N))
    tol = tol + 2 * (V / 512 + 100) * U * r.abs() + 4 * U + (2.0 ** -8 * r.abs() if dtype == "bf16" else 0.0)
    assert ((d.cpu().double() - r).abs() <= tol).all()


@pytest.mark.gpu
def test_empty_and_repeatable(dev):
    z = torch.empty((0, 64), device=dev)
    logp, h, stats, tl, ti = cci.token_logprobs(z, torch.empty(0, dtype=torch.int64, device=dev), top=3)
    assert logp.shape == (0,) and stats.shape == (0, 2) and ti.shape == (0, 3)
    assert cci.token_logprobs_backward(z, None, stats).shape == (0, 64)
    x, t = logits_of(3, 100000, "bf16", 5)
    a, b = (cci.token_logprobs(x.to(dev), t.to(dev), top=32) for _ in range(2))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.gpu
def test_row_offsets_past_32_bits(dev):
    """More than 2^32 logits in one matrix (bf16, 9 GB): the last rows are read and written where they are."""
    N, V = 33000, 131072
    x = torch.zeros((N, V), dtype=torch.bfloat16, device=dev)
    tail, t = logits_of(2, V, "bf16", 8)
    x[-2:] = tail.to(dev)
    tokens = torch.zeros(N, dtype=torch.int64, device=dev)
    tokens[-2:] = t.to(dev)
    logp, h, stats, tl, ti = cci.token_logprobs(x, tokens, top=2)
    check(tail, t, 2, [a[-2:] for a in (logp, h, stats, tl, ti)])
    assert (ti[:-2] == torch.arange(2, device=dev, dtype=torch.int32)).all()
    d = cci.token_logprobs_backward(x, tokens, stats, dlogp=torch.ones(N, device=dev), out=x)
    small = cci.token_logprobs_backward(tail.to(dev), t.to(dev), stats[-2:].contiguous(), dlogp=torch.ones(2, device=dev))
    assert torch.equal(d[-2:], small)


FAKE = 0x10000
OK, NULL, SHAPE, DTYPE, ALIGN = 0, 1, 2, 4, 5


def test_refusals():
    f, b = cci.lib().cci_token_logprobs, cci.lib().cci_token_logprobs_backward

    def fwd(x=FAKE, dt=0, N=4, V=64, ld=64, t=FAKE, top=0, lp=FAKE, h=FAKE, s=FAKE, tl=None, ti=None):
        return f(x, dt, N, V, ld, t, -100, top, lp, h, s, tl, ti, None, None)

    assert fwd(dt=9) == DTYPE
    assert fwd(x=None) == NULL and fwd(t=None) == NULL and fwd(lp=None) == NULL and fwd(h=None) == NULL and fwd(s=None) == NULL
    assert fwd(top=1) == NULL
    assert fwd(N=-1) == SHAPE and fwd(V=0) == SHAPE and fwd(ld=63) == SHAPE and fwd(top=-1) == SHAPE
    assert fwd(top=33, tl=FAKE, ti=FAKE) == SHAPE and fwd(V=2, top=3, tl=FAKE, ti=FAKE) == SHAPE
    assert fwd(V=1 << 31, ld=1 << 31) == SHAPE and fwd(N=1 << 31) == SHAPE and fwd(N=1 << 30, ld=1 << 40) == SHAPE
    assert fwd(x=FAKE + 2) == ALIGN and fwd(t=FAKE + 4) == ALIGN and fwd(lp=FAKE + 2) == ALIGN
    assert fwd(N=0, x=None, t=None, lp=None, h=None, s=None) == OK

    def bwd(x=FAKE, dt=0, N=4, V=64, ld=64, s=FAKE, t=FAKE, g=FAKE, h=FAKE, ge=FAKE, d=FAKE, ldd=64):
        return b(x, dt, N, V, ld, s, t, -100, g, h, ge, d, ldd, None, None)

    assert bwd(dt=9) == DTYPE and bwd(x=None) == NULL and bwd(s=None) == NULL and bwd(d=None) == NULL
    assert bwd(t=None) == NULL and bwd(h=None) == NULL
    assert bwd(ldd=63) == SHAPE and bwd(ld=63) == SHAPE and bwd(V=0) == SHAPE
    assert bwd(d=FAKE + 2) == ALIGN and bwd(ge=FAKE + 2) == ALIGN
    host, tok = torch.zeros((4, 8)), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError):
        cci.token_logprobs(host, tok)
    with pytest.raises(ValueError):
        cci.token_logprobs_backward(host, tok, host[:, :2])
