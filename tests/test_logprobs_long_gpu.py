"""Rows past 262144 logits, whose runs are ranked against each other in shared memory, up to the longest accepted:
alternatives against a stable sort, ties and masks among them, with rows that clusters share and rows that one block
takes.  Log probabilities with the tolerances of the shorter rows."""
import math

import pytest
import torch

import paper_1910_11971_gb300 as cci

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def check(x, t, top):
    N, V = x.shape
    logp, h, stats, top_logp, top_idx = cci.token_logprobs(x, t, top=top)
    for n in range(N):  # row by row: 64 bits of a long row take room
        y = x[n].double()
        order = torch.sort(y, descending=True, stable=True).indices[:top]
        assert torch.equal(top_idx[n].long(), order), n
        m = float(y.max())
        assert float(stats[n, 0]) == m
        y = y - (0.0 if m == -INF else m)
        s = float(torch.exp(y).sum())
        log_s = math.log(s) if s else 0.0
        lp = y - log_s
        p = torch.exp(lp)
        ref = float(-torch.where(p > 0, p * lp, 0.0).sum())
        E = (V / 512 + 64) * U + 4 * U * ref
        assert abs(float(stats[n, 1]) - log_s) <= E + 2 * U * log_s
        assert abs(float(h[n]) - ref) <= E * (2 + math.log(V))
        for got, want in ((logp[n:n + 1].double(), lp[t[n]][None]), (top_logp[n].double(), lp[order])):
            fine = torch.isfinite(want)
            assert torch.equal(got[~fine], want[~fine])
            assert ((got[fine] - want[fine]).abs() <= E + 4 * U * want[fine].abs()).all()


def shapes_of_values(V, dtype, dev):
    """Random, all equal, rising, falling, few distinct values, masked but for a few, all masked."""
    g = torch.Generator(device=dev).manual_seed(V)
    x = torch.randn((7, V), generator=g, device=dev) * 2.0
    x[1] = 1.5
    x[2] = x[2].sort().values
    x[3] = x[3].sort(descending=True).values
    x[4] = torch.randint(-2, 3, (V,), generator=g, device=dev).float()
    keep = torch.rand(V, generator=g, device=dev) < 7.0 / V
    x[5].masked_fill_(~keep, -INF)
    x[6] = -INF
    t = torch.randint(0, V, (7,), generator=g, device=dev)
    return x.to(DTYPES[dtype]), t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [262145, 300001, (1 << 20) + 3, (1 << 22) + 5, 1 << 24])
def test_few_rows(dev, V, dtype):
    x, t = shapes_of_values(V, dtype, dev)
    for top in (1, 20, 32):
        check(x, t, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(310, 300001), (305, 262152)])
def test_rows_that_one_block_takes(dev, N, V, dtype):
    x, t = shapes_of_values(V, dtype, dev)
    many = x.repeat(-(-N // 7), 1)[:N].contiguous()
    tokens = t.repeat(-(-N // 7))[:N].contiguous()
    got = cci.token_logprobs(many, tokens, top=20)
    check(many[:7], tokens[:7], 20)  # few rows: clusters
    order = torch.stack([torch.sort(r.double(), descending=True, stable=True).indices[:20] for r in x])
    assert torch.equal(got[4].long(), order.repeat(-(-N // 7), 1)[:N])
    few = cci.token_logprobs(x, t, top=20)
    E = (V / 512 + 64) * U * 2 + 8 * U * math.log(V)
    for a, b in zip(got[:4], few[:4]):
        b = b.repeat((-(-N // 7),) + (1,) * (b.dim() - 1))[:N]
        fine = torch.isfinite(b)
        assert torch.equal(a[~fine], b[~fine])
        assert ((a[fine] - b[fine]).abs() <= E * (2 + math.log(V)) + 8 * U * b[fine].abs()).all()


def test_one_block_and_the_most_runs(dev):
    """Rows of 2^20 + 3 logits that one block takes: a few hundred of them, bf16."""
    N, V = 305, (1 << 20) + 3
    x, t = shapes_of_values(V, "bf16", dev)
    many = x.repeat(-(-N // 7), 1)[:N].contiguous()
    idx = cci.token_logprobs(many, t.repeat(-(-N // 7))[:N].contiguous(), top=32)[4]
    order = torch.stack([torch.sort(r.double(), descending=True, stable=True).indices[:32] for r in x])
    assert torch.equal(idx.long(), order.repeat(-(-N // 7), 1)[:N])
