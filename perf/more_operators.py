"""What a pruned language model's last sub-layer hands its head, and what the head learns from, as cases that can be
timed and compared: the root-mean-square norm with the residual's addition, softmax cross entropy over a large
vocabulary straight from the head's inputs, and distillation from a teacher's top logits.

A case is a dict of plain values.  ``kind`` says which call it is:

  rms             ``rms_norm``: rows x, residual, weight -> y, h = x + residual, rstd
  rms_fp8         ``rms_norm_fp8``: the same with y in 8 bits (e4m3) and a scale per row or per 128 columns
  rms_backward    ``rms_norm_backward``: dy, h, rstd, weight, and the gradient that h has besides -> dx, dweight
  head            ``linear_cross_entropy``: rows X, head W, targets -> loss, (maximum, log of the sum) of the logits
  head_step       ``linear_cross_entropy`` and ``linear_cross_entropy_backward``: loss, dX, dW
  distill         ``distillation_loss``: logits, a teacher's top indices and log probabilities -> the teacher's cross
                  entropy against the softmax of the logits; per row (maximum, log of the sum, log of the sum
                  over what the teacher does not list, the teacher's sum or its normaliser's log)
  distill_backward  ``distillation_loss_backward``: its gradient to the logits

With ``own`` false, ``run`` computes them in elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IGNORE = -100  # a target of this value is left out: loss 0, no gradient
EPS = 1e-5
E4M3_MAX = 448.0


def _rms(name, kind, N, D, dtype, residual=True, group=0):
    return {"name": name, "kind": kind, "N": N, "D": D, "dtype": dtype, "residual": residual, "group": group}


def _head(name, kind, N, D, V, dtype):
    return {"name": name, "kind": kind, "N": N, "D": D, "V": V, "dtype": dtype}


def _distill(name, kind, N, V, k, dtype, T=1.0, tail=False, pad=0):
    return {"name": name, "kind": kind, "N": N, "V": V, "k": k, "dtype": dtype, "T": T, "tail": tail, "pad": pad}


def listed():
    return [
        # one token of a model 4096 wide, as in every decoding step: launch and latency are all there is
        _rms("rms_token", "rms", 1, 4096, "bf16"),
        # a training batch of 16384 tokens, its residual stream updated on the way
        _rms("rms_batch", "rms", 16384, 4096, "bf16"),
        # a prompt's rows for a product in 8 bits, a scale per 128 columns
        _rms("rms_fp8_prompt", "rms_fp8", 4000, 8192, "bf16", True, 128),
        # the gradient of the training batch, the residual stream's own added, with the sum over rows for the weight
        _rms("rms_batch_backward", "rms_backward", 16384, 4096, "bf16"),
        # rows whose width fits no vector load, an odd number of them
        _rms("rms_odd_backward", "rms_backward", 5003, 1001, "bf16"),
        # scoring one token: the head's weights are all that is read
        _head("head_token", "head", 1, 4096, 131072, "bf16"),
        # scoring a prompt of no round length over an odd vocabulary
        _head("head_score", "head", 1999, 4096, 50257, "bf16"),
        # a training pass over a large vocabulary, forward and backward
        _head("head_step", "head_step", 4096, 2048, 131072, "bf16"),
        # a training pass of a small model in fp32 over an odd vocabulary
        _head("head_step_f32", "head_step", 500, 1024, 32003, "f32"),
        # a decoding step's eight rows against their teacher, the rest of the vocabulary as one more outcome
        _distill("distill_token", "distill", 8, 131072, 32, "f32", 1.0, True),
        # a batch of a large vocabulary against its teacher's twenty best
        _distill("distill_batch", "distill", 2048, 131072, 20, "bf16", 1.0, True),
        # the gradient over an odd vocabulary, its logits in rows padded to whole vectors, at a temperature
        _distill("distill_backward", "distill_backward", 4096, 50001, 64, "bf16", 2.0, False, 7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any number of rows or tokens, widths and vocabularies odd and round, both types."""
    kind = rng.choice(("rms", "rms_fp8", "rms_backward", "head", "head", "head_step", "distill", "distill", "distill_backward"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind.startswith("rms"):
        D = _log_int(rng, 16, 16384)
        if kind == "rms_fp8" or rng.random() < 0.6:
            D = -(-D // 8) * 8
        most = 16384 * 4096 // (2 if dtype == "f32" else 1)
        return {"kind": kind, "N": _log_int(rng, 1, min(65536, max(1, most // D))), "D": D, "dtype": dtype,
                "residual": rng.random() < 0.7, "group": rng.choice((0, 128)) if kind == "rms_fp8" else 0}
    if kind.startswith("head"):
        D = 8 * max(1, _log_int(rng, 64, 4096) // 8)
        V = _log_int(rng, 2, 131072)
        if rng.random() < 0.5:
            V = -(-V // 8) * 8
        # at most the listed training pass's products in bf16, a sixteenth of them in fp32
        most = 4096 * 2048 * 131072 // (16 if dtype == "f32" else 1)
        return {"kind": kind, "N": _log_int(rng, 1, min(8192, max(1, most // (D * V)))), "D": D, "V": V, "dtype": dtype}
    V = _log_int(rng, 2, 131072)
    if rng.random() < 0.5:
        V = -(-V // 8) * 8
    most = 2048 * 131072 // (2 if dtype == "f32" else 1) // (2 if kind == "distill_backward" else 1)
    return {"kind": kind, "N": _log_int(rng, 1, min(8192, max(1, most // V))), "V": V,
            "k": min(V, rng.choice((1, 5, 20, 32, 64, 128))), "dtype": dtype, "T": rng.choice((1.0, 1.0, 2.0, 0.7)),
            "tail": rng.random() < 0.5, "pad": rng.choice((0, 0, (-V) % 8, 3))}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _normal(shape, std, dtype, seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + stream)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(DTYPES[dtype])


def _uniform(shape, seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + stream)
    return torch.rand(shape, generator=g, device="cuda")


def _rms_inputs(case, seed):
    """Rows as a residual stream has them: a spread of their own, a few channels far out, and a sub-layer's output."""
    N, D, dt = case["N"], case["D"], case["dtype"]
    stream = _normal((N, D), 1.0, "f32", seed, 1) * (0.5 + 2.0 * _uniform((N, 1), seed, 2))
    stream += 8.0 * (_uniform((1, D), seed, 3) > 0.99)
    s = {"w": 1.0 + _normal((D,), 0.2, "f32", seed, 4)}
    if case["kind"] == "rms_backward":
        s["h"] = stream.to(DTYPES[dt])
        s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
        s["dy"] = _normal((N, D), 0.05, dt, seed, 6)
        s["dh"] = _normal((N, D), 0.05, dt, seed, 7) if case["residual"] else None
    elif case["residual"]:
        s["x"], s["residual"] = _normal((N, D), 0.3, dt, seed, 5), stream.to(DTYPES[dt])
    else:
        s["x"], s["residual"] = stream.to(DTYPES[dt]), None
    return s


def _head_inputs(case, seed):
    """Normed rows and a head whose logits spread by about two; the targets' logits stand out by as much as a model
    has learned of each, from nothing to nearly all; some tokens are left out."""
    N, D, V, dt = case["N"], case["D"], case["V"], case["dtype"]
    W = _normal((V, D), 2.0 / math.sqrt(D), dt, seed, 1)
    targets = (_uniform((N,), seed, 2) * V).long().clamp_(max=V - 1)
    x = _normal((N, D), 1.0, "f32", seed, 3) + 6.0 * _uniform((N, 1), seed, 4) * 0.5 * W[targets].float()
    targets[_uniform((N,), seed, 5) < 0.05] = IGNORE
    s = {"X": x.to(DTYPES[dt]), "W": W, "targets": targets}
    if case["kind"] == "head_step":
        s["dloss"] = torch.full((N,), 1.0 / N, device="cuda") * (0.5 + _uniform((N,), seed, 6))
    return s


def _distill_inputs(case, seed):
    """A student's logits of a spread that differs from row to row, and its teacher's best: near the student's own
    largest logits, in descending order, as its log probabilities.  Some rows list fewer (index -1), one of eight rows
    and more none; some rows have a part of the vocabulary masked."""
    N, V, k, dt, T = case["N"], case["V"], case["k"], case["dtype"], case["T"]
    full = _normal((N, V + case["pad"]), 1.0, "f32", seed, 1) * (0.5 + 3.0 * _uniform((N, 1), seed, 2))
    teacher = full[:, :V] + _normal((N, V), 0.5, "f32", seed, 3)
    value, idx = torch.sort(torch.log_softmax(teacher / T if case["tail"] else teacher, 1), dim=1, descending=True, stable=True)
    value, idx = value[:, :k].contiguous(), idx[:, :k].to(torch.int32).contiguous()
    del teacher
    masked = (_uniform((N, 1), seed, 4) < 0.2) & (_uniform((N, V + case["pad"]), seed, 5) < 0.4)
    masked[:, :V].scatter_(1, idx.long(), False)  # a masked token is none of the teacher's
    full.masked_fill_(masked, float("-inf"))
    short = (_uniform((N, 1), seed, 6) < 0.1) & (torch.arange(k, device="cuda") >= max(1, k // 2))
    if N >= 8:
        short[N // 2] = True
    idx = torch.where(short, -1, idx).to(torch.int32)
    s = {"logits": full.to(DTYPES[dt])[:, :V], "idx": idx, "value": value}
    if case["kind"] == "distill_backward":
        z, m, e, total, rest, q, listed_q, log_z = _distill_parts(s["logits"], idx, value, T, case["tail"])
        s["stats"] = torch.stack([m, torch.log(total), torch.log(rest), listed_q if case["tail"] else log_z], 1)
        s["dloss"] = T * T / N * (0.5 + _uniform((N,), seed, 7))
    return s


def prepare(case, seed):
    make = _rms_inputs if case["kind"].startswith("rms") else _head_inputs if case["kind"].startswith("head") else _distill_inputs
    return {"case": case, **make(case, seed)}


# ---------------------------------------------------------------------------
# the plain forms: elementary operations in 32 bits
# ---------------------------------------------------------------------------

def _distill_parts(logits, idx, value, T, tail):
    """z = logits / T, its rows' maxima, exp(z - m), their sums over all and over the unlisted, the teacher's
    probabilities, their sum and the logarithm of what normalised them."""
    z = logits.float() / T
    N, V = z.shape
    valid = idx >= 0
    m = z.max(1).values
    e = torch.exp(z - m[:, None])
    unlisted = torch.ones((N, V + 1), dtype=torch.bool, device=z.device)
    unlisted.scatter_(1, torch.where(valid, idx, V).long(), False)
    rest = torch.where(unlisted[:, :V], e, 0.0).sum(1)
    if tail:
        q = torch.where(valid, torch.exp(value), 0.0)
        log_z = torch.zeros_like(m)
    else:
        t = torch.where(valid, value / T, float("-inf"))
        top = t.max(1, keepdim=True).values
        top = torch.where(top == float("-inf"), 0.0, top)
        q = torch.exp(t - top)
        log_z = torch.log(q.sum(1)) + top[:, 0]
        q = q / torch.where(log_z == float("-inf"), 1.0, q.sum(1))[:, None]
    return z, m, e, e.sum(1), rest, q, q.sum(1), log_z


def _plain_rms(s, case):
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "rms_backward":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh = s["h"].float() * rstd
        g = dy * s["w"]
        dx = rstd * (g - xh * (g * xh).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return dx.to(dt), (dy * xh).sum(0)
    x = s["x"].float()
    if s["residual"] is not None:
        x = x + s["residual"].float()
    rstd = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    y = x * rstd * s["w"]
    h = x.to(dt)
    if case["kind"] == "rms":
        return y.to(dt), h, rstd[:, 0]
    N, D = x.shape
    group = case["group"] or D
    groups = -(-D // group)
    padded = torch.zeros((N, groups * group), device=x.device)
    padded[:, :D] = y
    padded = padded.view(N, groups, group)
    scale = (padded.abs().max(2, keepdim=True).values / E4M3_MAX).clamp(min=2.0 ** -126)
    q = (padded / scale).view(N, -1)[:, :D].contiguous()
    return q.to(torch.float8_e4m3fn), scale[:, :, 0], h, rstd[:, 0]


def _plain_head(s, case):
    dt = DTYPES[case["dtype"]]
    X, W, targets = s["X"].float(), s["W"].float(), s["targets"]
    kept, at = targets != IGNORE, targets.clamp(min=0)[:, None]
    z = X @ W.t()
    m = z.max(1, keepdim=True).values
    z = z - m
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    log_s = torch.log(total)
    loss = torch.where(kept, (log_s - z.gather(1, at))[:, 0], 0.0)
    if case["kind"] == "head":
        return loss, torch.cat([m, log_s], 1)
    d = torch.where(kept, s["dloss"], 0.0)[:, None]
    p = e * (d / total)
    p.scatter_add_(1, at, -d)
    return loss, (p @ W).to(dt), (p.t() @ X).to(dt)


def _plain_distill(s, case):
    T, tail, idx = case["T"], case["tail"], s["idx"]
    z, m, e, total, rest, q, listed_q, log_z = _distill_parts(s["logits"], idx, s["value"], T, tail)
    valid = idx >= 0
    at = idx.clamp(min=0).long()
    # what the teacher leaves to the unlisted, where the student leaves them anything
    left = torch.where(rest > 0, (1.0 - listed_q).clamp(min=0.0), 0.0) if tail else torch.zeros_like(m)
    if case["kind"] == "distill":
        log_p = z.gather(1, at) - m[:, None] - torch.log(total)[:, None]
        loss = torch.where(valid & (q > 0), -q * log_p, 0.0).sum(1)
        loss = loss + torch.where(left > 0, left * (torch.log(total) - torch.log(rest)), 0.0)
        return loss, torch.stack([m, torch.log(total), torch.log(rest), listed_q if tail else log_z], 1)
    m, log_s, log_rest = s["stats"][:, 0], s["stats"][:, 1], s["stats"][:, 2]
    weight = s["dloss"] / T
    whole = listed_q + left
    p = torch.exp(z - m[:, None] - log_s[:, None]) * whole[:, None]
    if tail:
        r = torch.exp(z - m[:, None] - torch.where(rest > 0, log_rest, 0.0)[:, None])
        off = r * (torch.exp(log_rest - log_s) * whole - left)[:, None]
    else:
        off = p
    off = torch.cat([off, torch.zeros_like(off[:, :1])], 1)
    off.scatter_(1, torch.where(valid, at, z.shape[1]), p.gather(1, at) - q)
    return (off[:, :-1] * weight[:, None]).to(DTYPES[case["dtype"]])


def _plain(s):
    case = s["case"]
    make = _plain_rms if case["kind"].startswith("rms") else _plain_head if case["kind"].startswith("head") else _plain_distill
    return make(s, case)


def _own(s):
    import paper_1910_11971_gb300 as cci

    case = s["case"]
    kind = case["kind"]
    if kind == "rms":
        return cci.rms_norm(s["x"], s["w"], residual=s["residual"], eps=EPS)
    if kind == "rms_fp8":
        return cci.rms_norm_fp8(s["x"], s["w"], residual=s["residual"], group=case["group"], eps=EPS)
    if kind == "rms_backward":
        return cci.rms_norm_backward(s["dy"], s["h"], s["rstd"], s["w"], dh=s["dh"])
    if kind.startswith("head"):
        loss, stats = cci.linear_cross_entropy(s["X"], s["W"], s["targets"], ignore_index=IGNORE)
        if kind == "head":
            return loss, stats
        return (loss, *cci.linear_cross_entropy_backward(s["dloss"], s["X"], s["W"], s["targets"], stats, ignore_index=IGNORE))
    if kind == "distill":
        return cci.distillation_loss(s["logits"], s["idx"], s["value"], temperature=case["T"], tail=case["tail"])
    return cci.distillation_loss_backward(s["dloss"], s["logits"], s["idx"], s["value"], s["stats"], temperature=case["T"],
                                          tail=case["tail"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# work and the results in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    kind, es, N = case["kind"], 4 if case["dtype"] == "f32" else 2, case["N"]
    if kind.startswith("rms"):
        D, more = case["D"], 1 if case["residual"] else 0
        if kind == "rms_backward":
            return {"bytes": (3 + more) * N * D * es + 8 * D + 4 * N, "flops": 10 * N * D}
        rows = (1 + 2 * more) * es  # without a residual h is x
        if kind == "rms":
            return {"bytes": N * D * (rows + es) + 4 * D + 4 * N, "flops": 5 * N * D}
        groups = -(-D // (case["group"] or D))
        return {"bytes": N * D * (rows + 1) + 4 * D + 4 * N * (1 + groups), "flops": 8 * N * D}
    V = case["V"]
    if kind.startswith("head"):
        D = case["D"]
        if kind == "head":
            return {"bytes": (N + V) * D * es + N * (8 + 4 + 8), "flops": 2 * N * D * V}
        # the logits, dX and dW: that the logits come twice, where nothing keeps them, is not counted
        return {"bytes": 2 * (N + V) * D * es + N * (8 + 4 + 4), "flops": 6 * N * D * V}
    teacher = 8 * N * case["k"]
    if kind == "distill":
        return {"bytes": N * V * es + teacher + 20 * N, "flops": 4 * N * V}
    return {"bytes": 2 * N * V * es + teacher + N * (16 + 4), "flops": 5 * N * V}


def _exact_rms(s, case):
    w = s["w"].double()
    if case["kind"] == "rms_backward":
        h, dy, rstd = s["h"].double(), s["dy"].double(), s["rstd"].double()
        dot = torch.einsum("nd,nd,d->n", dy, h, w)
        dx = torch.einsum("nd,d,n->nd", dy, w, rstd) - h * (rstd ** 3 * dot / case["D"])[:, None]
        if s["dh"] is not None:
            dx += s["dh"].double()
        return dx, torch.einsum("nd,nd,n->d", dy, h, rstd)
    h = s["x"].double()
    if s["residual"] is not None:
        h = torch.add(h, s["residual"].double())
    rstd = (torch.linalg.vector_norm(h, dim=1) ** 2 / case["D"] + EPS) ** -0.5
    y = torch.einsum("nd,d,n->nd", h, w, rstd)
    if case["kind"] == "rms":
        return y, h, rstd
    q, scales = torch.empty_like(y), []
    width = case["group"] or case["D"]
    for at in range(0, case["D"], width):
        part = y[:, at:at + width]
        scales.append(torch.clamp(torch.linalg.vector_norm(part, ord=float("inf"), dim=1) / E4M3_MAX, min=2.0 ** -126))
        q[:, at:at + width] = part / scales[-1][:, None]
    return q, torch.stack(scales, 1), h, rstd


def _exact_head(s, case):
    X, W, targets = s["X"].double(), s["W"].double(), s["targets"]
    logits = torch.nn.functional.linear(X, W)
    lse = torch.logsumexp(logits, 1)
    m = logits.amax(1)
    loss = torch.nn.functional.nll_loss(logits - lse[:, None], targets, ignore_index=IGNORE, reduction="none")
    if case["kind"] == "head":
        return loss, torch.stack([m, lse - m], 1)
    kept = targets != IGNORE
    logits -= lse[:, None]
    p = logits.exp_()
    p[torch.arange(case["N"], device=X.device)[kept], targets[kept]] -= 1.0
    p *= torch.where(kept, s["dloss"].double(), 0.0)[:, None]
    return loss, torch.mm(p, W), torch.mm(p.t(), X)


def _exact_distill(s, case):
    T, tail, idx = case["T"], case["tail"], s["idx"].long()
    V = case["V"]
    log_p = torch.log_softmax(torch.cat([s["logits"].double() / T, torch.full_like(s["logits"][:, :1], float("-inf")).double()], 1), 1)
    places = torch.where(idx < 0, V, idx)  # one more column takes what is not listed
    others = log_p.scatter(1, places, float("-inf"))
    value = s["value"].double()
    if tail:
        log_q = torch.where(idx < 0, float("-inf"), value)
    else:
        log_q = torch.where(idx < 0, float("-inf"), value / T)
        log_q = log_q - torch.where((idx < 0).all(1), 0.0, torch.logsumexp(log_q, 1))[:, None]
    q = torch.exp(log_q)
    log_rest = torch.logsumexp(others, 1)
    left = torch.clamp(1.0 - q.sum(1), min=0.0) if tail else torch.zeros_like(q[:, 0])
    left = torch.where(log_rest == float("-inf"), 0.0, left)
    if case["kind"] == "distill":
        loss = -torch.where(q > 0, q * log_p.gather(1, places), 0.0).sum(1) - torch.where(left > 0, left * log_rest, 0.0)
        z = s["logits"].double() / T
        m, lse = z.amax(1), torch.logsumexp(z, 1)
        given = q.sum(1) if tail else torch.logsumexp(torch.where(idx < 0, float("-inf"), value / T), 1)
        return loss, torch.stack([m, lse - m, log_rest + lse - m, given], 1)
    target = torch.zeros_like(log_p).scatter_add_(1, places, q)
    if tail:
        target += torch.where(others == float("-inf"), 0.0, torch.exp(others - log_rest[:, None])) * left[:, None]
    d = torch.exp(log_p) * (q.sum(1) + left)[:, None] - target
    return (d * (s["dloss"].double() / T)[:, None])[:, :V]


def exact(case, seed):
    s = prepare(case, seed)
    make = _exact_rms if case["kind"].startswith("rms") else _exact_head if case["kind"].startswith("head") else _exact_distill
    return make(s, case)
