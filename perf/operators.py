"""The operators of a pruned language model's feed-forward sub-layer and of what its head answers, as cases
that can be timed and compared: layer norm, the gated feed-forward block and the log probabilities of tokens.

A case is a dict of plain values.  ``kind`` says which call it is:

  norm            ``layer_norm``: rows x, weight, bias -> y, mean, rstd
  norm_backward   ``layer_norm_backward``: dy, x, mean, rstd, weight -> dx, dweight, dbias
  gated           ``gated_linear``: h = act(x Wg^T) * (x Wu^T) with dense weights
  gated_packed    ``gated_linear_packed``: the same with both weights in the packed (G, K) format
  gated_step      ``gated_linear`` and ``gated_linear_backward``: one training pass, h, dx, dWg, dWu
  logprobs        ``token_logprobs``: log probability of one token per row, entropy, top alternatives
  logprobs_backward  ``token_logprobs_backward``: the gradient of both to the logits

With ``own`` false, ``run`` computes them in elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("silu", "gelu", "gelu_tanh", "relu", "sigmoid")
IGNORE = -100  # a token of this value is left out: log probability 0, no gradient
EPS = 1e-5


def _norm(name, kind, N, D, dtype):
    return {"name": name, "kind": kind, "N": N, "D": D, "dtype": dtype}


def _gated(name, kind, N, D, F, act, dtype, G=0, K=0):
    return {"name": name, "kind": kind, "N": N, "D": D, "F": F, "act": act, "dtype": dtype, "G": G, "K": K}


def _logprobs(name, kind, N, V, dtype, top=0, pad=0):
    return {"name": name, "kind": kind, "N": N, "V": V, "dtype": dtype, "top": top, "pad": pad}


def listed():
    return [
        # one token of a model 4096 wide, as in every decoding step: launch and latency are all there is
        _norm("norm_token", "norm", 1, 4096, "bf16"),
        # a training batch of 16384 tokens
        _norm("norm_batch", "norm", 16384, 4096, "bf16"),
        # the gradient of that batch, with the sums over its rows for weight and bias
        _norm("norm_batch_backward", "norm_backward", 16384, 4096, "bf16"),
        # fp32 rows whose width fits no vector load, an odd number of them
        _norm("norm_odd_backward_f32", "norm_backward", 5003, 1001, "f32"),
        # one token through the block: the weights are all that is read
        _gated("gated_token", "gated", 1, 4096, 8192, "silu", "bf16"),
        # a prompt of no round length
        _gated("gated_prompt", "gated", 1999, 4096, 8192, "silu", "bf16"),
        # a training pass, forward and backward
        _gated("gated_step", "gated_step", 4096, 4096, 8192, "silu", "bf16"),
        # a training pass of a small model in fp32
        _gated("gated_step_f32", "gated_step", 1000, 1024, 2048, "gelu", "f32"),
        # sixteen requests through a pruned block: packed weights, 2 of 8 kept
        _gated("gated_packed_serve", "gated_packed", 16, 4096, 4096, "relu", "bf16", 8, 2),
        # a decoding step of eight requests: alternatives reported beside each chosen token
        _logprobs("logprobs_token", "logprobs", 8, 131072, "f32", 20),
        # scoring a prompt
        _logprobs("logprobs_prompt", "logprobs", 1024, 131072, "bf16", 5),
        # the loss's gradient over an odd vocabulary, its logits in rows padded to whole vectors
        _logprobs("logprobs_backward", "logprobs_backward", 4096, 50001, "bf16", 0, 7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any number of rows or tokens, widths odd and round, every activation and both types."""
    kind = rng.choice(("norm", "norm_backward", "gated", "gated", "gated_packed", "gated_step", "logprobs",
                       "logprobs", "logprobs_backward"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind.startswith("norm"):
        D = _log_int(rng, 16, 16384)
        if rng.random() < 0.6:
            D = -(-D // 8) * 8
        most = 16384 * 4096 // (2 if dtype == "f32" else 1)
        return {"kind": kind, "N": _log_int(rng, 1, min(65536, max(1, most // D))), "D": D, "dtype": dtype}
    if kind.startswith("gated"):
        G, K = rng.choice(((4, 1), (4, 2), (8, 1), (8, 2), (8, 4), (16, 2), (16, 4), (32, 8))) if kind == "gated_packed" else (0, 0)
        D = 8 * max(1, _log_int(rng, 64, 4096) // 8)
        F = max(8, G) * max(1, _log_int(rng, 64, 8192) // max(8, G))
        # at most the listed training pass's products in bf16, a sixteenth of them in fp32
        most = 4096 * 4096 * 8192 // (16 if dtype == "f32" else 1)
        return {"kind": kind, "N": _log_int(rng, 1, min(8192, max(1, most // (D * F)))), "D": D, "F": F,
                "act": rng.choice(ACTS), "dtype": dtype, "G": G, "K": K}
    V = _log_int(rng, 2, 131072)
    if rng.random() < 0.5:
        V = -(-V // 8) * 8
    most = 1024 * 131072 // (2 if dtype == "f32" else 1)
    top = min(V, rng.choice((0, 1, 5, 20))) if kind == "logprobs" else 0
    return {"kind": kind, "N": _log_int(rng, 1, min(8192, max(1, most // V))), "V": V, "dtype": dtype, "top": top,
            "pad": rng.choice((0, 0, (-V) % 8, 3))}


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


def _packed(W, G, K):
    """The K weights of largest magnitude of every group of G output channels at one input, ties to the lower
    index, in increasing index: values and idx [F/G][D][K]."""
    F, D = W.shape
    w = W.view(F // G, G, D)
    keep = torch.sort(w.abs(), dim=1, descending=True, stable=True).indices[:, :K].sort(dim=1).values
    values = w.gather(1, keep).permute(0, 2, 1).contiguous()
    return values, keep.permute(0, 2, 1).contiguous().to(torch.uint8)


def _norm_inputs(case, seed):
    """Rows as a residual stream has them: an offset, a spread of their own, a few channels far out."""
    N, D, dt = case["N"], case["D"], case["dtype"]
    x = _normal((N, D), 1.0, "f32", seed, 1) * (0.5 + 2.0 * _uniform((N, 1), seed, 2)) + 0.3
    x += 8.0 * (_uniform((1, D), seed, 3) > 0.99)
    s = {"x": x.to(DTYPES[dt]), "w": 1.0 + _normal((D,), 0.2, "f32", seed, 4), "b": _normal((D,), 0.1, "f32", seed, 5)}
    if case["kind"] == "norm_backward":
        xf = s["x"].float()
        s["mean"] = xf.mean(1)
        s["rstd"] = torch.rsqrt((xf - s["mean"][:, None]).square().mean(1) + EPS)
        s["dy"] = _normal((N, D), 0.05, dt, seed, 6)
    return s


def _gated_inputs(case, seed):
    N, D, F, dt = case["N"], case["D"], case["F"], case["dtype"]
    s = {"x": _normal((N, D), 1.0, dt, seed, 1)}
    s["wg"] = _normal((F, D), math.sqrt(2.0 / D), dt, seed, 2)
    s["wu"] = _normal((F, D), math.sqrt(1.0 / D), dt, seed, 3)
    if case["kind"] == "gated_step":
        s["dh"] = _normal((N, F), 0.02, dt, seed, 4)
    if case["kind"] == "gated_packed":
        s["gate"] = _packed(s.pop("wg"), case["G"], case["K"])
        s["up"] = _packed(s.pop("wu"), case["G"], case["K"])
    return s


def _logprobs_inputs(case, seed):
    """Logits of a head: a spread that differs from row to row, some rows with a part of the vocabulary masked,
    from eight rows on one with all of it masked; some tokens left out."""
    N, V, dt = case["N"], case["V"], case["dtype"]
    full = _normal((N, V + case["pad"]), 1.0, "f32", seed, 1) * (0.5 + 3.0 * _uniform((N, 1), seed, 2))
    masked = (_uniform((N, 1), seed, 3) < 0.2) & (_uniform((N, V + case["pad"]), seed, 4) < 0.4)
    full.masked_fill_(masked, float("-inf"))
    if N >= 8:
        full[N // 2] = float("-inf")
    logits = full.to(DTYPES[dt])[:, :V]
    tokens = (_uniform((N,), seed, 5) * V).long().clamp_(max=V - 1)
    tokens[_uniform((N,), seed, 6) < 0.05] = IGNORE
    s = {"logits": logits, "tokens": tokens}
    if case["kind"] == "logprobs_backward":
        x = logits.float()
        m = x.max(1, keepdim=True).values
        y = x - torch.where(m == float("-inf"), 0.0, m)
        e = torch.exp(y)
        total = e.sum(1, keepdim=True)
        empty = total == 0
        log_s = torch.where(empty, 0.0, torch.log(total))
        s["stats"] = torch.cat([m, log_s], 1)
        s["entropy"] = torch.where(empty, 0.0, log_s - torch.where(e > 0, e * y, 0.0).sum(1, keepdim=True) / total)[:, 0]
        s["dlogp"] = _normal((N,), 1.0 / N, "f32", seed, 7) - 1.0 / N
        s["dentropy"] = _normal((N,), 0.1 / N, "f32", seed, 8)
    return s


def prepare(case, seed):
    make = _norm_inputs if case["kind"].startswith("norm") else _gated_inputs if case["kind"].startswith("gated") else _logprobs_inputs
    return {"case": case, **make(case, seed)}


# ---------------------------------------------------------------------------
# the plain forms: elementary operations in 32 bits
# ---------------------------------------------------------------------------

def _act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    if act == "gelu":
        return 0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))
    if act == "relu":
        return torch.where(g > 0, g, 0.0)
    return 1.0 / (1.0 + torch.exp(-g))


def _act_slope(g, act):
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return p * (1.0 + g * (1.0 - p))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)
    if act == "relu":
        return torch.where(g > 0, 1.0, 0.0)
    p = 1.0 / (1.0 + torch.exp(-g))
    return p * (1.0 - p)


def _dense(packed, F, G):
    """The fp32 matrix of packed weights."""
    values, idx = packed
    w = torch.zeros((F // G, values.shape[1], G), dtype=torch.float32, device=values.device)
    w.scatter_(2, idx.long(), values.float())
    return w.permute(0, 2, 1).reshape(F, -1)


def _plain(s):
    case = s["case"]
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    if kind == "norm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        return ((x - mean) * rstd * s["w"] + s["b"]).to(dt), mean[:, 0], rstd[:, 0]
    if kind == "norm_backward":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh = (s["x"].float() - s["mean"][:, None]) * rstd
        g = dy * s["w"]
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return dx.to(dt), (dy * xh).sum(0), dy.sum(0)
    if kind.startswith("gated"):
        x = s["x"].float()
        if kind == "gated_packed":
            wg, wu = _dense(s["gate"], case["F"], case["G"]), _dense(s["up"], case["F"], case["G"])
        else:
            wg, wu = s["wg"].float(), s["wu"].float()
        g, u = x @ wg.t(), x @ wu.t()
        h = (_act(g, case["act"]) * u).to(dt)
        if kind != "gated_step":
            return h
        dh = s["dh"].float()
        dg, du = dh * u * _act_slope(g, case["act"]), dh * _act(g, case["act"])
        return h, (dg @ wg + du @ wu).to(dt), (dg.t() @ x).to(dt), (du.t() @ x).to(dt)
    x, tokens = s["logits"].float(), s["tokens"]
    at = tokens.clamp(min=0)[:, None]
    kept = tokens != IGNORE
    if kind == "logprobs":
        m = x.max(1, keepdim=True).values
        empty = m == float("-inf")
        y = x - torch.where(empty, 0.0, m)
        e = torch.exp(y)
        total = torch.where(empty, 1.0, e.sum(1, keepdim=True))
        log_s = torch.log(total)
        entropy = log_s - torch.where(e > 0, e * y, 0.0).sum(1, keepdim=True) / total
        logp = torch.where(kept, (y.gather(1, at) - log_s)[:, 0], 0.0)
        out = [logp, entropy[:, 0], torch.cat([m, log_s], 1)]
        if case["top"]:
            best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            out += [y.gather(1, best) - log_s, best.to(torch.int32)]
        return tuple(out)
    m, log_s = s["stats"][:, :1], s["stats"][:, 1:]
    empty = m == float("-inf")
    lp = x - torch.where(empty, 0.0, m) - log_s
    p = torch.exp(lp)
    dlogp = torch.where(kept, s["dlogp"], 0.0)[:, None]
    dx = -dlogp * p - s["dentropy"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    dx.scatter_add_(1, at, dlogp)
    return torch.where(empty, 0.0, dx).to(dt)


def _own(s):
    import paper_1910_11971_gb300 as cci

    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        return cci.layer_norm(s["x"], s["w"], s["b"], eps=EPS)
    if kind == "norm_backward":
        return cci.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["w"])
    if kind == "gated":
        return cci.gated_linear(s["x"], s["wg"], s["wu"], act=case["act"])
    if kind == "gated_packed":
        return cci.gated_linear_packed(s["x"], s["gate"], s["up"], case["F"], case["G"], case["K"], act=case["act"])
    if kind == "gated_step":
        h, g, u = cci.gated_linear(s["x"], s["wg"], s["wu"], act=case["act"], save=True)
        return (h, *cci.gated_linear_backward(s["dh"], s["x"], s["wg"], s["wu"], g, u, act=case["act"]))
    if kind == "logprobs":
        logp, entropy, stats, top_logp, top_idx = cci.token_logprobs(s["logits"], s["tokens"], top=case["top"], ignore_index=IGNORE)
        return (logp, entropy, stats) + ((top_logp, top_idx) if case["top"] else ())
    return cci.token_logprobs_backward(s["logits"], s["tokens"], s["stats"], dlogp=s["dlogp"], entropy=s["entropy"],
                                       dentropy=s["dentropy"], ignore_index=IGNORE)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# work and the results in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    kind, es = case["kind"], 4 if case["dtype"] == "f32" else 2
    N = case["N"]
    if kind == "norm":
        D = case["D"]
        return {"bytes": 2 * N * D * es + 8 * D + 8 * N, "flops": 7 * N * D}
    if kind == "norm_backward":
        D = case["D"]
        return {"bytes": 3 * N * D * es + 4 * D + 8 * N + 8 * D, "flops": 14 * N * D}
    if kind.startswith("gated"):
        D, F = case["D"], case["F"]
        if kind == "gated":
            return {"bytes": (N * D + 2 * F * D + N * F) * es, "flops": 4 * N * D * F}
        if kind == "gated_packed":
            G, K = case["G"], case["K"]
            return {"bytes": (N * D + N * F) * es + 2 * F // G * D * K * (es + 1), "flops": 4 * N * D * F * K // G}
        return {"bytes": (2 * N * D + 4 * F * D + 2 * N * F) * es, "flops": 12 * N * D * F}
    V = case["V"]
    if kind == "logprobs":
        return {"bytes": N * V * es + N * (8 + 4 + 4 + 8 + 8 * case["top"]), "flops": 5 * N * V}
    return {"bytes": 2 * N * V * es + N * (8 + 8 + 4 + 4 + 4), "flops": 7 * N * V}


def _exact_act(g, act):
    """(act(g), act'(g)) in 64 bits, the slope by differentiating act."""
    g = g.detach().requires_grad_(True)
    with torch.enable_grad():
        if act == "silu":
            a = g * torch.sigmoid(g)
        elif act == "gelu":
            a = g * torch.special.ndtr(g)
        elif act == "gelu_tanh":
            a = g * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3))
        elif act == "relu":
            a = g * (g.detach() > 0)
        else:
            a = torch.sigmoid(g)
        slope, = torch.autograd.grad(a.sum(), g)
    return a.detach(), slope


def _exact_dense(packed, F, G):
    values, idx = packed
    groups, D, K = values.shape
    one = torch.nn.functional.one_hot(idx.long(), G).double()  # [group][d][slot][row]
    return torch.einsum("gdkj,gdk->gjd", one, values.double()).reshape(F, D)


def exact(case, seed):
    kind = case["kind"]
    if kind.startswith("norm"):
        s = _norm_inputs(case, seed)
        x, w = s["x"].double(), s["w"].double()
        if kind == "norm":
            var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
            rstd = (var + EPS) ** -0.5
            return torch.addcmul(s["b"].double(), (x - mean) * rstd, w), mean[:, 0], rstd[:, 0]
        dy, rstd, D = s["dy"].double(), s["rstd"].double()[:, None], case["D"]
        xh = (x - s["mean"].double()[:, None]) * rstd
        wdy = dy * w
        a, b = wdy.sum(1, keepdim=True) / D, torch.einsum("nd,nd->n", wdy, xh)[:, None] / D
        return (wdy - a - xh * b) * rstd, torch.einsum("nd,nd->d", dy, xh), torch.ones_like(rstd[:, 0]) @ dy
    if kind.startswith("gated"):
        s = _gated_inputs(case, seed)
        x = s["x"].double()
        if kind == "gated_packed":
            wg, wu = (_exact_dense(s[k], case["F"], case["G"]) for k in ("gate", "up"))
        else:
            wg, wu = s["wg"].double(), s["wu"].double()
        g, u = torch.nn.functional.linear(x, wg), torch.nn.functional.linear(x, wu)
        a, slope = _exact_act(g, case["act"])
        if kind != "gated_step":
            return a * u
        dh = s["dh"].double()
        dg, du = dh * u * slope, dh * a
        return a * u, torch.addmm(dg @ wg, du, wu), dg.t() @ x, du.t() @ x
    s = _logprobs_inputs(case, seed)
    x, tokens = s["logits"].double(), s["tokens"]
    rows = torch.arange(case["N"], device=x.device)
    kept, at = tokens != IGNORE, tokens.clamp(min=0)
    if kind == "logprobs":
        lse = torch.logsumexp(x, 1)
        empty = lse == float("-inf")
        lp = torch.where(empty[:, None], float("-inf"), x - lse[:, None])
        p = torch.exp(lp)
        entropy = torch.special.entr(p).sum(1)
        m = x.amax(1)
        out = [torch.where(kept, lp[rows, at], 0.0), entropy, torch.stack([m, torch.where(empty, 0.0, lse - m)], 1)]
        if case["top"]:
            best = torch.argsort(-x, dim=1, stable=True)[:, :case["top"]]
            out += [lp.gather(1, best), best.to(torch.int32)]
        return tuple(out)
    m, log_s = s["stats"].double().unbind(1)
    empty = m == float("-inf")
    lp = x - (torch.where(empty, 0.0, m) + log_s)[:, None]
    p = torch.exp(lp)
    dlogp = torch.where(kept, s["dlogp"].double(), 0.0)
    d = -p * dlogp[:, None] - s["dentropy"].double()[:, None] * (p * s["entropy"].double()[:, None] - torch.special.entr(p))
    d[rows, at] += dlogp
    return torch.where(empty[:, None], 0.0, d)
