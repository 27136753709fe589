"""Train a small language model's feed-forward sub-layer with targeted dropout, pack it, and serve it.

The model sees one token and predicts the next:

    y = layer_norm(embedding[token])          cci.layer_norm
    h = silu(y Wg^T) * (y Wu^T)               cci.gated_linear (training), cci.gated_linear_packed (serving)
    logits = h Wh^T                           cci.dense_linear_tc
    log p(next), entropy, alternatives        cci.token_logprobs

Every training step masks Wg and Wu with targeted dropout (``cci.td_mask``, Sec. 5.1 of arXiv 1910.11971), so
that in the end the K of every G weights that packing keeps carry the model; their gradients go through the
masked weights.  Master weights are fp32, the products bf16.  The data are a seeded Markov chain whose tokens
have a few likely successors each: the entropy of that chain is the loss to reach.

    python examples/pruned_feed_forward.py [--steps 150]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1910_11971_gb300 as cci

TOKENS, WIDTH, HIDDEN, BATCH = 512, 256, 512, 1024
G, K = 8, 2
SUCCESSORS = 4  # likely next tokens of each token


class Adam:
    """Adam on fp32 master weights (PyTorch arithmetic; not part of the library)."""

    def __init__(self, params, lr):
        self.params, self.lr, self.t = params, lr, 0
        self.m = [torch.zeros_like(p) for p in params]
        self.v = [torch.zeros_like(p) for p in params]

    def step(self, grads):
        self.t += 1
        for p, m, v, g in zip(self.params, self.m, self.v, grads):
            m.lerp_(g, 0.1)
            v.lerp_(g * g, 0.01)
            p -= self.lr * (m / (1 - 0.9 ** self.t)) / ((v / (1 - 0.99 ** self.t)).sqrt() + 1e-8)


def chain(gen, device):
    """(successors [TOKENS][SUCCESSORS], their cumulative probabilities, entropy per token in nats)."""
    nxt = torch.rand((TOKENS, TOKENS), generator=gen, device=device).argsort(1)[:, :SUCCESSORS]
    p = torch.tensor([0.5, 0.25, 0.15, 0.1], device=device)
    return nxt, p.cumsum(0), float(-(p * p.log()).sum())


def batch(nxt, cum, gen, n, device):
    token = torch.randint(0, TOKENS, (n,), generator=gen, device=device)
    pick = (torch.rand((n, 1), generator=gen, device=device) > cum[:-1]).sum(1)
    return token, nxt[token, pick]


def main(steps=150, seed=0):
    device = torch.device("cuda:0")
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    nxt, cum, floor = chain(gen, device)

    def normal(*shape, std):
        return torch.randn(shape, generator=gen, device=device) * std

    emb = normal(TOKENS, WIDTH, std=1.0).bfloat16()
    norm_w, norm_b = torch.ones(WIDTH, device=device), torch.zeros(WIDTH, device=device)
    wg, wu = normal(HIDDEN, WIDTH, std=math.sqrt(2.0 / WIDTH)), normal(HIDDEN, WIDTH, std=math.sqrt(1.0 / WIDTH))
    wh = normal(TOKENS, HIDDEN, std=math.sqrt(1.0 / HIDDEN))
    opt = Adam([norm_w, norm_b, wg, wu, wh], lr=4e-3)
    status = cci.new_status(device)
    losses = []
    for step in range(steps):
        token, target = batch(nxt, cum, gen, BATCH, device)
        # the pruning candidates are dropped more and more often; from two thirds of the steps on, always
        rate = cci.td_drop_rate(step, 2 * steps // 3, 0.0, 1.0)
        draws = [torch.rand(w.shape, generator=gen, device=device) for w in (wg, wu)]
        (wg_kept, mask_g), (wu_kept, mask_u) = (cci.td_mask(w, G, K, rate, u, status=status) for w, u in zip((wg, wu), draws))
        wg16, wu16, wh16 = wg_kept.bfloat16(), wu_kept.bfloat16(), wh.bfloat16()
        # forward
        x = emb[token]
        y, mean, rstd = cci.layer_norm(x, norm_w, norm_b)
        h, g, u = cci.gated_linear(y, wg16, wu16, act="silu", save=True, status=status)
        logits = cci.dense_linear_tc(h, wh16, TOKENS, status=status)
        logp, _, stats, _, _ = cci.token_logprobs(logits, target, status=status)
        losses.append(-logp.mean())
        # backward
        dlogits = cci.token_logprobs_backward(logits, target, stats, dlogp=torch.full_like(logp, -1.0 / BATCH)).bfloat16()
        dh, dwh = dlogits @ wh16, dlogits.t() @ h
        dy, dwg, dwu = cci.gated_linear_backward(dh, y, wg16, wu16, g, u, act="silu", status=status)
        _, dnw, dnb = cci.layer_norm_backward(dy, x, mean, rstd, norm_w)
        opt.step([dnw, dnb, dwg.float() * mask_g, dwu.float() * mask_u, dwh.float()])

    # serving: packed weights, a prompt's log probabilities and one token's alternatives
    gate, up = cci.pack(wg.bfloat16(), G, K), cci.pack(wu.bfloat16(), G, K)
    wh16 = wh.bfloat16()

    def answer(token, target, top=0):
        y, _, _ = cci.layer_norm(emb[token], norm_w, norm_b)
        h = cci.gated_linear_packed(y, gate, up, HIDDEN, G, K, act="silu", status=status)
        return cci.token_logprobs(cci.dense_linear_tc(h, wh16, TOKENS, status=status), target, top=top, status=status)

    token, target = batch(nxt, cum, gen, 4 * BATCH, device)
    logp, entropy, _, _, _ = answer(token, target)
    one = torch.arange(8, device=device)
    alone = [answer(t, nxt[t, 0], top=SUCCESSORS) for t in one.split(1)]
    found = torch.cat([a[4] for a in alone])
    hits = (found[:, :, None] == nxt[one][:, None, :]).any(2).float().mean()
    return {"first": float(losses[0]), "last": float(torch.stack(losses[-10:]).mean()), "packed": float(-logp.mean()),
            "entropy": float(entropy.mean()), "floor": floor, "hits": float(hits), "status": cci.read_status(status)}


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=150)
    r = main(parser.parse_args().steps)
    print(f"loss per token: {r['first']:.3f} at the start (uniform {math.log(TOKENS):.3f}), {r['last']:.3f} at the end of "
          f"training, {r['packed']:.3f} with packed weights ({K} of {G} kept); the chain's entropy is {r['floor']:.3f}")
    print(f"entropy of the answers {r['entropy']:.3f}; {100 * r['hits']:.0f} % of the alternatives of single tokens are "
          f"successors in the chain")
