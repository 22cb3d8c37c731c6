"""Training a small language model with an expert layer, on synthetic data.

Tokens enter by their rows of a table (embed), a router sends each to its best
experts (route, dispatch, expert_gather), the experts' outputs come back under the
router's weights (expert_combine), and the same table scores the next token
(linear_logprobs). The gradients are the operators' own, put together by hand; the
experts' products are torch's.

    python examples/expert_model.py [--steps 60]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2602_10729_amd as bo  # noqa: E402


def parameters(vocab, width, experts, hidden, seed, dtype=torch.float32):
    """Table [vocab, width], router [width, experts], the experts' two matrices."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda")
    return dict(table=(draw(vocab, width) / width ** 0.5).to(dtype), router=draw(width, experts) / width ** 0.5,
                up=(draw(experts, width, hidden) / width ** 0.5).to(dtype),
                down=(draw(experts, hidden, width) / hidden ** 0.5).to(dtype))


def step(p, tokens, targets, top, capacity=0):
    """(mean log probability of the targets, its gradient by parameter, the
    router's choices). Tokens and targets < 0 are padding."""
    experts, (vocab, width) = p["router"].shape[1], p["table"].shape
    scale = width ** 0.5
    x = bo.embed(tokens, p["table"], scale=scale)
    logits = (x.float() @ p["router"]).contiguous()
    to = bo.route(logits, top)
    d = bo.dispatch(to.ids, experts, capacity=capacity)
    rows = bo.expert_gather(x, d.order, d.position)
    at = d.offsets.tolist()
    inner, z = [], torch.zeros_like(rows)
    for e in range(experts):
        inner.append(rows[at[e]:at[e + 1]] @ p["up"][e])
        z[at[e]:at[e + 1]] = torch.relu(inner[e]) @ p["down"][e]
    y = x + bo.expert_combine(z, d.position, to.weights)
    r = bo.linear_logprobs(y, p["table"], targets)
    count = (targets >= 0).sum()

    g = bo.linear_logprobs_grad(y, p["table"], targets, r.stats, r.entropy,
                                torch.full_like(r.logprob, 1.0) / count)
    c = bo.expert_combine_grad(g.hidden, z, d.order, d.position, to.weights)
    grads = dict(up=torch.zeros_like(p["up"]), down=torch.zeros_like(p["down"]))
    back = torch.zeros_like(rows)
    for e in range(experts):
        s = slice(at[e], at[e + 1])
        grads["down"][e] = torch.relu(inner[e]).T @ c.rows[s]
        du = (c.rows[s] @ p["down"][e].T) * (inner[e] > 0)
        grads["up"][e] = rows[s].T @ du
        back[s] = du @ p["up"][e].T
    dl = bo.route_grad(logits, to.ids, c.weights)
    grads["router"] = x.float().T @ dl
    dx = g.hidden + bo.expert_combine(back, d.position) + (dl @ p["router"].T).to(x.dtype)
    grads["table"] = g.weight + bo.embed_grad(tokens, dx, vocab, scale=scale)
    return r.logprob.sum() / count, grads, to.ids


def main(vocab=512, width=64, experts=8, hidden=96, top=2, batch=1024, steps=60, rate=3.0, seed=0,
         verbose=True):
    """Learns a fixed successor of every token; returns the mean log probability
    after each step."""
    p = parameters(vocab, width, experts, hidden, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    successor = torch.randperm(vocab, generator=g, device="cuda")
    history = []
    for i in range(steps):
        tokens = torch.randint(vocab, (batch,), generator=g, device="cuda")
        tokens[::16] = -1
        targets = torch.where(tokens >= 0, successor[tokens.clamp(min=0)], -1)
        value, grads, _ = step(p, tokens, targets, top, capacity=2 * batch * top // experts)
        for k in p:
            p[k] = p[k] + rate * grads[k]
        history.append(float(value))
        if verbose and i % 10 == 9:
            print(f"step {i + 1}: mean log probability {history[-1]:.3f}")
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    main(steps=ap.parse_args().steps)
