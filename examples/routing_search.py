"""A routing search from served outputs to the next configuration, on synthetic data.

Three models of rising quality and cost serve a trace of queries. The smallest
one's answers are scored by their log probabilities and entropies; a router
learns from them which model a query needs; a configuration theta (how much the
router favours each model, and the replicas behind each) is evaluated by routing
the trace under it, grouping the queries by model and reading off latency and
quality; and the search picks the next theta by expected hypervolume improvement.

    python examples/routing_search.py [--queries 4096] [--iterations 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2602_10729_amd as bo  # noqa: E402

MODELS = 3
COST = torch.tensor([1.0, 3.0, 9.0])          # work of a query, by model


def trace(queries, tokens, vocab, seed):
    """Logits of the small model's answers [queries * tokens, vocab], the answers'
    tokens, and every model's quality on every query [queries, MODELS]."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    hard = torch.rand(queries, generator=g, device="cuda")
    logits = torch.randn((queries * tokens, vocab), generator=g, device="cuda")
    answer = torch.randint(vocab, (queries * tokens,), generator=g, device="cuda")
    rows = torch.arange(queries * tokens, device="cuda")
    logits[rows, answer] += 12.0 * (1.0 - hard).repeat_interleave(tokens)
    skill = torch.tensor([0.35, 0.65, 0.95], device="cuda")
    quality = torch.sigmoid(10.0 * (skill - hard[:, None]))
    return logits.to(torch.bfloat16), answer, quality


def calibrate(logits, answer, steps=3):
    """A scale of the logits fitted to the answers: the gradient of their log
    probabilities, summed against the logits."""
    scale = 0.7
    for _ in range(steps):
        r = bo.token_logprobs(logits, answer, inv_temperature=scale)
        one = torch.full_like(r.logprob, 1.0 / len(r.logprob))
        grad = bo.token_logprobs_grad(logits, answer, r.stats, r.entropy, one, inv_temperature=scale)
        # d/d scale = sum over logits of grad / scale * logit
        scale += 0.2 * float((grad.float() * logits.float()).sum()) / scale
        scale = min(max(scale, 0.2), 3.0)
    return scale


def features(logits, answer, queries, scale):
    """Per query: mean log probability, mean entropy, share of tokens that were
    the model's first choice, gap to its best alternative; and 1."""
    r = bo.token_logprobs(logits, answer, top=2, inv_temperature=scale)
    per = lambda t: t.view(queries, -1).float().mean(1)
    f = torch.stack([per(r.logprob), per(r.entropy), per(r.rank == 1),
                     per(r.top_logprobs[:, 0] - r.top_logprobs[:, 1])], 1)
    f = (f - f.mean(0)) / (f.std(0) + 1e-6)
    return torch.cat([f, torch.ones((queries, 1), device="cuda")], 1)


def train_router(x, quality, steps=60, rate=4.0):
    """A linear router: the quality expected under its weights, less a little for
    cost, climbed along route_grad's gradient."""
    value = quality - 0.02 * COST.to(quality.device)
    w = torch.zeros((x.shape[1], MODELS), device="cuda")
    for _ in range(steps):
        logits = (x @ w).contiguous()
        r = bo.route(logits, MODELS, renormalise=False)
        g = value.gather(1, r.ids.long())
        w += rate * x.T @ bo.route_grad(logits, r.ids, g.contiguous(), renormalise=False) / len(x)
    return w


def evaluate(theta, router_logits, quality):
    """(-log latency, logit of mean quality) of a configuration: theta[0..2] how
    much each model is favoured, theta[3..5] its share of the replicas."""
    t = torch.as_tensor(theta, dtype=torch.float32, device="cuda")
    bias = t[:MODELS].contiguous()
    r = bo.route(router_logits, 1, bias=bias)
    d = bo.dispatch(r.ids, MODELS)
    replicas = 0.5 + 3.5 * t[MODELS:]
    busy = d.load.float() * COST.to(t.device) / replicas
    latency = float(busy.max()) / len(router_logits) + 0.05 * float(replicas.sum())
    # the queries of each model, as its replicas would take them
    got = torch.cat([quality[d.order[d.offsets[m]:d.offsets[m + 1]].long(), m] for m in range(MODELS)])
    q = float(got.mean())
    return [-float(np.log(latency)), float(np.log(q / (1.0 - q)))]


def hypervolume(Y, ref):
    front = Y[bo.pareto_front(Y, ref)]
    total, low = 0.0, ref[1]
    for a, b in front[np.argsort(-front[:, 0])]:
        if b > low:
            total += (a - ref[0]) * (b - low)
            low = b
    return total


def main(queries=4096, tokens=16, vocab=4096, iterations=8, seed=0, verbose=True):
    """Runs the search; returns the hypervolume after each iteration."""
    logits, answer, quality = trace(queries, tokens, vocab, seed)
    scale = calibrate(logits, answer)
    x = features(logits, answer, queries, scale)
    router_logits = (x @ train_router(x, quality)).contiguous()
    rng = np.random.default_rng(seed)
    dims = 2 * MODELS
    thetas = rng.random((24, dims)).astype(np.float32)
    raw = np.array([evaluate(t, router_logits, quality) for t in thetas], np.float32)
    ref_raw = raw.min(0) - 0.1
    history = [hypervolume(raw, ref_raw)]
    Z = torch.randn((256, 1, 2), device="cuda")
    for it in range(iterations):
        mean, std = raw.mean(0), raw.std(0) + 1e-6
        X = torch.from_numpy(thetas).cuda()
        Y = torch.from_numpy((raw - mean) / std).cuda()
        model = bo.fit(X, Y, np.full((2, dims), 0.5, np.float32), [1.0, 1.0], [1e-3, 1e-3])
        cand = torch.from_numpy(rng.random((8192, 1, dims)).astype(np.float32)).cuda()
        ehvi = bo.score(model, cand, (ref_raw - mean) / std, Z)
        best, _ = bo.argmax(ehvi)
        theta = cand[int(best), 0].cpu().numpy()
        thetas = np.vstack([thetas, theta])
        raw = np.vstack([raw, np.array(evaluate(theta, router_logits, quality), np.float32)])
        history.append(hypervolume(raw, ref_raw))
        if verbose:
            print(f"iteration {it}: latency {np.exp(-raw[-1, 0]):.3f}, quality "
                  f"{1 / (1 + np.exp(-raw[-1, 1])):.3f}, hypervolume {history[-1]:.4f}")
    if verbose:
        for i in bo.pareto_front(raw, None):
            print(f"  theta {np.round(thetas[i], 2)}: latency {np.exp(-raw[i, 0]):.3f}, "
                  f"quality {1 / (1 + np.exp(-raw[i, 1])):.3f}")
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--queries", type=int, default=4096)
    ap.add_argument("--iterations", type=int, default=8)
    a = ap.parse_args()
    main(queries=a.queries, iterations=a.iterations)
