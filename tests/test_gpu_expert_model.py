"""The operators together, as a language model with an expert layer uses them: the
example's gradients against torch's differentiation of the same function in 64
bits, against differences, and the example itself."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
EPS = 2.0 ** -24


def _value(p, tokens, targets, ids, kept, width):
    """The model's mean log probability in plain torch, the choices given."""
    import torch
    scale = width ** 0.5
    has = tokens >= 0
    x = torch.where(has[:, None], p["table"][tokens.clamp(min=0)] * scale, 0.0)
    logits = x @ p["router"]
    chosen = torch.gather(torch.softmax(logits, 1), 1, ids.clamp(min=0))
    w = chosen / chosen.sum(1, keepdim=True)
    y = x
    for k in range(ids.shape[1]):
        e = ids[:, k].clamp(min=0)
        out = torch.stack([torch.relu(x[t] @ p["up"][e[t]]) @ p["down"][e[t]] for t in range(len(x))])
        y = y + torch.where(kept[:, k:k + 1], w[:, k:k + 1] * out, 0.0)
    lsm = torch.log_softmax(y @ p["table"].T, 1)
    live = targets >= 0
    return torch.where(live, lsm.gather(1, targets.clamp(min=0)[:, None])[:, 0], 0.0).sum() / live.sum()


def _case(seed, V=300, H=24, E=5, F=20, T=90, top=2, dtype=None):
    import torch
    import expert_model as M
    p = M.parameters(V, H, E, F, seed, dtype or torch.float32)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    tokens = torch.randint(V, (T,), generator=g, device="cuda")
    tokens[:T // 3] = tokens[0]                       # a frequent one
    targets = torch.randint(V, (T,), generator=g, device="cuda")
    tokens[5::11] = -1
    targets[4::9] = -1
    return p, tokens, targets


@pytest.mark.parametrize("capacity", [0, 20])
def test_gradients(capacity):
    import torch
    import paper_2602_10729_amd as bo
    import expert_model as M
    print("[case] expert model gradients", capacity, flush=True)
    p, tokens, targets = _case(3)
    value, grads, ids = M.step(p, tokens, targets, 2, capacity=capacity)
    kept = bo.dispatch(ids, 5, capacity=capacity).position >= 0
    q = {k: v.double().requires_grad_(True) for k, v in p.items()}
    want = _value(q, tokens, targets, ids.long(), kept, 24)
    want.backward()
    # every number is a chain of six sums of at most 300 terms, each off by
    # (2 sqrt(300) + 4) eps of the size of its terms; with cancellation, terms are
    # up to ten times the largest result
    tol = 6 * 10 * (2 * 300 ** 0.5 + 4) * EPS
    assert abs(float(value) - float(want)) <= tol * abs(float(want))
    for k in p:
        off = float((grads[k].double() - q[k].grad).abs().max())
        assert off <= tol * float(q[k].grad.abs().max()), (k, off)
    # differences of the 64-bit function along random directions
    for k in p:
        v = torch.randn_like(q[k])
        h = 1e-6
        with torch.no_grad():
            a, b = ({**q, k: q[k] + s * h * v} for s in (1, -1))
            num = float(_value(a, tokens, targets, ids.long(), kept, 24)
                        - _value(b, tokens, targets, ids.long(), kept, 24)) / (2 * h)
        got = float((grads[k].double() * v).sum())
        assert abs(num - got) <= 1e-6 + tol * float((grads[k].double() * v).abs().sum()), k


def test_half_types_run():
    """The same step in 16 bits: finite, and near the single-precision gradients
    (a handful of roundings of 2^-8 in a row)."""
    import torch
    import expert_model as M
    print("[case] expert model bf16", flush=True)
    p, tokens, targets = _case(4)
    low = {k: v.bfloat16() if k != "router" else v for k, v in p.items()}
    same = {k: v.float() for k, v in low.items()}
    _, a, ids_a = M.step(same, tokens, targets, 5)        # (all experts: the choices agree)
    _, b, ids_b = M.step(low, tokens, targets, 5)
    for k in p:
        off, size = (a[k] - b[k].float()).norm(), a[k].norm()
        assert torch.isfinite(b[k]).all() and float(off) <= 16 * 2.0 ** -8 * float(size), k


def test_example_runs():
    import numpy as np
    import expert_model as M
    print("[case] expert model example", flush=True)
    h = M.main(vocab=200, width=32, experts=4, hidden=32, batch=256, steps=5, verbose=False)
    assert len(h) == 5 and np.isfinite(h).all()
