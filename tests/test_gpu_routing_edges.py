"""Routing and dispatch in the forms that only large calls take, and beside NaN,
against the fp64 reference. Tolerances are those of the other served-output
tests (see there).
"""
import numpy as np
import pytest

from oracle import serving as R
from test_gpu_serving import EPS, HALF_ULP, TINY, _announce, _close, _logits, _np, _route_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [16500, 33000])          # a lane holds two and four eights
@pytest.mark.parametrize("kind,score,biased,groups,top_groups,group_best", [
    ("bf16", "sigmoid", True, 8, 4, 2), ("f32", "softmax", False, 8, 3, 1), ("f16", "softmax", True, 4, 2, 2),
    ("f32", "sigmoid", False, 32, 9, 2)])
def test_route_groups_over_many_rows(T, kind, score, biased, groups, top_groups, group_best):
    """Groups of whole eights in calls with enough rows that a lane holds several
    eights: every row gives what the reference gives."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("route groups, many rows", T, kind, score, biased, groups)
    rng = np.random.default_rng(T + groups)
    E, top, few = 256, 8, 300
    x, bias, how = _route_case(rng, few, E, kind, biased, score, top, groups, top_groups, group_best)
    tile = lambda a: np.tile(a, (-(-T // few), 1))[:T]
    on_gpu = lambda a: torch.from_numpy(tile(a)).cuda()
    y = x.repeat(-(-T // few), 1)[:T].contiguous()
    l = _np(x)
    size = np.where(np.isfinite(l), np.abs(l), 0).max(1, keepdims=True)
    rel = (2 * size + E / 8 + 32) * 2 * EPS
    g = rng.standard_normal((few, top)).astype(np.float32)
    for renorm in (True, False):
        r = bo.route(y, top, **{**how, "bias": None if bias is None else torch.from_numpy(bias).cuda()},
                     renormalise=renorm, scale=2.5)
        o = R.route(l, top, **how, renormalise=renorm, scale=2.5)
        ids, w = o["ids"], np.abs(o["weights"])
        assert torch.equal(r.ids.long(), on_gpu(ids))
        _close(r.weights, tile(o["weights"]), tile(rel * w + 1e-37), "weights")
        grad = bo.route_grad(y, r.ids, on_gpu(g), score=score, renormalise=renorm, scale=2.5)
        want = R.route_grad(l, ids, g, score, renorm, 2.5)
        most = np.zeros((few, E))                      # the weight behind each element of the gradient
        for i in range(few):
            on = ids[i] >= 0
            if on.any() and score == "softmax" and not renorm:
                most[i] = 2.5 * R._scores(l[i], "softmax")
            most[i, ids[i][on]] = np.maximum(most[i, ids[i][on]], w[i][on])
        tol = 4 * rel * most * np.abs(g).max(1, keepdims=True) * (1 + w.sum(1, keepdims=True) / 2.5)
        tol = tol + HALF_ULP[kind] * 1.01 * (np.abs(want) + tol) + TINY[kind]
        _close(grad, tile(want), tile(tol), "grad")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("how", [dict(), dict(groups=4, top_groups=2), dict(groups=16, top_groups=5, group_best=2)])
def test_routing_chooses_no_nan(kind, score, how):
    """NaNs of every kind among a router's logits: an expert with one is never
    chosen, with and without a bias."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("routing and NaN", kind, score, how)
    rng = np.random.default_rng(41)
    word, bits = {"f32": (torch.int32, [0x7F800001, 0x7FC00000, -0x7FFFFF, -1]),
                  "bf16": (torch.int16, [0x7F81, 0x7FC0, -0x7F, -1]),
                  "f16": (torch.int16, [0x7C01, 0x7E00, -0x3FF, -1])}[kind]
    T, E, top = 64, 64, 6
    # well apart, so that no rounding decides the order
    x = _logits(rng, T, E, kind)
    x.copy_(torch.from_numpy(rng.permuted(np.tile(np.linspace(-4, 4, E), (T, 1)), axis=1).astype(np.float32)))
    for t in range(T - 4):                             # (the last rows hold none)
        at = torch.from_numpy(rng.choice(E, 9, replace=False)).cuda()
        x[t].view(word)[at] = bits[t % 4]
    for bias in (None, np.zeros(E, np.float32)):
        for renorm in (True, False):
            r = bo.route(x, top, score=score, renormalise=renorm, **how,
                         bias=None if bias is None else torch.from_numpy(bias).cuda())
            o = R.route(_np(x), top, score=score, renormalise=renorm, bias=bias, **how)
            assert np.array_equal(r.ids.cpu().numpy(), o["ids"])
            _close(r.weights, o["weights"], 64 * EPS * np.abs(o["weights"]), "weights")


@pytest.mark.parametrize("N,E,capacity", [(300_007, 100, 0), (300_007, 100, 2500), (700_001, 256, 0), (700_001, 3, 90_000),
                                          (2 ** 21 + 4097, 64, 20_000), (2 ** 21 + 4097, 1024, 0)])
def test_dispatch_in_every_width(N, E, capacity):
    """Two, four and eight pairs a lane, one and several tiles a block, with
    capacities that run out in the middle of a block."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("dispatch widths", N, E, capacity)
    ids = np.random.default_rng(N + E).integers(-1, E + 1, N).astype(np.int32)
    d = bo.dispatch(torch.from_numpy(ids).cuda(), E, capacity=capacity)
    o = R.dispatch(ids, E, capacity)
    for name in ("load", "offsets", "order", "position"):
        assert np.array_equal(getattr(d, name).cpu().numpy(), o[name]), name
