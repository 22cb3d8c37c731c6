"""The served-output operators on the GPU against their fp64 references.

Tolerances come from the arithmetic: with eps = 2^-24, a sum of V exponentials
over at least 256 lanes is off by at most V/256 roundings plus a few for the
exponents (their argument is rounded twice, and an exponent of -d carries d
roundings); integers are exact. Outputs in 16 bits add one rounding.
"""
import numpy as np
import pytest

from oracle import serving as R

pytestmark = pytest.mark.gpu
INF = np.inf
EPS = 2.0 ** -24
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # 24, 8 and 11 significant bits
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}


def _announce(*a):
    print("[case]", *a, flush=True)


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _logits(rng, T, V, kind, pad=0, shift=0, spread=2.0):
    """A [T, V] tensor of this type in rows of V + pad elements, `shift` elements
    past an aligned start; what lies outside holds NaN."""
    import torch
    buf = torch.full((T * (V + pad) + shift,), float("nan"), dtype=_dtype(kind), device="cuda")
    x = buf[shift:].view(T, V + pad)[:, :V]
    x.copy_(torch.from_numpy((spread * rng.standard_normal((T, V))).astype(np.float32)))
    return x


def _np(x):
    return x.double().cpu().numpy()


def _close(got, want, tol, what):
    got = _np(got)
    with np.errstate(over="ignore"):           # past fp32's range the fp32 result is infinite
        want = np.where(np.isinf(np.float32(want)), np.float32(want), want).astype(np.float64)
    assert got.shape == want.shape, what
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= tol)
    assert ok.all(), (what, int((~ok).sum()), got[~ok][:4], want[~ok][:4], np.broadcast_to(tol, got.shape)[~ok][:4])


def _sum_tol(V):
    return (V / 256 + 64) * EPS


def _check_logprobs(r, x, tokens, top, it):
    l = _np(x)
    V = l.shape[1]
    o = R.token_logprobs(l, tokens, top, it)
    ts = _sum_tol(V)
    fin = np.where(np.isfinite(o["stats"]), np.abs(o["stats"]), 0.0)

    def tol(lp):
        return ts + 8 * EPS * (np.where(np.isfinite(lp), np.abs(lp), 0.0) + 1)

    _close(r.logprob, o["logprob"], tol(o["logprob"]) + 2 * EPS * fin[:, 1], "logprob")
    _close(r.stats[:, 0], o["stats"][:, 0], 0.0, "max")
    _close(r.stats[:, 1], o["stats"][:, 1], ts + 2 * EPS * fin[:, 1], "log sum")
    _close(r.entropy, o["entropy"], ts * (8 + 2 * o["spread"]), "entropy")
    assert np.array_equal(r.rank.cpu().numpy(), o["rank"]), "rank"
    if top:
        assert np.array_equal(r.top_ids.cpu().numpy(), o["top_ids"]), "top_ids"
        _close(r.top_logprobs, o["top_logprobs"], tol(o["top_logprobs"]) + 2 * EPS * fin[:, 1:], "top_logprobs")
    return o


def _tokens(tokens):
    import torch
    return torch.from_numpy(np.asarray(tokens, np.int64)).cuda()


SIZES = [(1, 1, 1), (1, 2, 2), (3, 7, 7), (5, 63, 20), (2, 64, 64), (4, 257, 33), (7, 1000, 64),
         (3, 2047, 5), (2, 4099, 0), (1, 8192, 20), (2, 8193, 1), (3, 32000, 20), (1, 128000, 64),
         (65, 513, 3), (300, 4097, 2), (1100, 1031, 4)]


@pytest.mark.parametrize("T,V,top", SIZES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_logprobs_sizes(T, V, top, kind):
    import paper_2602_10729_amd as bo
    _announce("logprobs", T, V, top, kind)
    rng = np.random.default_rng(T * 1000003 + V)
    x = _logits(rng, T, V, kind)
    tok = rng.integers(0, V, T)
    r = bo.token_logprobs(x, _tokens(tok), top=top)
    _check_logprobs(r, x, tok, top, 1.0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (7, 2), (8, 0)])
def test_logprobs_strides_and_alignment(kind, pad, shift):
    import paper_2602_10729_amd as bo
    _announce("logprobs alignment", kind, pad, shift)
    rng = np.random.default_rng(pad * 10 + shift)
    for T, V in ((4, 3), (5, 1003), (2, 9001)):
        x = _logits(rng, T, V, kind, pad, shift)
        tok = rng.integers(0, V, T)
        top = min(V, 9)
        r = bo.token_logprobs(x, _tokens(tok), top=top, inv_temperature=1 / 0.7)
        _check_logprobs(r, x, tok, top, 1 / 0.7)
        out = _logits(rng, T, V, kind, pad + 1, shift)
        _check_grad(x, tok, r, rng, 1 / 0.7, top, kind, out=out)


@pytest.mark.parametrize("V", [40, 3001, 20000])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_logprobs_masks(V, kind):
    """Rows with masks, no live logit, the lowest value, infinities and NaN."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs masks", V, kind)
    rng = np.random.default_rng(V)
    T, top = 14, 12
    x = _logits(rng, T, V, kind)
    low = torch.finfo(x.dtype).min
    cut = torch.from_numpy(rng.random(V) < 0.9).cuda()
    tok = rng.integers(0, V, T)
    x[0] = -INF                                    # nothing left
    x[1, cut] = -INF
    x[2, cut] = low
    x[3] = low                                     # uniform over the lowest value
    x[4] = -INF
    x[4, V - 1] = -7.0                             # one left, at the end
    x[5] = -INF
    x[5, 0] = low                                  # one left, the lowest value
    x[6, V // 2] = float("nan")
    x[7, V // 3] = INF
    x[8] = 0.5                                     # all equal
    x[9] = torch.arange(V, device="cuda") / (V / 16.0)     # rising
    x[10] = 0.0
    x[10, ::2] = -0.0                              # zeros of both signs are equal
    x[11, : V - 3] = -INF                          # fewer than top, at the end
    tok[4], tok[5], tok[12], tok[13] = V - 1, 1, -1, V
    for it in (1.0, 2.0):
        if it == 2.0:
            x[3] = 0.0                             # 2 * lowest leaves fp32's range
            x[5, 0] = 0.0
        r = bo.token_logprobs(x, _tokens(tok), top=top, inv_temperature=it)
        _check_logprobs(r, x, tok, top, it)
        _check_grad(x, tok, r, rng, it, top, kind)
    r = bo.token_logprobs(x, None, top=top)
    assert not r.logprob.any() and not r.rank.any()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_signalling_nans_hide_nothing(kind):
    """NaNs of every kind among the logits: never alternatives, never counted, and
    they cost no other logit its place."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs NaN kinds", kind)
    rng = np.random.default_rng(21)
    bits = {"f32": (torch.int32, [0x7F800001, 0x7FC00000, -0x7FFFFF, -1]),
            "bf16": (torch.int16, [0x7F81, 0x7FC0, -0x7F, -1]),
            "f16": (torch.int16, [0x7C01, 0x7E00, -0x3FF, -1])}[kind]
    x = _logits(rng, 4, 9000, kind)
    for r in range(4):
        at = torch.from_numpy(rng.choice(9000, 900, replace=False)).cuda()
        x[r].view(bits[0])[at] = bits[1][r]
    tok = np.array([5, 6, 7, 8])
    r = bo.token_logprobs(x, _tokens(tok), top=16)
    o = R.token_logprobs(_np(x), tok, 16)
    assert np.array_equal(r.top_ids.cpu().numpy(), o["top_ids"])
    assert np.array_equal(r.rank.cpu().numpy(), o["rank"])
    assert bool(r.entropy.isnan().all()) and bool(r.logprob.isnan().all())


def test_logprobs_far_from_zero():
    """Rows whose logits all lie far from 0, and rows whose largest comes late."""
    import paper_2602_10729_amd as bo
    _announce("logprobs offsets")
    rng = np.random.default_rng(8)
    x = _logits(rng, 6, 20011, "f32")
    for i, c in enumerate((-1000.0, 1000.0, 3e5, -3e5)):
        x[i] += c
    x[4, -1] = 60.0
    x[5, 12000] = 200.0
    tok = np.array([0, 1, 2, 3, 20010, 12000])
    r = bo.token_logprobs(x, _tokens(tok), top=5)
    _check_logprobs(r, x, tok, 5, 1.0)


def _check_grad(x, tok, r, rng, it, top, kind, out=None, use=(True, True, True)):
    import torch
    import paper_2602_10729_amd as bo
    T, V = x.shape
    gl, gh = rng.standard_normal(T), rng.standard_normal(T)
    gt = rng.standard_normal((T, top))
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    gl, gh, gt = f(gl), f(gh), f(gt)
    a = dict(grad_logprob=gl if use[0] else None, grad_entropy=gh if use[1] else None)
    ids = r.top_ids.cpu().numpy() if use[2] and top else None
    if ids is not None:
        a.update(top_ids=r.top_ids, grad_top=gt)
    l = _np(x)
    g = bo.token_logprobs_grad(x, _tokens(tok), r.stats, r.entropy, inv_temperature=it, out=out, **a)
    want = R.token_logprobs_grad(l, tok, _np(gl) if use[0] else None, _np(gh) if use[1] else None,
                                 ids, _np(gt) if ids is not None else None, it)
    o = R.token_logprobs(l, tok, 0, it)
    m, ls = o["stats"][:, :1], o["stats"][:, 1:]
    with np.errstate(invalid="ignore", over="ignore"):
        u = np.where(l > -INF, (l - m) * it - ls, -1e4)
        u = np.where(np.isfinite(u), np.maximum(u, -1e4), -1e4)
        p = np.exp(u)
    a_l = np.abs(_np(gl))[:, None] * use[0] + (np.abs(_np(gt)).sum(1, keepdims=True) if ids is not None else 0)
    a_h = np.abs(_np(gh))[:, None] * use[1]
    ent = np.where(np.isfinite(o["entropy"]), np.abs(o["entropy"]), 0)[:, None]
    ts = _sum_tol(V)
    rel = ts + 8 * EPS * (np.abs(u) + 2)
    tol = it * (p * (a_l + a_h * (np.abs(u) + ent)) * (rel + 4 * top * EPS) +
                p * a_h * ts * (8 + 2 * o["spread"][:, None]) + 4 * EPS * a_l * (p > 0.5)
                + EPS * (top + 2) * np.abs(want / it))
    tol = tol + HALF_ULP[kind] * 1.01 * (np.abs(want) + tol) + TINY[kind]
    _close(g, want, np.where(np.isfinite(tol), tol, 0.0), "grad")
    return g


@pytest.mark.parametrize("T,V,top", SIZES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_logprobs_grad_sizes(T, V, top, kind):
    import paper_2602_10729_amd as bo
    _announce("logprobs grad", T, V, top, kind)
    rng = np.random.default_rng(T * 999 + V)
    x = _logits(rng, T, V, kind)
    tok = rng.integers(-1, V, T)
    r = bo.token_logprobs(x, _tokens(tok), top=top, inv_temperature=0.5)
    _check_grad(x, tok, r, rng, 0.5, top, kind)


@pytest.mark.parametrize("use", [(True, False, False), (False, True, False), (False, False, True),
                                 (False, False, False)])
def test_logprobs_grad_parts_and_in_place(use):
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs grad parts", use)
    rng = np.random.default_rng(11)
    x = _logits(rng, 6, 9003, "bf16", pad=5)
    tok = rng.integers(0, 9003, 6)
    r = bo.token_logprobs(x, _tokens(tok), top=7)
    r.top_ids[2, 3] = r.top_ids[2, 1]              # an id given twice counts twice
    r.top_ids[3, 0] = int(tok[3])
    r.top_ids[4, 2] = 9003                         # out of range: ignored
    g = _check_grad(x, tok, r, rng, 1.0, 7, "bf16", use=use)
    gl, gh = torch.randn(6, device="cuda"), torch.randn(6, device="cuda")
    gt = torch.randn(6, 7, device="cuda")
    args = (_tokens(tok), r.stats, r.entropy, gl, gh, r.top_ids, gt)
    g = bo.token_logprobs_grad(x, *args)
    y = x.clone()
    bo.token_logprobs_grad(y, *args, out=y)
    assert torch.equal(y, g)


def test_logprobs_gradient_against_differences():
    """The GPU's gradient against central differences of the fp64 definition."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs differences")
    rng = np.random.default_rng(12)
    x = _logits(rng, 3, 50, "f32")
    tok = np.array([4, 49, 0])
    r = bo.token_logprobs(x, _tokens(tok), top=3, inv_temperature=0.5)
    gl, gh, gt = rng.standard_normal(3), rng.standard_normal(3), rng.standard_normal((3, 3))
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    g = _np(bo.token_logprobs_grad(x, _tokens(tok), r.stats, r.entropy, f(gl), f(gh), r.top_ids, f(gt), 0.5))
    ids, l = r.top_ids.cpu().numpy(), _np(x)

    def total(a):
        o = R.token_logprobs(a, tok, 0, 0.5)
        v = gl * o["logprob"] + gh * o["entropy"]
        return v + sum(gt[:, i] * R.token_logprobs(a, ids[:, i], 0, 0.5)["logprob"] for i in range(3))

    for j in range(50):
        a, b = l.copy(), l.copy()
        a[:, j] += 1e-5
        b[:, j] -= 1e-5
        assert np.abs((total(a) - total(b)) / 2e-5 - g[:, j]).max() < 2e-5


def test_logprobs_past_32_bit_offsets():
    """Rows that start past 2^31 elements (and 2^32 bytes)."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs offsets past 32 bits")
    T, V = 17001, 128003
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.empty((T, V), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    tok = torch.randint(V, (T,), generator=g, device="cuda")
    r = bo.token_logprobs(x, tok, top=3)
    last = slice(T - 3, T)
    part = bo.TokenLogprobs(*(t[last] for t in r))
    _check_logprobs(part, x[last], tok[last].cpu().numpy(), 3, 1.0)
    gl = torch.ones(T, device="cuda")
    grad = bo.token_logprobs_grad(x, tok, r.stats, r.entropy, gl, out=x.clone())
    alone = bo.token_logprobs_grad(x[last], tok[last], r.stats[last].contiguous(),
                                   r.entropy[last].contiguous(), gl[last].contiguous())
    assert torch.equal(grad[last], alone)


@pytest.mark.parametrize("kind,T,V,pad,shift", [("f16", 2051, 50021, 3, 1), ("bf16", 2300, 40001, 0, 5),
                                                ("f32", 2100, 20003, 1, 3), ("f32", 4100, 100003, 2, 1)])
def test_logprobs_past_the_caches(kind, T, V, pad, shift):
    """Logits and gradients too large for the caches give the bits of the same
    rows in smaller calls, whatever their stride and alignment."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs past the caches", kind, T, V, pad, shift)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    buf = torch.full((T * (V + pad) + shift,), float("nan"), dtype=_dtype(kind), device="cuda")
    x = buf[shift:].view(T, V + pad)[:, :V]
    x.copy_(torch.randn((T, V), generator=g, device="cuda"))
    tok = torch.randint(V, (T,), generator=g, device="cuda")
    gl = torch.randn(T, generator=g, device="cuda")
    # whole rows a workgroup in both (below 1024 rows they are split otherwise)
    r = bo.token_logprobs(x, tok, top=3)
    for a in (0, T - 1024):
        b = slice(a, a + 1024)
        part = bo.token_logprobs(x[b], tok[b], top=3)
        assert all(torch.equal(u[b], v) for u, v in zip(r, part))
    out = torch.full((T * (V + 1) + 1,), 7.0, dtype=x.dtype, device="cuda")
    grad = bo.token_logprobs_grad(x, tok, r.stats, r.entropy, gl, gl, out=out[1:].view(T, V + 1)[:, :V])
    assert bool((out[1:].view(T, V + 1)[:, V] == 7.0).all()) and float(out[0]) == 7.0
    for a in range(0, T, 512):
        b = slice(a, min(a + 512, T))
        part = bo.token_logprobs_grad(x[b], tok[b], r.stats[b], r.entropy[b], gl[b], gl[b])
        assert torch.equal(grad[b], part)


# ---- routing -----------------------------------------------------------------

ROUTES = [  # T, E, top, groups, top_groups, group_best
    (1, 1, 1, 1, 1, 1), (3, 2, 1, 1, 1, 1), (9, 3, 2, 1, 1, 1), (17, 8, 2, 1, 1, 1),
    (64, 64, 6, 1, 1, 1), (33, 61, 4, 1, 1, 1), (5, 64, 32, 1, 1, 1), (130, 256, 8, 8, 4, 2),
    (65, 256, 8, 8, 4, 1), (31, 160, 6, 8, 3, 2), (12, 96, 5, 12, 5, 1), (7, 60, 3, 20, 7, 2),
    (3, 1024, 32, 1, 1, 1), (6, 1023, 10, 33, 4, 2), (4, 1024, 8, 512, 40, 2), (19, 384, 16, 16, 16, 1),
    (1001, 128, 8, 1, 1, 1), (2049, 16, 4, 4, 2, 2), (5000, 3, 1, 1, 1, 1)]


def _route_case(rng, T, E, kind, biased, score, top, groups, top_groups, group_best, pad=0, shift=0,
                masked=True):
    """Logits and bias whose choices do not hang on the last bits: rows with a
    gap under 1e-5 of the largest value (a hundred roundings) are replaced."""
    import torch
    x = _logits(rng, T, E, kind, pad, shift, spread=1.0)
    bias = None
    if biased:
        bias = ((0.05 if score == "sigmoid" else 0.25 / E) * rng.standard_normal(E)).astype(np.float32)
        if masked and E > 4:
            bias[E // 3] = -INF
    if masked:
        cut = torch.from_numpy(rng.random((T, E)) < 0.4).cuda()
        cut[::2] = False
        x[cut] = -INF
    how = dict(bias=bias, score=score, groups=groups, top_groups=top_groups, group_best=group_best)
    for _ in range(40):
        bad = R.route(_np(x), top, **how)["gap"] < 1e-5
        if not bad.any():
            break
        n = int(bad.sum())
        x[torch.from_numpy(bad).cuda()] = torch.from_numpy(rng.standard_normal((n, E)).astype(np.float32)).cuda().to(x.dtype)
    assert not bad.any()
    if masked and T > 2:
        x[T // 2] = -INF
    return x, bias, how


def _check_route(x, bias, how, top, renorm, scale):
    import torch
    import paper_2602_10729_amd as bo
    l = _np(x)
    b = None if bias is None else torch.from_numpy(bias).cuda()
    r = bo.route(x, top, **{**how, "bias": b}, renormalise=renorm, scale=scale)
    o = R.route(l, top, **how, renormalise=renorm, scale=scale)
    assert np.array_equal(r.ids.cpu().numpy(), o["ids"]), "ids"
    with np.errstate(invalid="ignore"):
        size = np.where(np.isfinite(l), np.abs(l), 0).max(1, keepdims=True)
    rel = (2 * size + l.shape[1] / 8 + 32) * 2 * EPS
    _close(r.weights, o["weights"], rel * np.abs(o["weights"]) + 1e-37, "weights")
    return r, o, rel


def _check_route_grad(x, r, rel, rng, score, renorm, scale, kind, out=None):
    import torch
    import paper_2602_10729_amd as bo
    g = torch.from_numpy(rng.standard_normal(tuple(r.ids.shape)).astype(np.float32)).cuda()
    got = bo.route_grad(x, r.ids, g, score=score, renormalise=renorm, scale=scale, out=out)
    ids, l = r.ids.cpu().numpy(), _np(x)
    want = R.route_grad(l, ids, _np(g), score, renorm, scale)
    big = R.route_grad(l, ids, np.zeros(ids.shape), score, renorm, scale)   # shape only
    w = R.route_weights(l, ids, score, renorm, scale)
    gmax = np.abs(_np(g)).max(1, keepdims=True) * (1 + np.abs(w / scale).sum(1, keepdims=True))
    size = np.zeros_like(big)
    for i in range(l.shape[0]):
        on = ids[i] >= 0
        size[i, ids[i][on]] = np.abs(w[i][on])
        if on.any() and score == "softmax" and not renorm:
            size[i] = np.maximum(size[i], abs(scale) * R._scores(l[i], "softmax"))
    tol = 4 * rel * gmax * size
    tol = tol + HALF_ULP[kind] * 1.01 * (np.abs(want) + tol) + TINY[kind]
    _close(got, want, tol, "route grad")
    return got, g


@pytest.mark.parametrize("T,E,top,groups,top_groups,group_best", ROUTES)
@pytest.mark.parametrize("kind,score,biased,renorm", [
    ("f32", "softmax", False, True), ("bf16", "sigmoid", True, True), ("f16", "softmax", True, False),
    ("bf16", "softmax", False, False), ("f32", "sigmoid", False, False)])
def test_route(T, E, top, groups, top_groups, group_best, kind, score, biased, renorm):
    _announce("route", T, E, top, groups, top_groups, group_best, kind, score, biased, renorm)
    rng = np.random.default_rng(E * 131 + T)
    x, bias, how = _route_case(rng, T, E, kind, biased, score, top, groups, top_groups, group_best)
    r, o, rel = _check_route(x, bias, how, top, renorm, 2.5)
    _check_route_grad(x, r, rel, rng, score, renorm, 2.5, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("E,pad,shift", [(64, 0, 1), (64, 3, 0), (61, 2, 3), (256, 8, 0), (7, 1, 1), (256, 1, 5)])
def test_route_strides_and_alignment(kind, E, pad, shift):
    import torch
    import paper_2602_10729_amd as bo
    _announce("route alignment", kind, E, pad, shift)
    rng = np.random.default_rng(E + pad)
    x, bias, how = _route_case(rng, 37, E, kind, True, "softmax", 4, 1, 1, 1, pad, shift)
    r, o, rel = _check_route(x, bias, how, 4, True, 1.0)
    out = _logits(rng, 37, E, kind, pad + 2, shift)
    got, g = _check_route_grad(x, r, rel, rng, "softmax", False, 1.0, kind, out=out)
    y = x.clone()
    bo.route_grad(y, r.ids, g, renormalise=False, out=y)
    assert torch.equal(y, got)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_ties_and_special_values(score):
    """Exact ties go to the lowest index; NaN and infinities; far logits."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("route ties", score)
    rng = np.random.default_rng(2)
    E, top = 70, 8
    x = _logits(rng, 12, E, "f32", spread=1.0)
    x[0] = 1.0
    x[1, ::3] = 2.0
    x[2] = 0.0
    x[2, ::2] = -0.0
    x[3, 7] = float("nan")
    x[4, 9] = INF
    x[5] = -INF
    x[5, 60] = -200.0                              # one left, its score underflows
    x[6] = -300.0
    x[6, 11] = -299.0                              # renormalised exactly all the same
    x[7] = torch.finfo(torch.float32).min
    x[8, :66] = -INF                               # fewer than top
    x[9] = torch.from_numpy(np.round(2 * rng.standard_normal(E)).astype(np.float32))
    for groups, tg in ((1, 1), (7, 3)):
        for biased in (False, True):
            bias = np.zeros(E, np.float32) if biased else None
            rows = [0, 1, 2, 3, 4, 5, 8, 9] if biased or groups > 1 else list(range(12))
            y = x[rows].contiguous()
            how = dict(bias=bias, score=score, groups=groups, top_groups=tg, group_best=1)
            for renorm in (True, False):
                b = None if bias is None else torch.from_numpy(bias).cuda()
                r = bo.route(y, top, **{**how, "bias": b}, renormalise=renorm)
                l = _np(y)
                o = R.route(l, top, **how, renormalise=renorm)
                assert np.array_equal(r.ids.cpu().numpy(), o["ids"]), (groups, biased)
                size = np.minimum(np.where(np.isfinite(l), np.abs(l), 0).max(1, keepdims=True), 400.0)
                _close(r.weights, o["weights"],
                       (2 * size + E / 8 + 32) * 2 * EPS * np.abs(o["weights"]) + 1e-37, "weights")


def test_route_many_rows():
    """More rows than one sweep of the grid; offsets past 2^31 bytes."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("route many rows")
    T, E = 9_000_017, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.empty((T, E), device="cuda").normal_(generator=g)
    r = bo.route(x, 2)
    for sl in (slice(0, 50), slice(T - 50, T)):
        o = R.route(_np(x[sl]), 2)
        assert np.array_equal(r.ids[sl].cpu().numpy(), o["ids"])
    gw = torch.randn((T, 2), generator=g, device="cuda")
    grad = bo.route_grad(x, r.ids, gw)
    last = slice(T - 100, T)
    assert torch.equal(grad[last], bo.route_grad(x[last], r.ids[last].contiguous(), gw[last].contiguous()))
    d = bo.dispatch(r.ids, E)
    assert int(d.offsets[-1]) == 2 * T
    assert torch.equal(d.load.long(), torch.bincount(r.ids.view(-1).long(), minlength=E))
    pos = d.position.view(-1).long()
    assert torch.equal(d.order[pos].long(), torch.arange(2 * T, device="cuda"))
    key = r.ids.view(-1).long()[d.order.long()] * (2 * T) + d.order.long()
    assert bool((key[1:] > key[:-1]).all())


@pytest.mark.parametrize("biased", [False, True])
def test_route_groups_of_one(biased):
    """Groups of one expert each, over enough rows that a lane holds 32 experts."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("route groups of one", biased)
    T, E, top = 150_001, 64, 4
    rng = np.random.default_rng(5)
    few, bias, how = _route_case(rng, 300, E, "f32", biased, "sigmoid", top, E, 6, 1)
    x = few.repeat(501, 1)[:T].contiguous()
    b = None if bias is None else torch.from_numpy(bias).cuda()
    r = bo.route(x, top, **{**how, "bias": b})
    o = R.route(_np(few), top, **how)
    want = torch.from_numpy(o["ids"]).cuda().repeat(501, 1)[:T]
    assert torch.equal(r.ids.long(), want.long())
    _check_route(few, bias, how, top, True, 1.0)


# ---- dispatch ------------------------------------------------------------------

@pytest.mark.parametrize("N,E", [(0, 5), (1, 1), (1, 8), (63, 3), (64, 64), (65, 7), (2048, 256),
                                 (2049, 256), (5000, 2), (10007, 61), (40000, 1024), (100003, 256)])
@pytest.mark.parametrize("capacity", [0, 3, 200])
def test_dispatch(N, E, capacity):
    import torch
    import paper_2602_10729_amd as bo
    _announce("dispatch", N, E, capacity)
    rng = np.random.default_rng(N + E)
    ids = np.minimum((E + 1) * rng.random(N) ** 2, E).astype(np.int32) - 1
    if N > 10:
        ids[3], ids[5], ids[6] = E, 2 ** 31 - 1, -2 ** 31   # outside: nowhere
    d = bo.dispatch(torch.from_numpy(ids).cuda(), E, capacity=capacity)
    o = R.dispatch(ids, E, capacity)
    for name in ("load", "offsets", "order", "position"):
        assert np.array_equal(getattr(d, name).cpu().numpy(), o[name]), name


def test_dispatch_most_experts_full_tiles():
    """All experts and the largest tile, a ragged last one: the most shared memory."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("dispatch most experts")
    N, E = 1_500_007, 1024
    ids = np.random.default_rng(8).integers(-1, E + 1, N).astype(np.int32)
    d = bo.dispatch(torch.from_numpy(ids).cuda(), E, capacity=1400)
    o = R.dispatch(ids, E, 1400)
    for name in ("load", "offsets", "order", "position"):
        assert np.array_equal(getattr(d, name).cpu().numpy(), o[name]), name


def test_dispatch_one_expert_takes_all():
    import torch
    import paper_2602_10729_amd as bo
    _announce("dispatch one expert")
    N = 300_001
    d = bo.dispatch(torch.full((N,), 5, dtype=torch.int32, device="cuda"), 9)
    assert torch.equal(d.order.long(), torch.arange(N, device="cuda"))
    assert d.load.tolist() == [0, 0, 0, 0, 0, N, 0, 0, 0]
    d = bo.dispatch(torch.full((N,), -1, dtype=torch.int32, device="cuda"), 9)
    assert bool((d.order == -1).all()) and bool((d.position == -1).all()) and int(d.offsets[-1]) == 0


# ---- how they are called ---------------------------------------------------------

def _all_calls(bo, x, tok, rl, stream=None):
    r = bo.token_logprobs(x, tok, top=5, stream=stream)
    g = bo.token_logprobs_grad(x, tok, r.stats, r.entropy, r.logprob, r.entropy, r.top_ids,
                               r.top_logprobs, stream=stream)
    w = bo.route(rl, 3, stream=stream)
    h = bo.route_grad(rl, w.ids, w.weights, renormalise=False, stream=stream)
    d = bo.dispatch(w.ids, rl.shape[1], stream=stream)
    return [*r, g, *w, h, *d]


@pytest.mark.parametrize("T,V", [(2, 50000), (700, 3001)])
def test_other_streams_give_the_same_bits(T, V):
    import torch
    import paper_2602_10729_amd as bo
    _announce("streams", T, V)
    rng = np.random.default_rng(5)
    sets = [(_logits(rng, T, V, "bf16"), _tokens(rng.integers(0, V, T)), _logits(rng, 5 * T, 48, "f32"))
            for _ in range(2)]
    want = [_all_calls(bo, *s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(3):
        for s, st in zip(sets, streams):
            st.wait_stream(torch.cuda.current_stream())
            got.append(_all_calls(bo, *s, stream=st))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))


@pytest.mark.parametrize("T,V", [(1, 40000), (300, 2000)])
def test_graph_replays(T, V):
    """Every call captured; replays with new inputs, with eager work between."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("graph", T, V)
    rng = np.random.default_rng(6)
    new = lambda: (_logits(rng, T, V, "bf16"), _tokens(rng.integers(0, V, T)), _logits(rng, 3 * T, 48, "f32"))
    cur = new()
    _all_calls(bo, *cur)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _all_calls(bo, *cur)
    for _ in range(4):
        nxt = new()
        for a, b in zip(cur, nxt):
            a.copy_(b)
        want = _all_calls(bo, *nxt)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_out_is_written_and_empty_batches():
    import torch
    import paper_2602_10729_amd as bo
    _announce("out")
    rng = np.random.default_rng(7)
    x, tok = _logits(rng, 4, 900, "f16"), _tokens(rng.integers(0, 900, 4))
    r = bo.token_logprobs(x, tok, top=2)
    s = bo.TokenLogprobs(*(torch.zeros_like(t) for t in r))
    assert bo.token_logprobs(x, tok, top=2, out=s) is s
    assert all(torch.equal(a, b) for a, b in zip(r, s))
    w = bo.route(x, 3)
    v = bo.Routing(torch.zeros_like(w.ids), torch.zeros_like(w.weights))
    bo.route(x, 3, out=v)
    assert torch.equal(w.ids, v.ids) and torch.equal(w.weights, v.weights)
    d = bo.dispatch(w.ids, 900)
    e = bo.Dispatch(*(torch.zeros_like(t) for t in d))
    bo.dispatch(w.ids, 900, out=e)
    assert all(torch.equal(a, b) for a, b in zip(d, e))
    none = bo.token_logprobs(x[:0], tok[:0], top=2)
    assert none.top_ids.shape == (0, 2)
    assert bo.token_logprobs_grad(x[:0], tok[:0], none.stats, none.entropy).shape == (0, 900)
    assert bo.route_grad(x[:0], bo.route(x[:0], 3).ids, w.weights[:0]).shape == (0, 900)


def test_refusals_on_the_device():
    import torch
    import paper_2602_10729_amd as bo
    _announce("refusals")
    x = torch.zeros((4, 100), device="cuda")
    tok = torch.zeros(4, dtype=torch.int64, device="cuda")
    r = bo.token_logprobs(x, tok)
    bad = [
        lambda: bo.token_logprobs(x.double(), tok), lambda: bo.token_logprobs(x[:, ::2], tok),
        lambda: bo.token_logprobs(x[:1].expand(4, 100), tok), lambda: bo.token_logprobs(x, tok.int()),
        lambda: bo.token_logprobs(x, tok[:3]), lambda: bo.token_logprobs(x, tok, top=101),
        lambda: bo.token_logprobs(x, tok, top=65), lambda: bo.token_logprobs(x, tok, top=-1),
        lambda: bo.token_logprobs(x, tok, inv_temperature=0.0),
        lambda: bo.token_logprobs(x, tok, inv_temperature=float("nan")),
        lambda: bo.token_logprobs(x.cpu(), tok), lambda: bo.token_logprobs(x, tok.cpu()),
        lambda: bo.token_logprobs(x, tok, out=tuple(torch.zeros(4, device="cuda") for _ in range(6))),
        lambda: bo.token_logprobs_grad(x, tok, r.stats[:, :1], r.entropy),
        lambda: bo.token_logprobs_grad(x, tok, r.stats, r.entropy, top_ids=r.top_ids),
        lambda: bo.token_logprobs_grad(x, tok, r.stats, r.entropy, out=x.half()),
        lambda: bo.token_logprobs_grad(x[:3], tok[:3], r.stats[:3], r.entropy[:3], out=x[1:]),
        lambda: bo.route(x, 0), lambda: bo.route(x, 33), lambda: bo.route(x, 2, groups=3),
        lambda: bo.route(x, 2, groups=4, top_groups=5), lambda: bo.route(x, 30, groups=4, top_groups=1),
        lambda: bo.route(x, 2, score="relu"), lambda: bo.route(x, 2, scale=float("inf")),
        lambda: bo.route(x, 2, groups=100, top_groups=2, group_best=2),
        lambda: bo.route(x, 2, bias=torch.zeros(99, device="cuda")),
        lambda: bo.route(torch.zeros((2, 1025), device="cuda"), 2),
        lambda: bo.route_grad(x, torch.zeros((4, 2), device="cuda"), torch.zeros((4, 2), device="cuda")),
        lambda: bo.dispatch(torch.zeros(4, device="cuda"), 3),
        lambda: bo.dispatch(torch.zeros(4, dtype=torch.int32, device="cuda"), 0),
        lambda: bo.dispatch(torch.zeros(4, dtype=torch.int32, device="cuda"), 1025),
        lambda: bo.dispatch(torch.zeros(4, dtype=torch.int32, device="cuda"), 3, capacity=-1),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((bo.BoError, ValueError, TypeError)):
            f()
            print("accepted", i, flush=True)
    torch.cuda.synchronize()
