"""Log probabilities from hidden rows and their gradients where values, sizes and
arguments are at their limits, on the GPU against the definitions in 64 bits.

Inputs are drawn on the CPU, so that what a test needs of them (a clear largest
logit, say) holds on every device. Roundings are counted as in test_gpu_linear: eps =
2^-24 for fp32 sums, n additions within (2 sqrt(n) + 4) eps of the sum of the terms'
sizes; d once to a 16-bit type (twice, so squared, up to 128 rows), outputs once.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
INF = np.inf
EPS = 2.0 ** -24
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-36, "bf16": 1e-36, "f16": 2.0 ** -24}
KINDS = ["f32", "bf16", "f16"]


def _announce(*a):
    print("[case]", *a, flush=True)


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _gen(seed):
    import torch
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _close(got, want, tol, what):
    import torch
    half = got.dtype is torch.float16
    got = got.double()
    assert got.shape == want.shape, what
    ok = (got == want) | (got.isnan() & want.isnan()) | ((got - want).abs() <= tol)
    if half:                       # from 65520 on, the nearest f16 is infinity
        ok |= got.isinf() & (got.sign() == want.sign()) & (want.abs() + tol >= 65520.0)
    if not bool(ok.all()):
        bad = ~ok
        raise AssertionError((what, int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist(),
                              tol.expand_as(want)[bad][:4].tolist(), bad.nonzero()[:4].tolist()))


def _product_check(got, d, other, kind, T, what, extra=None):
    """got = d @ other: d off by a relative step of its own and `extra`, the sum and
    the output by their roundings."""
    n = d.shape[1]
    own = 16 * EPS + (0.0 if kind == "f32" else HALF_ULP[kind] ** (2 if T <= 128 else 1) * 1.01)
    ref = d @ other
    tol = (own + (2 * n ** 0.5 + 4) * EPS) * (d.abs() @ other.abs())
    if extra is not None:
        tol = tol + extra @ other.abs()
    _close(got, ref, tol + HALF_ULP[kind] * 1.01 * (ref.abs() + tol) + TINY[kind], what)


def clear_rows(T, V, H, kind, seed, masked=0):
    """(hidden, weight, tokens, favourites) with logits that are whole numbers, exact
    in any order of summation: every row's largest is its favourite's, alone. The last
    `masked` words have logits of -inf; column 0 is what masks."""
    import torch
    g = _gen(seed)
    n = V - masked
    w = torch.randint(-1, 2, (V, H), generator=g).double()
    w[:, 0] = 0.0
    w[:, 1] = 1.0
    fav = torch.randint(n, (T,), generator=g)
    h = 2.0 * w[fav]
    h[:, 0] = 1.0
    x = h @ w[:n].T
    best = x.topk(2, 1)
    assert bool((best.values[:, 0] >= best.values[:, 1] + 1).all()) and bool((best.indices[:, 0] == fav).all())
    w[n:, 0] = -INF
    tok = torch.randint(n, (T,), generator=g)
    return h.to(_dtype(kind)), w.to(_dtype(kind)), tok, fav


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("it,masked", [(1e9, 30), (1e20, 0), (1e20, 30)])
def test_entropy_gradients_of_words_without_probability(T, kind, it, masked):
    """Far logits under a large inverse temperature: the largest has probability 1,
    all others 0, and words of probability 0 have no part in the entropy's gradient,
    however large it is (0 times what passes fp32 is no number)."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear no probability", T, kind, it, masked)
    V, H = 700, 40
    h, w, tok, fav = (t.cuda() for t in clear_rows(T, V, H, kind, 5, masked))
    it = float(np.float32(it))
    r = bo.linear_logprobs(h, w, tok, inv_temperature=it)
    assert not r.entropy.any() and not r.stats[:, 1].any()
    g, gh = torch.randn(T, generator=_gen(6)).cuda() / it, torch.ones(T, device="cuda")
    got = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, g, gh, inv_temperature=it)
    d = torch.zeros((T, V), dtype=torch.float64, device="cuda")
    rows = torch.arange(T, device="cuda")
    d[rows, tok] += it * g.double()
    d[rows, fav] -= it * g.double()
    # (f16: a step of 2^-38 of what a gradient may be, log V + 1 times the entropy's)
    extra = torch.full_like(d, 2.0 ** -38 * it * float((np.log(V) + 1) * gh[0] + g.abs().max()) if kind == "f16" else 0.0)
    first, n = (1, V - masked) if masked else (0, V)
    if masked:
        assert bool(got.hidden[:, 0].isnan().all()) and not got.weight[n:].any()
    kept = w.double()
    kept[:, 0] = 0.0
    _product_check(got.hidden[:, first:], d, kept[:, first:], kind, T, "grad hidden", extra)
    _product_check(got.weight[:n], d.T[:n], h.double(), kind, T, "grad weight", extra.T[:n])


def test_most_tokens():
    """As many tokens as are taken, 2^28: every launch of the call fits its limits."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear most tokens")
    T, V, H = 2 ** 28, 4, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    h = torch.empty((T, H), dtype=torch.float16, device="cuda").normal_(generator=g)
    w = torch.randn((V, H), generator=g, device="cuda").half()
    tok = torch.randint(-1, V, (T,), generator=g, device="cuda")
    r = bo.linear_logprobs(h, w, tok)
    torch.cuda.synchronize()
    for a in range(0, T, 2 ** 24):
        s = slice(a, a + 2 ** 24)
        x = h[s].double() @ w.double().T
        lsm = torch.log_softmax(x, 1)
        has = tok[s] >= 0
        lp = torch.where(has, lsm.gather(1, tok[s].clamp(min=0)[:, None])[:, 0], 0.0)
        m = x.amax(1)
        # the bounds of test_gpu_linear at H = 2 (a logit within 7 eps of its products'
        # sizes) and V = 4 (a sum within 65 eps, an entropy of at most 1.4)
        size = (h[s].double().abs() @ w.double().abs().T).amax(1)
        _close(r.logprob[s], lp, EPS * (28 * size + 80 + 8 * lp.abs()), "logprob")
        _close(r.entropy[s], -(lsm.exp() * lsm).sum(1), EPS * (40 * size + 704), "entropy")
        _close(r.stats[s, 0], m, EPS * 8 * size, "max")
        _close(r.stats[s, 1], torch.logsumexp(x, 1) - m, EPS * (21 * size + 80), "log sum")


def test_outputs_that_share_memory_are_refused():
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear overlaps")
    T, V, H = 8, 100, 16
    g = _gen(14)
    h, w = torch.randn((T, H), generator=g).cuda(), torch.randn((V, H), generator=g).cuda()
    tok = torch.randint(V, (T,), generator=g).cuda()
    r = bo.linear_logprobs(h, w, tok)
    lp, en, st = (torch.empty_like(t) for t in r)
    gl, gh = torch.ones(T, device="cuda"), torch.ones(T, device="cuda")
    words = tok.view(torch.float32)                  # the tokens' memory
    grad = lambda out: bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh, out=out)
    row = lambda t: t.view(T, 1)                     # a gradient of one column in a vector's place
    h1, w1 = h[:, :1].contiguous(), w[:, :1].contiguous()
    narrow = lambda out: bo.linear_logprobs_grad(h1, w1, tok, r.stats, r.entropy, gl, gh, out=out)
    big = torch.empty(3 * T, device="cuda")
    bad = [
        lambda: bo.linear_logprobs(h, w, tok, out=(lp, lp, st)), lambda: bo.linear_logprobs(h, w, tok, out=(big[4:12], big[:8], st)),
        lambda: bo.linear_logprobs(h, w, tok, out=(lp, big[:8], big[4:20].view(T, 2))),
        lambda: bo.linear_logprobs(h, w, tok, out=(h.view(-1)[:T], en, st)), lambda: bo.linear_logprobs(h, w, tok, out=(lp, w[1, :8], st)),
        lambda: bo.linear_logprobs(h, w, tok, out=(words[:T], en, st)), lambda: bo.linear_logprobs(h, w, tok, out=(lp, en, words.view(T, 2))),
        lambda: narrow((row(gl), None)), lambda: narrow((row(gh), None)), lambda: narrow((row(r.entropy), None)),
        lambda: narrow((r.stats[:, :1], None)), lambda: narrow((words[:T].view(T, 1), None)),
    ]
    keep = [t.clone() for t in (h, w, tok, *r, gl, gh)]
    for i, f in enumerate(bad):
        with pytest.raises(bo.BoError, match="overlap"):
            f()
            print("accepted", i, flush=True)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(keep, (h, w, tok, *r, gl, gh)))
    # side by side, and vectors in the columns that a matrix leaves, share nothing
    out = bo.linear_logprobs(h, w, tok, out=(big[:8], big[8:16], torch.empty_like(st)))
    assert all(torch.equal(a, b) for a, b in zip(out, r))
    wide = torch.zeros((V, H + 8), device="cuda")
    wide[:, :H] = w
    out = bo.linear_logprobs(h, wide[:, :H], tok, out=(wide[3, H:], wide[4, H:], st))
    assert all(torch.equal(a, b) for a, b in zip(out, r)) and torch.equal(wide[:, :H], w)
    both = torch.empty((T, 2 * H), device="cuda")
    both[:, :H] = h
    g1 = bo.linear_logprobs_grad(both[:, :H], w, tok, r.stats, r.entropy, gl, gh, out=(both[:, H:], torch.empty_like(w)))
    g2 = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    assert torch.equal(g1[0], g2.hidden) and torch.equal(g1[1], g2.weight)


@pytest.mark.parametrize("T", [45, 600])
@pytest.mark.parametrize("outlier", [False, True])
def test_small_rows_beside_large_ones_in_half_precision(T, outlier):
    """A row's hidden gradient is as exact beside rows whose gradients are 2^28 times
    its own, or infinite, as by itself."""
    import torch
    import paper_2602_10729_amd as bo
    from test_gpu_linear import Reference
    _announce("linear f16 rows", T, outlier)
    V, H = 3000, 64
    g = _gen(12)
    w = (0.25 * torch.randn((V, H), generator=g)).half().cuda()
    h = torch.randn((T, H), generator=g).half().cuda()
    tok = torch.randint(V, (T,), generator=g).cuda()
    gl, gh = torch.randn(T, generator=g).cuda(), (0.3 * torch.randn(T, generator=g)).cuda()
    groups = [(torch.arange(i, T, 3, device="cuda"), s) for i, s in enumerate((2.0 ** 14, 2.0 ** -2, 2.0 ** -14))]
    for rows, s in groups:
        gl[rows] *= s
        gh[rows] *= s
    r = bo.linear_logprobs(h, w, tok)
    if outlier:
        gl[3] = INF
        groups[0] = (groups[0][0][groups[0][0] != 3], 1.0)
    got = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    for rows, _ in groups:                           # (a bound over the group's rows alone)
        few = bo.LinearLogprobsGrad(got.hidden[rows], None)
        Reference(h[rows], w, tok[rows], 1.0).check_grad(few, gl[rows], gh[rows], "f16", want=(True, False))
    if not outlier:
        both = bo.LinearLogprobsGrad(None, got.weight)
        Reference(h, w, tok, 1.0).check_grad(both, gl, gh, "f16", want=(False, True))
    for want in ((True, False), (False, True)):
        one = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh, want=want)
        for a, b, on in zip(one, got, want):
            assert not on or outlier and a.shape[0] == V or torch.equal(a.nan_to_num(), b.nan_to_num())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [6, 200])
def test_rows_with_infinite_logits(T, kind):
    """A logit of +inf makes its row's results NaN, those of the given token and both
    gradients among them; other rows' hidden gradients are what they are without it."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear +inf", T, kind)
    V, H, bad = 300, 40, 3
    g = _gen(11)
    h = torch.randn((T, H), generator=g).to(_dtype(kind)).cuda()
    w = (0.3 * torch.randn((V, H), generator=g)).to(_dtype(kind)).cuda()
    tok = torch.randint(100, V, (T,), generator=g).cuda()
    gl, gh = torch.randn(T, generator=g).cuda(), (0.3 * torch.randn(T, generator=g)).cuda()
    h[:, 0], w[:, 0], w[10:50, 0] = 1.0, 0.0, -INF
    h[bad, 0] = -1.0
    r = bo.linear_logprobs(h, w, tok)
    others = torch.arange(T, device="cuda") != bad
    for out in (r.logprob, r.entropy, r.stats[:, 1]):
        assert bool(out[bad].isnan()) and not bool(out[others].isnan().any())
    assert r.stats[bad, 0] == INF
    got = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    assert bool(got.hidden[bad].isnan().all()) and bool(got.weight.isnan().all())
    gl[bad] = gh[bad] = 0.0
    want = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    assert torch.equal(got.hidden[others, 1:], want.hidden[others, 1:])
    assert not want.hidden[bad].any() and bool(want.hidden[others, 1:].isfinite().all())
    assert bool(want.weight.isfinite().all()) and not want.weight[10:50].any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [40, 128])
def test_few_tokens_with_a_vocabulary_in_pieces(T, kind):
    """Sums of grad_hidden carried from piece to piece, with d in two parts."""
    import torch
    import paper_2602_10729_amd as bo
    from test_gpu_linear import Reference
    _announce("linear pieces, few tokens", T, kind)
    V, H = 2 ** 26 // T + 70_001, 24                 # (a piece is at most 2^28 bytes of d)
    g = _gen(13)
    w = (0.4 * torch.randn((V, H), generator=g)).to(_dtype(kind)).cuda()
    h = torch.randn((T, H), generator=g).to(_dtype(kind)).cuda()
    tok = torch.randint(V, (T,), generator=g).cuda()
    tok[0], tok[1], tok[2] = 0, V - 1, -1
    gl, gh = torch.randn(T, generator=g).cuda(), (0.3 * torch.randn(T, generator=g)).cuda()
    r = bo.linear_logprobs(h, w, tok)
    ref = Reference(h, w, tok, 1.0)
    ref.check(r)
    ref.check_grad(bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh), gl, gh, kind)


def test_far_gradients():
    """Both gradients whole, of a matrix past 2^32 bytes."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear far gradients")
    V, H, T = 300_000, 8192, 40
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    w = torch.empty((V, H), dtype=torch.bfloat16, device="cuda")
    w.normal_(generator=g).mul_(0.02)
    h = torch.randn((T, H), generator=g, device="cuda").bfloat16()
    tok = torch.randint(V, (T,), generator=g, device="cuda")
    tok[0], tok[1] = V - 1, V - 2
    gl = torch.randn(T, generator=g, device="cuda")
    r = bo.linear_logprobs(h, w, tok)
    got = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl)
    parts = [slice(a, a + 50_000) for a in range(0, V, 50_000)]
    hd = h.double()
    x = torch.cat([hd @ w[s].double().T for s in parts], 1)
    size = float(max((hd.abs() @ w[s].double().abs().T).amax() for s in parts))
    d = -torch.softmax(x, 1) * gl.double()[:, None]
    d.scatter_add_(1, tok[:, None], gl.double()[:, None])
    # d: four logits' errors in its exponent, its own roundings, two parts of 8 bits
    off = 4 * (2 * H ** 0.5 + 4) * EPS * size + (V / 256 + 64) * EPS + 16 * EPS + 2.0 ** -16
    hot = torch.zeros_like(d).scatter_(1, tok[:, None], 4 * EPS * gl.double().abs()[:, None])
    ref, around = torch.zeros_like(hd), torch.zeros_like(hd)
    for s in parts:
        ws = w[s].double()
        ref += d[:, s] @ ws
        around += (d[:, s].abs() * (off + (2 * V ** 0.5 + 4) * EPS) + hot[:, s]) @ ws.abs()
        gw = d[:, s].T @ hd
        tol = (d[:, s].abs() * (off + (2 * T ** 0.5 + 4) * EPS) + hot[:, s]).T @ hd.abs()
        _close(got.weight[s], gw, tol + 2.0 ** -8 * 1.01 * (gw.abs() + tol) + 1e-36, "grad weight")
    _close(got.hidden, ref, around + 2.0 ** -8 * 1.01 * (ref.abs() + around) + 1e-36, "grad hidden")
