"""Log probabilities from hidden rows, and their gradients, on the GPU against
the definitions in 64 bits.

Tolerances come from the arithmetic, with eps = 2^-24 and S_tj the sum of the
sizes of a logit's H products (exact in fp32 for 16-bit types, part of an fma for
fp32). H additions round partial sums of at most S: their errors add up as
independent ones, within (2 sqrt(H) + 4) eps S. A log probability is off by that of
its own logit, by the mean of the others' under p, and by the sum's own roundings;
an entropy by p |u + entropy| times each. d is rounded to 16-bit types once (up to
128 rows what that leaves is rounded too, and added; f16 with a step of 2^-38 of the
call's largest bound, where d is small), sums of d are held in fp32, outputs rounded
once.
"""
import numpy as np
import pytest

from oracle import serving as R

pytestmark = pytest.mark.gpu
INF = np.inf
EPS = 2.0 ** -24
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-36, "bf16": 1e-36, "f16": 2.0 ** -24}


def _announce(*a):
    print("[case]", *a, flush=True)


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _matrix(g, n, m, kind, pad=0, shift=0, spread=1.0):
    """[n, m] of this type in rows of m + pad elements, `shift` elements past an
    aligned start; what lies outside holds NaN."""
    import torch
    buf = torch.full((n * (m + pad) + shift,), float("nan"), dtype=_dtype(kind), device="cuda")
    x = buf[shift:].view(n, m + pad)[:, :m]
    x.copy_(spread * torch.randn((n, m), generator=g, device="cuda"))
    return x


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _sum_tol(V):
    return (V / 256 + 64) * EPS


class Reference:
    """The definitions in float64, with the bounds of each output's error."""

    def __init__(self, hidden, weight, tokens, it):
        import torch
        self.it = it = float(np.float32(it))
        self.h, self.w, self.tok = hidden.double(), weight.double(), tokens
        (T, H), V = self.h.shape, self.w.shape[0]
        self.x = self.h @ self.w.T
        self.lt = (2 * H ** 0.5 + 4) * EPS * (self.h.abs() @ self.w.abs().T)     # of a logit
        self.m = self.x.amax(1)
        d = (self.x - self.m[:, None]) * it
        self.ls = torch.log(torch.exp(d).sum(1))
        self.u = d - self.ls[:, None]
        self.p = torch.exp(self.u)
        self.entropy = -(self.p * self.u).sum(1)
        self.mean = (self.p * self.lt).sum(1)
        self.top = self.lt.gather(1, self.x.argmax(1)[:, None])[:, 0]
        self.ts = _sum_tol(V)
        spread = -(self.p * d).sum(1)
        self.entropy_tol = self.ts * (8 + 2 * spread) + it * (
            self.p * (self.u + self.entropy[:, None]).abs() * (self.lt + self.mean[:, None])).sum(1)

    def check(self, r, what=""):
        import torch
        it, tok = self.it, self.tok
        has = (tok >= 0) & (tok < self.w.shape[0])
        at = torch.where(has, tok, 0)[:, None]
        lp = torch.where(has, self.u.gather(1, at)[:, 0], 0.0)
        lp = torch.where(tok >= self.w.shape[0], float("nan"), lp)
        tol = it * (self.lt.gather(1, at)[:, 0] + self.mean + 2 * self.top) + self.ts + 8 * EPS * (
            lp.abs() + 1) + 2 * EPS * self.ls.abs()
        _close(r.logprob, lp, tol, what + "logprob")
        _close(r.entropy, self.entropy, self.entropy_tol + 2 * EPS * self.entropy.abs(), what + "entropy")
        _close(r.stats[:, 0], self.m, self.lt.amax(1) + EPS * self.m.abs(), what + "max")
        _close(r.stats[:, 1], self.ls, self.ts + it * (2 * self.lt.amax(1) + self.mean) + 4 * EPS * (self.ls.abs() + 1),
               what + "log sum")

    def check_grad(self, r, gl, gh, kind, what="", want=(True, True)):
        import torch
        it, (T, V) = self.it, self.x.shape
        tok, zero = self.tok, torch.zeros(T, dtype=torch.float64, device="cuda")
        gl = zero if gl is None else torch.where(tok >= 0, gl.double(), 0.0)
        gh = zero if gh is None else gh.double()
        live = ((gl != 0) | (gh != 0))[:, None]
        hot = torch.zeros_like(self.x)
        hot.scatter_(1, tok.clamp(min=0)[:, None], gl[:, None])
        lin = self.u + self.entropy[:, None]
        d = it * (hot - self.p * (gl[:, None] + gh[:, None] * lin))
        d = torch.where(live, d, 0.0)
        # d's own error: of the exponent, of the entropy, of its few operations
        du = it * (self.lt + self.mean[:, None] + 2 * self.lt.amax(1, keepdim=True)) + self.ts + 8 * EPS * (self.u.abs() + 2)
        size = gl.abs()[:, None] + gh.abs()[:, None] * (self.u.abs() + self.entropy[:, None].abs())
        td = it * (self.p * (size * (du + 8 * EPS) + gh.abs()[:, None] * (du + self.entropy_tol[:, None]))
                   + 4 * EPS * hot.abs() + EPS * self.p * size)
        if kind != "f32":
            td = td + HALF_ULP[kind] ** (2 if T <= 128 else 1) * (d.abs() + td)
        if kind == "f16":
            td = td + 2.0 ** -38 * it * float((gl.abs() + (np.log(V) + 1) * gh.abs()).max())
        td = torch.where(live, td, 0.0)
        for name, got, on, a, b, c, n in (("hidden", r.hidden, want[0], d, td, self.w, V),
                                          ("weight", r.weight, want[1], d.T, td.T, self.h, T)):
            if not on:
                assert got is None
                continue
            c = torch.where(live, c, 0.0) if name == "weight" else c
            ref = a @ c
            tol = b @ c.abs() + (2 * n ** 0.5 + 4) * EPS * (a.abs() @ c.abs())
            tol = tol + HALF_ULP[kind] * 1.01 * (ref.abs() + tol) + TINY[kind]
            _close(got, ref, tol, f"{what}grad {name}")
        return d


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


def _inputs(T, V, H, kind, seed, pad=0, shift=0):
    import torch
    g = _gen(seed)
    w = _matrix(g, V, H, kind, pad, shift, 2.0 / H ** 0.5)
    h = _matrix(g, T, H, kind, pad, shift)
    tok = torch.randint(V, (T,), generator=g, device="cuda")
    h.copy_(h + 2.0 * torch.rand((T, 1), generator=g, device="cuda") * w[tok])
    if T > 2:
        tok[T // 2] = -1
        tok[T - 1] = V - 1
    gl = torch.randn(T, generator=g, device="cuda")
    gh = 0.3 * torch.randn(T, generator=g, device="cuda")
    if T > 4:
        gh[T // 2] = 0.0                              # takes no part
        gl[1] = gh[1] = 0.0
    return h, w, tok, gl, gh


SIZES = [(1, 1, 1), (1, 2, 3), (2, 33, 8), (3, 127, 16), (31, 129, 64), (32, 1000, 65), (33, 1000, 130),
         (64, 513, 100), (65, 2000, 72), (129, 777, 200), (257, 300, 33), (600, 3001, 264), (1, 5000, 1024),
         (300, 40001, 70), (2000, 5, 40), (4000, 130, 129)]


@pytest.mark.parametrize("T,V,H", SIZES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_sizes(T, V, H, kind):
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear", T, V, H, kind)
    h, w, tok, gl, gh = _inputs(T, V, H, kind, T * 7 + V + H)
    ref = Reference(h, w, tok, 1.0)
    r = bo.linear_logprobs(h, w, tok)
    ref.check(r)
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    ref.check_grad(g, gl, gh, kind)
    a = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh, want=(True, False))
    b = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh, want=(False, True))
    assert a.weight is None and b.hidden is None
    assert bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh, want=(False, False)) == (None, None)
    assert torch.equal(a.hidden, g.hidden) and torch.equal(b.weight, g.weight)
    assert all(torch.equal(x, y) for x, y in zip(r, bo.linear_logprobs(h, w, tok)))


@pytest.mark.parametrize("T,V,H", [(4, 9, 5), (70, 700, 201), (300, 2100, 64)])
def test_oracle_agrees(T, V, H):
    """The same check against the independent reference in numpy."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear oracle", T, V, H)
    h, w, tok, gl, gh = _inputs(T, V, H, "f32", 5)
    n = lambda t: t.double().cpu().numpy()
    o = R.linear_logprobs(n(h), n(w), n(tok).astype(int), 0.75)
    ref = Reference(h, w, tok, 0.75)
    for a, b in ((ref.entropy, o["entropy"]), (ref.m, o["stats"][:, 0]), (ref.ls, o["stats"][:, 1])):
        assert np.allclose(n(a), b, rtol=1e-10, atol=1e-12)
    r = bo.linear_logprobs(h, w, tok, inv_temperature=0.75)
    ref.check(r)
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh, inv_temperature=0.75)
    d = ref.check_grad(g, gl, gh, "f32")
    gh_, gw_, d_ = R.linear_logprobs_grad(n(h), n(w), n(tok).astype(int), n(gl), n(gh), 0.75)
    assert np.allclose(n(d), d_, rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (2, 2), (3, 5), (6, 4), (8, 0)])
def test_strides_and_alignment(kind, pad, shift):
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear alignment", kind, pad, shift)
    for T, V, H in ((3, 50, 9), (40, 300, 127), (130, 1030, 66)):
        h, w, tok, gl, gh = _inputs(T, V, H, kind, pad * 10 + shift, pad, shift)
        ref = Reference(h, w, tok, 1 / 0.7)
        r = bo.linear_logprobs(h, w, tok, inv_temperature=1 / 0.7)
        ref.check(r)
        bufs = [torch.full((n * (H + pad + 1) + shift + 9,), 7.0, dtype=h.dtype, device="cuda") for n in (T, V)]
        out = bo.LinearLogprobsGrad(*(b[shift:shift + n * (H + pad + 1)].view(n, -1)[:, :H] for b, n in zip(bufs, (T, V))))
        g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh, inv_temperature=1 / 0.7, out=out)
        ref.check_grad(g, gl, gh, kind)
        for b, o in zip(bufs, out):
            inside = torch.zeros_like(b, dtype=torch.bool)
            torch.as_strided(inside, o.shape, o.stride(), o.storage_offset()).fill_(True)
            assert bool((b[~inside] == 7.0).all())


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gradients_alone_and_temperatures(kind):
    import paper_2602_10729_amd as bo
    _announce("linear gradients alone", kind)
    h, w, tok, gl, gh = _inputs(90, 1500, 96, kind, 4)
    for it in (0.5, 3.0):
        ref = Reference(h, w, tok, it)
        r = bo.linear_logprobs(h, w, tok, inv_temperature=it)
        ref.check(r)
        for a, b in ((gl, None), (None, gh), (None, None)):
            g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, a, b, inv_temperature=it)
            ref.check_grad(g, a, b, kind)
    r = bo.linear_logprobs(h, w)
    assert not r.logprob.any()
    g = bo.linear_logprobs_grad(h, w, None, r.stats, r.entropy, gl)
    assert not g.hidden.any() and not g.weight.any()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V", [(40, 300), (300, 1100)])
def test_rows_that_take_no_part(kind, T, V):
    """Padding rows may hold anything; rows that take part and hold NaN, infinite
    logits or a token outside show it."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear padding", kind, T, V)
    H = 72
    h, w, tok, gl, gh = _inputs(T, V, H, kind, 9)
    few = torch.arange(T, device="cuda") % 5 != 2
    clean = bo.linear_logprobs(h[few], w, tok[few])
    want = bo.linear_logprobs_grad(h[few], w, tok[few], clean.stats, clean.entropy, gl[few], gh[few])
    h[~few] = float("nan")
    h[7] = INF
    tok[~few] = -1
    gh[~few] = 0.0
    ref = Reference(torch.where(few[:, None], h, 0.0), w, tok, 1.0)
    r = bo.linear_logprobs(h, w, tok)
    assert bool(r.entropy[~few].isnan().all()) and bool(r.stats[~few, 1].isnan().all())
    assert bool((r.logprob[~few] == 0).all()) and not bool(r.entropy[few].isnan().any())
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    ref.check_grad(g, gl, gh, kind)
    assert not g.hidden[~few].any() and bool((g.weight - want.weight).abs().max() < 0.1)
    # a row that takes part
    tok[2] = 1
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    assert bool(g.hidden[2].isnan().all()) and bool(g.weight.isnan().all())
    assert not bool(g.hidden[few].isnan().any())
    # a token outside
    h[~few], tok[2], tok[0] = 0.0, -1, V
    r = bo.linear_logprobs(h, w, tok)
    assert bool(r.logprob[0].isnan()) and not bool(r.logprob[1:].isnan().any())
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    assert bool(g.hidden[0].isnan().all()) and bool(g.weight.isnan().all())


def test_infinite_logits():
    """Logits of minus infinity are masked, as in token_logprobs; rows of nothing
    else have no distribution."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear masks")
    T, V, H = 6, 300, 8
    h, w, tok, gl, gh = _inputs(T, V, H, "f32", 3)
    h[:, 0], w[:, 0] = 1.0, 0.0
    w[10:200, 0] = -INF                      # masks those words in every row
    logits = h.clone() @ torch.where(w == -INF, 0.0, w).T
    logits[:, 10:200] = -INF
    tok[0], tok[1] = 20, 5
    r = bo.linear_logprobs(h, w, tok)
    s = bo.token_logprobs(logits, tok)
    assert r.logprob[0] == -INF
    _close(r.logprob[1:], s.logprob[1:].double(), torch.tensor(1e-5, device="cuda"), "logprob")
    _close(r.entropy, s.entropy.double(), torch.tensor(2e-5, device="cuda"), "entropy")
    h[3, 0] = -1.0                           # +inf logits
    r = bo.linear_logprobs(h, w, tok)
    assert bool(r.logprob[3].isnan() | (tok[3] < 0)) and bool(r.entropy[3].isnan())
    w[:, 0] = -INF
    h[:, 0] = 1.0
    r = bo.linear_logprobs(h, w, tok)
    assert bool((r.logprob[tok >= 0] == -INF).all()) and not r.entropy.any() and bool((r.stats == -INF).all())
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    assert not g.hidden.any() and not g.weight.any()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1, 40, 300])
def test_gradients_beside_masked_words(T, kind):
    """Words masked by a matrix of minus infinity get no gradient and change no
    other word's; the column that masks has none in the hidden rows."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear masked words", T, kind)
    V, H, n = 700, 40, 30                    # the last n words are masked
    h, w, tok, gl, gh = _inputs(T, V, H, kind, 17)
    h[:, 0], tok[tok >= V - n] = 1.0, 5
    w[V - n:, 0] = -INF
    gl[T // 2:T // 2 + 3 * (T > 1)] = 0.0    # rows without a gradient, but for T = 1
    gh[T // 2:T // 2 + 3 * (T > 1)] = 0.0
    ref = Reference(h, w[:V - n], tok, 1.0)
    r = bo.linear_logprobs(h, w, tok)
    ref.check(r)
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    live = (torch.where(tok >= 0, gl, 0.0) != 0) | (gh != 0)
    assert bool(g.hidden[live, 0].isnan().all()) and not g.hidden[~live].any()
    assert not g.weight[V - n:].any()
    kept = bo.linear_logprobs_grad(h, w[:V - n], tok, r.stats, r.entropy, gl, gh)
    ref.check_grad(kept, gl, gh, kind)
    g.hidden[:, 0] = kept.hidden[:, 0]
    ref.check_grad(bo.LinearLogprobsGrad(g.hidden, g.weight[:V - n]), gl, gh, kind)


def test_unequal_gradients_in_half_precision():
    """f16 shares one scale over the call: small rows beside large ones, large and
    tiny gradients as loss scaling gives them."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear f16 scale")
    h, w, tok, gl, gh = _inputs(200, 3000, 64, "f16", 12)
    ref = Reference(h, w, tok, 1.0)
    r = bo.linear_logprobs(h, w, tok)
    for s in (2.0 ** 12, 2.0 ** -20):
        a, b = gl * s, gh * s
        a[::3] *= 2.0 ** -9
        b[::3] *= 2.0 ** -9
        g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, a, b)
        ref.check_grad(g, a, b, "f16", f"{s} ")
    huge = torch.full_like(gl, 3e38)
    assert not bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, huge).hidden.isnan().any()


@pytest.mark.parametrize("T", [3, 200])
def test_tiny_values_in_half_precision(T):
    """f16 values below its normal range count at their value."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear f16 subnormal", T)
    g = _gen(7)
    h = (torch.randint(1, 60, (T, 64), generator=g, device="cuda") * 2.0 ** -24).half()
    w = (torch.randint(-800, 800, (500, 64), generator=g, device="cuda") * 64.0).half()
    tok = torch.randint(500, (T,), generator=g, device="cuda")
    gl, gh = torch.randn(T, generator=g, device="cuda"), torch.zeros(T, device="cuda")
    ref = Reference(h, w, tok, 1.0)
    assert float(ref.x.abs().max()) > 0.3                 # (what the small values make)
    r = bo.linear_logprobs(h, w, tok)
    ref.check(r)
    ref.check_grad(bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh), gl, gh, "f16")


@pytest.mark.parametrize("kind,T,V,H", [("bf16", 4100, 8000, 4104), ("f16", 4100, 40000, 72), ("bf16", 4200, 33000, 1000),
                                        ("f32", 4100, 17000, 136), ("bf16", 30000, 700, 64)])
def test_large(kind, T, V, H):
    """Large tiles throughout; a vocabulary in several pieces; sums split over k."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear large", kind, T, V, H)
    h, w, tok, gl, gh = _inputs(T, V, H, kind, T + V)
    r = bo.linear_logprobs(h, w, tok)
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh)
    ref = Reference(h, w, tok, 1.0)
    ref.check(r)
    ref.check_grad(g, gl, gh, kind)


def test_far_rows():
    """Matrices past 2^32 bytes."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("linear far")
    V, H, T = 300_000, 8192, 40
    g = _gen(1)
    w = torch.empty((V, H), dtype=torch.bfloat16, device="cuda")
    w.normal_(generator=g).mul_(0.02)
    h = _matrix(g, T, H, "bf16")
    tok = torch.randint(V, (T,), generator=g, device="cuda")
    tok[0], tok[1] = V - 1, V - 2
    r = bo.linear_logprobs(h, w, tok)
    x = torch.cat([h.double() @ w[a:a + 50_000].double().T for a in range(0, V, 50_000)], 1)
    lsm = torch.log_softmax(x, 1)
    lt = (2 * H ** 0.5 + 4) * EPS * H * 0.02        # (sizes of the products: about 0.64 each)
    _close(r.logprob, lsm.gather(1, tok[:, None])[:, 0], torch.tensor(4 * lt + _sum_tol(V) * 20, device="cuda"), "logprob")
    gl = torch.randn(T, generator=g, device="cuda")
    got = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl)
    d = -lsm.exp() * gl.double()[:, None]
    d.scatter_add_(1, tok[:, None], gl.double()[:, None])
    for rows in (slice(0, 64), slice(V - 64, V), slice(262_140, 262_180)):
        ref = d[:, rows].T @ h.double()
        tol = 2.2 * 2.0 ** -8 * (d[:, rows].abs().T @ h.double().abs())       # (d, and the output)
        _close(got.weight[rows], ref, tol + 1e-30, "grad weight")


# ---- how they are called ---------------------------------------------------------

def _all_calls(bo, h, w, tok, gl, gh, stream=None):
    r = bo.linear_logprobs(h, w, tok, stream=stream)
    g = bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, gh, stream=stream)
    rows = bo.embed(tok, w, scale=2.0, stream=stream)
    t = bo.embed_grad(tok, rows, w.shape[0], stream=stream)
    to = bo.route(h[:, :8], 3, stream=stream)
    d = bo.dispatch(to.ids, 8, stream=stream)
    x = bo.expert_gather(h, d.order, d.position, stream=stream)
    y = bo.expert_combine(x, d.position, to.weights, stream=stream)
    c = bo.expert_combine_grad(y, x, d.order, d.position, to.weights, stream=stream)
    return [*r, *g, rows, t, x, y, *c]


@pytest.mark.parametrize("T,V,H", [(3, 5000, 64), (400, 3001, 200)])
def test_other_streams_give_the_same_bits(T, V, H):
    import torch
    import paper_2602_10729_amd as bo
    _announce("streams")
    sets = [_inputs(T, V, H, "bf16", s) for s in (1, 2)]
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


@pytest.mark.parametrize("T,V,H", [(1, 4000, 64), (300, 2000, 136)])
def test_graph_replays(T, V, H):
    """Every call captured; replays with new inputs, with eager work between."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("graph")
    cur = _inputs(T, V, H, "bf16", 1)
    _all_calls(bo, *cur)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _all_calls(bo, *cur)
    for i in range(4):
        nxt = _inputs(T, V, H, "bf16", 10 + i)
        for a, b in zip(cur, nxt):
            a.copy_(b)
        want = _all_calls(bo, *nxt)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_refusals_on_the_device():
    import torch
    import paper_2602_10729_amd as bo
    _announce("refusals")
    h, w, tok, gl, gh = _inputs(8, 100, 16, "f32", 1)
    r = bo.linear_logprobs(h, w, tok)
    grad = lambda **k: bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl, **k)
    z = torch.zeros_like
    bad = [
        lambda: bo.linear_logprobs(h.double(), w.double(), tok), lambda: bo.linear_logprobs(h.half(), w, tok),
        lambda: bo.linear_logprobs(h[:, :15], w, tok), lambda: bo.linear_logprobs(h, w, tok.int()),
        lambda: bo.linear_logprobs(h, w, tok[:7]), lambda: bo.linear_logprobs(h.cpu(), w, tok),
        lambda: bo.linear_logprobs(h[:, ::2], w[:, ::2], tok), lambda: bo.linear_logprobs(h, w[:0], tok),
        lambda: bo.linear_logprobs(h[:, :0], w[:, :0], tok), lambda: bo.linear_logprobs(h[0], w, tok),
        lambda: bo.linear_logprobs(h, w, tok, inv_temperature=0.0),
        lambda: bo.linear_logprobs(h, w, tok, inv_temperature=float("nan")),
        lambda: bo.linear_logprobs(h, w, tok, out=(r.logprob, r.entropy, r.entropy)),
        lambda: bo.linear_logprobs_grad(h, w, tok, r.stats[:, :1], r.entropy, gl),
        lambda: bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy[:3], gl),
        lambda: bo.linear_logprobs_grad(h, w, tok, r.stats, r.entropy, gl.double()),
        lambda: grad(out=(h, z(w))), lambda: grad(out=(z(h), w)), lambda: grad(out=(w[:8], None)),
        lambda: grad(out=(None, z(w).half())), lambda: grad(out=(z(w), None)),
        lambda: (lambda b: grad(out=(b[:8], b[4:104])))(torch.zeros((104, 16), device="cuda")),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((bo.BoError, ValueError, TypeError)):
            f()
            print("accepted", i, flush=True)
    none = bo.linear_logprobs(h[:0], w, tok[:0])
    assert none.stats.shape == (0, 2)
    g = bo.linear_logprobs_grad(h[:0], w, tok[:0], none.stats, none.entropy, out=(None, torch.ones_like(w)))
    assert not g[1].any()
    torch.cuda.synchronize()
