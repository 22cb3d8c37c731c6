"""Expert rows and embeddings on the GPU against their fp64 references.

Rows that are copied are equal bit for bit. A sum of n terms in fp32 is off by at
most n roundings of the sum of their sizes (each a product rounded once or not at
all), and an output by half a step of its type more.
"""
import numpy as np
import pytest

from oracle import serving as R

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-37, "bf16": 1e-37, "f16": 2.0 ** -24}


def _announce(*a):
    print("[case]", *a, flush=True)


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _matrix(rng, n, m, kind, pad=0, shift=0, spread=1.0):
    """[n, m] of this type in rows of m + pad elements, `shift` elements past an
    aligned start; what lies outside holds NaN."""
    import torch
    buf = torch.full((n * (m + pad) + shift,), float("nan"), dtype=_dtype(kind), device="cuda")
    x = buf[shift:].view(n, m + pad)[:, :m]
    x.copy_(torch.from_numpy((spread * rng.standard_normal((n, m))).astype(np.float32)))
    return x


def _blank(n, m, kind, pad, shift):
    """An output in a larger buffer of a known value, and that buffer."""
    import torch
    buf = torch.full((n * (m + pad) + shift + 7,), 7.0, dtype=_dtype(kind), device="cuda")
    return buf[shift:shift + n * (m + pad)].view(n, m + pad)[:, :m], buf


def _untouched(buf, out):
    """Whether everything but `out` still holds its value."""
    import torch
    inside = torch.zeros_like(buf, dtype=torch.bool)
    torch.as_strided(inside, out.shape, out.stride(), out.storage_offset()).fill_(True)
    return bool((buf[~inside] == 7.0).all())


def _np(x):
    return x.double().cpu().numpy()


def _close(got, want, tol, what):
    got = _np(got)
    assert got.shape == want.shape, what
    with np.errstate(invalid="ignore"):
        ok = (got == want) | (np.isnan(got) & np.isnan(want)) | (np.abs(got - want) <= tol)
    assert ok.all(), (what, int((~ok).sum()), got[~ok][:4], want[~ok][:4])


def _i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _i64(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).cuda()


def _ids(rng, T, top, E):
    """Distinct experts per token; some choices missing, one token without any."""
    ids = np.argsort(rng.random((T, E)), 1)[:, :top].astype(np.int32)
    ids[rng.random((T, top)) < 0.1] = -1
    if T > 3:
        ids[T // 2] = -1
    return ids


CASES = [  # T, top, E, H, capacity, pad, shift
    (1, 1, 1, 1, 0, 0, 0), (1, 8, 64, 4096, 0, 0, 0), (2, 3, 3, 7, 0, 1, 3), (16, 8, 64, 2050, 0, 0, 0),
    (33, 2, 5, 64, 4, 3, 1), (100, 32, 40, 130, 0, 2, 5), (257, 4, 61, 513, 9, 0, 0),
    (1000, 2, 8, 1111, 200, 5, 2), (4099, 6, 16, 72, 0, 0, 0), (9001, 1, 3, 24, 1500, 1, 1)]


@pytest.mark.parametrize("T,top,E,H,capacity,pad,shift", CASES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_expert_rows(T, top, E, H, capacity, pad, shift, kind):
    import torch
    import paper_2602_10729_amd as bo
    _announce("experts", T, top, E, H, capacity, kind)
    rng = np.random.default_rng(T * 100 + H)
    d = bo.dispatch(_i32(_ids(rng, T, top, E)), E, capacity=capacity)
    order, position = d.order.cpu().numpy(), d.position.cpu().numpy()
    N, kept = T * top, int(d.offsets[-1])
    x = _matrix(rng, T, H, kind, pad, shift)
    out, buf = _blank(N, H, kind, pad, shift)
    g = bo.expert_gather(x, d.order, d.position, out=out)
    assert g is out and _untouched(buf, out)
    assert np.array_equal(_np(g), R.expert_gather(_np(x), order, top))
    # as many rows as experts keep, where a capacity bounds them
    if kept:
        g = bo.expert_gather(x, d.order[:kept], d.position)
        assert np.array_equal(_np(g), R.expert_gather(_np(x), order[:kept], top))

    rows = _matrix(rng, N, H, kind, pad, shift)
    rows[kept:] = float("nan")                          # rows that nobody fills are not read
    w = torch.from_numpy(rng.standard_normal((T, top)).astype(np.float32)).cuda()
    w[d.position < 0] = float("nan")                    # nor their weights
    for weights in (w, None):
        out, buf = _blank(T, H, kind, pad, shift)
        y = bo.expert_combine(rows, d.position, weights, out=out)
        assert y is out and _untouched(buf, out)
        want, size = R.expert_combine(_np(rows), position, None if weights is None else _np(w))
        _close(y, want, (top + 1) * EPS * size + HALF_ULP[kind] * 1.01 * np.abs(want) + TINY[kind], "combine")

        dy = _matrix(rng, T, H, kind, pad, shift)
        out, buf = _blank(N, H, kind, pad, shift)
        gw = torch.full((T, top), 7.0, device="cuda")
        r = bo.expert_combine_grad(dy, rows, d.order, d.position, weights,
                                   out=bo.ExpertCombineGrad(out, gw))
        assert r[0] is out and _untouched(buf, out)
        g_rows, g_w, size = R.expert_combine_grad(_np(dy), _np(rows), order, position,
                                                  None if weights is None else _np(w))
        _close(r.rows, g_rows, HALF_ULP[kind] * 1.01 * np.abs(g_rows) + TINY[kind], "grad_rows")
        _close(r.weights, g_w, (H + 2) * EPS * size, "grad_weights")
        a = bo.expert_combine_grad(dy, rows, d.order, d.position, weights, want=(True, False))
        b = bo.expert_combine_grad(dy, rows, d.order, d.position, weights, want=(False, True))
        assert a.weights is None and b.rows is None
        assert torch.equal(a.rows, r.rows) and torch.equal(b.weights, r.weights)


def test_expert_rows_outside_are_none():
    """Positions past the rows that are given are left out; so are ids of experts
    that a rank does not hold, dispatched as such."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("experts outside")
    rng = np.random.default_rng(2)
    T, top, E, H = 50, 3, 9, 40
    ids = _ids(rng, T, top, E)
    d = bo.dispatch(_i32(ids), E)
    R_ = 31
    order, position = d.order[:R_].contiguous(), d.position
    rows, dy = _matrix(rng, R_, H, "f32"), _matrix(rng, T, H, "f32")
    y = bo.expert_combine(rows, position)
    want, size = R.expert_combine(_np(rows), position.cpu().numpy())
    _close(y, want, (top + 1) * EPS * size, "combine")
    r = bo.expert_combine_grad(dy, rows, order, position)
    g_rows, g_w, size = R.expert_combine_grad(_np(dy), _np(rows), order.cpu().numpy(), position.cpu().numpy())
    _close(r.rows, g_rows, 0.0, "grad_rows")
    _close(r.weights, g_w, (H + 2) * EPS * size, "grad_weights")
    none = bo.dispatch(torch.full((T, top), -1, dtype=torch.int32, device="cuda"), E)
    assert not bo.expert_gather(dy, none.order, none.position).any()
    assert not bo.expert_combine(_matrix(rng, T * top, H, "bf16"), none.position).any()
    r = bo.expert_combine_grad(dy, _matrix(rng, T * top, H, "f32"), none.order, none.position)
    assert not r.rows.any() and not r.weights.any()


def test_expert_gather_gradient_is_combine():
    """Against torch's own differentiation of the indexing, in 64 bits."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("experts autograd")
    rng = np.random.default_rng(3)
    T, top, E, H = 40, 4, 7, 33
    d = bo.dispatch(_i32(_ids(rng, T, top, E)), E, capacity=15)
    c = _matrix(rng, T * top, H, "f32")
    x = torch.zeros((T, H), dtype=torch.float64, device="cuda", requires_grad=True)
    kept = int(d.offsets[-1])
    (x[d.order[:kept].long() // top] * c[:kept].double()).sum().backward()
    got = bo.expert_combine(c, d.position)
    _close(got, x.grad.cpu().numpy(), (top + 1) * EPS * 4 * float(c.abs().max()), "gradient")


# ---- embeddings ----------------------------------------------------------------

EMBED = [  # T, V, H, pad, shift
    (1, 1, 1, 0, 0), (1, 128000, 256, 0, 0), (5, 3, 7, 1, 3), (31, 50, 64, 0, 0), (32, 4, 9, 2, 1),
    (33, 2, 520, 0, 0), (64, 1000, 2050, 3, 0), (1000, 37, 130, 0, 0), (1024, 1024, 24, 0, 0),
    (1025, 1023, 24, 1, 0), (3000, 70000, 8, 0, 0), (5000, 1, 40, 0, 0), (8193, 300, 17, 0, 5),
    (20000, 100003, 16, 0, 0)]


def _text(rng, T, V):
    """Tokens by a power of their rank, padding and strays among them."""
    tok = np.minimum(V ** rng.random(T), V).astype(np.int64) - 1
    if T > 4:
        tok[::7] = -1
        tok[3] = -2 ** 40
    return tok


@pytest.mark.parametrize("T,V,H,pad,shift", EMBED)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_embed(T, V, H, pad, shift, kind):
    import paper_2602_10729_amd as bo
    _announce("embed", T, V, H, kind)
    rng = np.random.default_rng(T + V)
    tok = _text(rng, T, V)
    table = _matrix(rng, V, H, kind, pad, shift)
    at = tok.copy()
    if T > 4:
        at[1], at[2] = V, 2 ** 40                       # no such row: NaN
    for scale in (1.0, 2.5):
        out, buf = _blank(T, H, kind, pad, shift)
        y = bo.embed(_i64(at), table, scale=scale, out=out)
        assert y is out and _untouched(buf, out)
        few = R.embed(at, _np(table), scale)
        _close(y, few, 0.0 if scale == 1.0 else HALF_ULP[kind] * 1.01 * np.abs(few) + TINY[kind], "rows")
        grad = _matrix(rng, T, H, kind, pad, shift)
        grad[_i64(np.flatnonzero((at < 0) | (at >= V)))] = float("nan")     # not read
        out, buf = _blank(V, H, kind, pad, shift)
        g = bo.embed_grad(_i64(at), grad, V, scale=scale, out=out)
        assert g is out and _untouched(buf, out)
        want, size, count = R.embed_grad(at, _np(grad), V, scale)
        tol = (count[:, None] + 1) * EPS * size + HALF_ULP[kind] * 1.01 * np.abs(want) + TINY[kind]
        _close(g, want, tol, "grad")


@pytest.mark.parametrize("T,V,H", [(100_003, 7, 33), (300_000, 1, 8), (70_001, 200_000, 4), (40_000, 3, 1031)])
def test_embed_grad_long_runs(T, V, H):
    """Many tokens of few rows: runs over many chunks, and all of one row."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("embed long", T, V, H)
    rng = np.random.default_rng(T)
    tok = _i64(rng.integers(-1, V, T))
    grad = _matrix(rng, T, H, "bf16")
    g = bo.embed_grad(tok, grad, V)
    want = torch.zeros((V + 1, H), dtype=torch.float64, device="cuda")
    size, count = torch.zeros_like(want), torch.zeros(V + 1, dtype=torch.float64, device="cuda")
    at = torch.where(tok >= 0, tok, V)
    want.index_add_(0, at, grad.double())
    size.index_add_(0, at, grad.double().abs())
    count.index_add_(0, at, torch.ones(T, dtype=torch.float64, device="cuda"))
    want, size, count = (t[:V].cpu().numpy() for t in (want, size, count))
    # no chain of additions is longer than a share of the chunks and a chunk
    steps = np.minimum(count, 32 + count / 128 + 8)[:, None]
    _close(g, want, steps * EPS * size + HALF_ULP["bf16"] * 1.01 * np.abs(want) + 1e-37, "grad")


@pytest.mark.parametrize("T,V,H", [(9000, 1000, 12), (7001, 600_000, 3), (100, 1_500_000, 2), (30_011, 3_000_001, 1)])
def test_embed_grad_sorts(T, V, H):
    """The widest digits and three of them, by one workgroup and by many; whole
    numbers, so that sums are exact, and every call gives the same bits."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("embed sorts", T, V, H)
    rng = np.random.default_rng(T)
    ids = rng.integers(0, V, T)
    ids[::3] = rng.integers(max(0, V - 20), V + 3, len(ids[::3]))       # some runs, some outside
    ids[::11], ids[-1] = -1, V - 1
    grad = rng.integers(-8, 9, (T, H)).astype(np.float32)
    want = np.zeros((V, H), np.float32)
    inside = (ids >= 0) & (ids < V)
    np.add.at(want, ids[inside], grad[inside])
    g = bo.embed_grad(_i64(ids), torch.from_numpy(grad).cuda(), V)
    assert torch.equal(g.cpu(), torch.from_numpy(want))
    noise = torch.randn((T, H), device="cuda")
    assert torch.equal(bo.embed_grad(_i64(ids), noise, V), bo.embed_grad(_i64(ids), noise, V))


def test_wide_and_far_rows():
    """Offsets past 2^31 elements, and rows wider than a wave's sweep."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("far rows")
    V, H = 300_000, 8192
    table = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    table[V - 1] = 3.0
    table[V - 2] = 5.0
    tok = _i64([V - 1, -1, V - 2, V - 1])
    y = bo.embed(tok, table)
    assert torch.equal(y, torch.tensor([[3.0], [0.0], [5.0], [3.0]], device="cuda").bfloat16().expand(4, H))
    g = bo.embed_grad(tok, y, V)
    assert bool((g[V - 1] == 6.0).all()) and bool((g[V - 2] == 5.0).all()) and not g[:V - 2].any()
    del table, g
    T, top = 150_001, 2
    x = torch.zeros((T, H), dtype=torch.bfloat16, device="cuda")
    x += (torch.arange(T, device="cuda") % 199)[:, None].bfloat16()
    ids = torch.stack([torch.arange(T, device="cuda") % 5, 5 + torch.arange(T, device="cuda") % 3], 1).int()
    d = bo.dispatch(ids, 8)
    rows = bo.expert_gather(x, d.order, d.position)
    assert torch.equal(rows[:, 0], x[d.order.long() // top, 0])
    assert torch.equal(rows[:, H - 1], rows[:, 0])
    y = bo.expert_combine(rows, d.position, torch.full((T, top), 0.5, device="cuda"))
    assert torch.equal(y, x)


def test_refusals_on_the_device():
    import torch
    import paper_2602_10729_amd as bo
    _announce("refusals")
    x = torch.zeros((4, 16), device="cuda")
    d = bo.dispatch(torch.zeros((4, 2), dtype=torch.int32, device="cuda"), 3)
    rows, tok = torch.zeros((8, 16), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    buf = torch.zeros((8, 32), device="cuda")
    bad = [
        lambda: bo.expert_gather(x.double(), d.order, d.position), lambda: bo.expert_gather(x[:3], d.order, d.position),
        lambda: bo.expert_gather(x[:, ::2], d.order, d.position), lambda: bo.expert_gather(x, d.order.long(), d.position),
        lambda: bo.expert_gather(x, d.order, d.position.view(-1)), lambda: bo.expert_gather(x.cpu(), d.order, d.position),
        lambda: bo.expert_gather(x, torch.zeros(9, dtype=torch.int32, device="cuda"), d.position),
        lambda: bo.expert_gather(x, d.order, d.position, out=rows.half()),
        lambda: bo.expert_gather(rows[:4], d.order, d.position, out=rows),
        lambda: bo.expert_gather(buf[:4, 4:20], d.order, d.position, out=buf[:, :16]),
        lambda: bo.expert_combine(torch.zeros((9, 16), device="cuda"), d.position),
        lambda: bo.expert_combine(rows, d.position, torch.zeros((4, 3), device="cuda")),
        lambda: bo.expert_combine(rows, d.position, torch.zeros((4, 2), device="cuda").half()),
        lambda: bo.expert_combine(rows, d.position, out=rows[:4]),
        lambda: bo.expert_combine_grad(x, rows.half(), d.order, d.position),
        lambda: bo.expert_combine_grad(x, rows[:7], d.order, d.position),
        lambda: bo.expert_combine_grad(x, rows, d.order, d.position, out=(rows, torch.zeros((4, 2), device="cuda"))),
        lambda: bo.embed(tok.int(), rows), lambda: bo.embed(tok, rows.double()), lambda: bo.embed(tok, rows, scale=float("nan")),
        lambda: bo.embed(tok.view(2, 2), rows), lambda: bo.embed(tok, rows, out=rows[:4]), lambda: bo.embed(tok, rows[:0]),
        lambda: bo.embed_grad(tok, x, 0), lambda: bo.embed_grad(tok[:3], x, 5), lambda: bo.embed_grad(tok, rows[:4], 8, out=rows),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((bo.BoError, ValueError, TypeError)):
            f()
            print("accepted", i, flush=True)
    # column ranges of one buffer do not overlap
    y = bo.expert_gather(buf[:4, 16:], d.order, d.position, out=buf[:, :16])
    assert y.shape == (8, 16)
    # nothing to do
    none = bo.dispatch(torch.zeros((0, 2), dtype=torch.int32, device="cuda"), 3)
    assert bo.expert_gather(x[:0], none.order, none.position).shape == (0, 16)
    assert bo.expert_combine(rows[:0], none.position).shape == (0, 16)
    assert bo.expert_combine_grad(x[:0], rows[:0], none.order, none.position).weights.shape == (0, 2)
    assert bo.expert_combine(rows[:0], d.position).abs().sum() == 0
    assert bo.embed(tok[:0], rows).shape == (0, 16)
    g = bo.embed_grad(tok[:0], x[:0], 5, out=torch.ones((5, 16), device="cuda"))
    assert not g.any()
    torch.cuda.synchronize()
