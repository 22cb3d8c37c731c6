"""Expert rows and embeddings where their memory lies: column ranges of one buffer,
shared memory, and rows past what the caches hold; on the GPU."""
import pytest

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _announce(*a):
    print("[case]", *a, flush=True)


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_one_row_in_other_columns_of_a_buffer(kind):
    """A single row beside its outputs, as one token's decoding step has it: the same
    layouts as with several rows."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("rows, one row", kind)
    H, top = 16, 8
    buf = torch.randn((top, 3 * H), device="cuda").to(_dtype(kind))
    x, order = buf[:1, H:2 * H].clone(), torch.randperm(top, device="cuda").int()
    position = torch.empty((1, top), dtype=torch.int32, device="cuda")
    position[0, order.long()] = torch.arange(top, device="cuda", dtype=torch.int32)
    bo.expert_gather(buf[:1, H:2 * H], order, position, out=buf[:, :H])
    assert torch.equal(buf[:, :H], x.expand(top, H)) and torch.equal(buf[:1, H:2 * H], x)
    # back into one row, in the columns after
    w = torch.full((1, top), 0.125, device="cuda")
    bo.expert_combine(buf[:, :H], position, w, out=buf[3:4, 2 * H:])
    # eighths of x add up exactly in 16-bit types (11 bits and 3 more); of 24 bits and 3
    # more each of the seven additions leaves half a step of a sum of at most |x|
    y = buf[3:4, 2 * H:].clone()
    assert bool(((y - x).abs() <= (8 * 2.0 ** -24 if kind == "f32" else 0.0) * x.abs()).all())
    g = bo.expert_combine_grad(buf[3:4, 2 * H:], buf[:, :H], order, position, w,
                               out=(buf[:, H:2 * H], torch.empty_like(w)))
    assert torch.equal(g[0], (0.125 * y.float()).to(x.dtype).expand(top, H))
    # one token of a table, and the gradient of a table of one row
    tok = torch.tensor([5], device="cuda")
    bo.embed(tok, buf[:, :H], out=buf[2:3, H:2 * H])
    assert torch.equal(buf[2:3, H:2 * H], x)
    many = torch.zeros(top, dtype=torch.int64, device="cuda")
    t = bo.embed_grad(many, buf[:, :H], 1, out=buf[6:7, 2 * H:])
    assert bool(((t - 8 * x).abs() <= (8 * 2.0 ** -24 if kind == "f32" else 0.0) * 8 * x.abs()).all())
    torch.cuda.synchronize()


def test_different_strides_of_one_buffer():
    """Every second row's columns beside other columns of every row."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("rows, strides")
    H = 16
    buf = torch.randn((8, 2 * H), device="cuda")
    x = buf[::2, H:].clone()
    order = torch.arange(8, dtype=torch.int32, device="cuda")
    bo.expert_gather(buf[::2, H:], order, order.view(4, 2), out=buf[:, :H])
    assert torch.equal(buf[:, :H], x.repeat_interleave(2, 0)) and torch.equal(buf[::2, H:], x)


def test_one_row_that_shares_memory_is_refused():
    import torch
    import paper_2602_10729_amd as bo
    _announce("rows, one row shared")
    top, H = 8, 16
    one = torch.ones((top, H), device="cuda")
    order = torch.arange(top, dtype=torch.int32, device="cuda")
    position, tok = order.view(1, top).clone(), torch.zeros(4, dtype=torch.int64, device="cuda")
    keep = one.clone()
    bad = [
        lambda: bo.expert_gather(one[2:3], order, position, out=one),
        lambda: bo.expert_gather(one[2:3, :8], order, position, out=one[:, 4:12]),
        lambda: bo.expert_combine(one, position, out=one[7:8]),
        lambda: bo.expert_combine(one[:, :8], position, out=one[7:8, 7:15]),
        lambda: bo.expert_combine_grad(one[2:3], one.clone(), order, position, out=(one, None)),
        lambda: bo.embed(tok[:1], one, out=one[1:2]),
        lambda: bo.embed_grad(tok, one[:4], 1, out=one[3:4]),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(bo.BoError, match="overlap"):
            f()
            print("accepted", i, flush=True)
    torch.cuda.synchronize()
    assert torch.equal(one, keep)


def test_outputs_in_the_place_of_vectors_are_refused():
    import torch
    import paper_2602_10729_amd as bo
    _announce("rows, vectors shared")
    T, top, H = 4, 2, 16
    x, rows = torch.ones((T, H), device="cuda"), torch.ones((T * top, H), device="cuda")
    order = torch.arange(T * top, dtype=torch.int32, device="cuda")
    position, w = order.view(T, top).clone(), torch.ones((T, top), device="cuda")
    gw, tok = torch.empty_like(w), torch.zeros(T, dtype=torch.int64, device="cuda")
    gx = torch.ones((T * top, H), device="cuda")
    floats = lambda t: t.view(-1).view(torch.float32)
    col = lambda t, n: floats(t)[:n].view(n, 1)      # a matrix of one column in its place
    bad = [
        lambda: bo.expert_gather(x[:, :1], order, position, out=col(order, 8)),
        lambda: bo.expert_gather(x[:, :1], order, position, out=col(position, 8)),
        lambda: bo.expert_combine(rows[:, :1], position, w, out=col(position, 4)),
        lambda: bo.expert_combine(rows[:, :1], position, w, out=col(w, 4)),
        lambda: bo.expert_combine_grad(x, rows, order, position, w, out=(gx, w)),
        lambda: bo.expert_combine_grad(x, rows, order, position, w, out=(gx, floats(position).view(T, top))),
        lambda: bo.expert_combine_grad(x, rows, order, position, w, out=(gx, rows[0, :8].view(T, top))),
        lambda: bo.expert_combine_grad(x, rows, order, position, w, out=(gx, x[0, 4:12].view(T, top))),
        lambda: bo.expert_combine_grad(x, rows, order, position, w, out=(gx, gx[7, 4:12].view(T, top))),
        lambda: bo.expert_combine_grad(x[:, :1], rows[:, :1], order, position, w, out=(col(w, 8), gw)),
        lambda: bo.expert_combine_grad(x[:, :1], rows[:, :1], order, position, w, out=(col(order, 8), gw)),
        lambda: bo.expert_combine_grad(x[:, :1], rows[:, :1], order, position, w, out=(col(position, 8), None)),
        lambda: bo.embed(tok, rows[:, :1], out=col(tok, 4)), lambda: bo.embed_grad(tok, x[:, :1], 3, out=col(tok, 3)),
    ]
    held = (x, rows, order, position, w, tok)
    keep = [t.clone() for t in held]
    for i, f in enumerate(bad):
        with pytest.raises(bo.BoError, match="overlap"):
            f()
            print("accepted", i, flush=True)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(keep, held))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("H", [2112, 2113])
def test_gradients_past_the_caches(kind, H):
    """More than 160 MB of rows, which are written past the caches; rows that no pair
    fills hold NaN and are cleared in the gradient."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("rows, past the caches", kind, H)
    T, top, E = 20_003, 2, 7
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda")
    ids = torch.rand((T, E), generator=g, device="cuda").topk(top, 1).indices.int()
    ids[::9] = -1
    d = bo.dispatch(ids, E, capacity=5000)
    kept = int(d.offsets[-1])
    rows = draw(T * top, H).to(_dtype(kind))
    rows[kept:] = float("nan")
    dy, w = draw(T, H).to(_dtype(kind)), draw(T, top)
    assert rows.numel() * rows.element_size() > 160 << 20
    got = bo.expert_combine_grad(dy, rows, d.order, d.position, w)
    pair = d.order[:kept].long()
    grad = dy[pair // top].double()
    want = w.view(-1)[pair].double()[:, None] * grad
    off = (got.rows[:kept].double() - want).abs()
    assert bool((off <= HALF_ULP[kind] * 1.01 * want.abs() + 2.0 ** -24).all())
    assert not got.rows[kept:].any()
    dots = torch.zeros(T * top, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(dots)
    dots[pair] = (grad * rows[:kept].double()).sum(1)
    size[pair] = (grad * rows[:kept].double()).abs().sum(1)
    assert bool(((got.weights.view(-1).double() - dots).abs() <= (H + 2) * EPS * size).all())
    again = bo.expert_combine_grad(dy, rows, d.order, d.position, w)
    assert torch.equal(again.rows, got.rows) and torch.equal(again.weights, got.weights)
