"""The two ends of a served or trained model and its expert layers, as cases
that can be timed and compared.

A language model's answers are scored from its last hidden rows and its output
matrix; an expert layer sends its tokens to the chosen experts' rows and back;
tokens enter by their rows of a table. Each case is a dict of plain values:

kind    "score"   log probability of the given tokens and entropy, straight
                  from hidden rows and output matrix, the logits not kept
        "score_train"  the same, then the gradients of both
        "experts" tokens into rows grouped by expert, and the experts' outputs
                  back under the router's weights
        "experts_train"  the same, then the gradients of all of it
        "embed"   rows of the table, scaled
        "embed_train"  the same, then the gradient of the table
type    "bf16", "f16" or "f32"
T       tokens
V, H    vocabulary, width of a row
pad     unused columns behind each row
top, E  experts per token, of so many; capacity: rows an expert takes at most

Padding tokens (without an id, half of them rows of zeros), pairs that no expert
took and tokens that were routed nowhere stand among the inputs where "masked" is
set; rows that no pair fills hold NaN.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
INF = float("inf")


def _sc(kind, T, V, H, type, pad=0, temperature=1.0, masked=True, name=None):
    c = dict(kind=kind, T=T, V=V, H=H, type=type, pad=pad, temperature=temperature, masked=masked)
    return dict(c, name=name) if name else c


def _ex(kind, T, H, top, E, type, pad=0, capacity=0, masked=True, name=None):
    c = dict(kind=kind, T=T, H=H, top=top, E=E, type=type, pad=pad, capacity=capacity, masked=masked)
    return dict(c, name=name) if name else c


def _em(kind, T, V, H, type, pad=0, scale=1.0, masked=True, name=None):
    c = dict(kind=kind, T=T, V=V, H=H, type=type, pad=pad, scale=scale, masked=masked)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step of one sequence: the output matrix is read once
        _sc("score", 1, 32000, 4096, "bf16", masked=False, name="score_one_token"),
        # one decoding step of a batch, at a temperature
        _sc("score", 64, 128000, 4096, "bf16", temperature=0.7, name="score_decode_batch"),
        # prompts scored over a large vocabulary
        _sc("score", 4096, 128000, 4096, "bf16", name="score_prompts"),
        # half precision, odd sizes, rows that start anywhere
        _sc("score", 2049, 50001, 1001, "f16", pad=2, name="score_ragged"),
        # a training step of a small model
        _sc("score_train", 8192, 32000, 2048, "bf16", name="score_train"),
        # a training step over a large vocabulary: logits would take 4 GB
        _sc("score_train", 8192, 128000, 4096, "bf16", name="score_train_large"),
        # single precision, odd sizes
        _sc("score_train", 1023, 20011, 515, "f32", temperature=1.5, name="score_train_ragged"),
        # one decoding step through an expert layer
        _ex("experts", 16, 4096, 8, 64, "bf16", masked=False, name="experts_decode"),
        # training an expert layer on a long batch
        _ex("experts_train", 32768, 2048, 8, 256, "bf16", name="experts_train"),
        # odd sizes, and experts that take no more than their share
        _ex("experts_train", 20011, 1111, 3, 61, "f16", pad=3, capacity=1000,
            name="experts_train_ragged"),
        # one decoding step of a batch enters the model
        _em("embed", 64, 128000, 4096, "f16", scale=64.0, name="embed_decode"),
        # training a table of embeddings: a few tokens are very frequent
        _em("embed_train", 32768, 128000, 2048, "bf16", name="embed_train"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    H = _log_int(rng, lo, hi)
    return H if rng.random() < 0.3 else max(8, H // 8 * 8)


def draw(rng):
    kind = rng.choice(["score", "score", "score_train", "score_train", "experts", "experts_train",
                       "embed", "embed_train"])
    type = rng.choice(["bf16", "bf16", "f16", "f32"])
    pad = rng.choice([0, 0, 0, 1, 8])
    masked = rng.random() < 0.7
    if kind.startswith("score"):
        V, H = _log_int(rng, 500, 128000), _width(rng, 32, 4096)
        most = 4e12 / (V * H) / (8 if type == "f32" else 1)
        T = _log_int(rng, 1, max(1, min(30000, 1e9 / V, most)))
        return _sc(kind, T, V, H, type, pad, rng.choice([1.0, 0.7, 1.5]), masked)
    if kind.startswith("experts"):
        E = _log_int(rng, 2, 256)
        top, H = min(E, rng.choice([1, 2, 4, 6, 8])), _width(rng, 64, 8192)
        T = _log_int(rng, 1, max(1, min(100000, 2.5e8 / (top * H))))
        return _ex(kind, T, H, top, E, type, pad, rng.choice([0, 0, max(1, T * top // E)]), masked)
    V, H = _log_int(rng, 500, 128000), _width(rng, 64, 4096)
    T = _log_int(rng, 1, max(1, min(200000, 2e8 / H)))
    return _em(kind, T, V, H, type, pad, rng.choice([1.0, 1.0, math.sqrt(H)]), masked)


# ---- inputs -----------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(n, every, at):
    """Rows at, at + every, .. (none where n has no such row)."""
    return torch.arange(min(at, n), n, every, device="cuda")


def _matrix(g, rows, cols, case, spread=1.0):
    """Normal values in rows of cols + pad; behind them NaN."""
    buf = torch.empty((rows, cols + case["pad"]), dtype=TYPES[case["type"]], device="cuda")
    buf.normal_(generator=g).mul_(spread)
    buf[:, cols:] = float("nan")
    return buf[:, :cols]


def _prepare_score(case, seed):
    """Hidden rows of unit size, logits with a spread of 2 and the given token
    up to 10 above that."""
    g = _gen(seed)
    T, V, H = case["T"], case["V"], case["H"]
    hidden = _matrix(g, T, H, case)
    weight = _matrix(g, V, H, case, 2.0 / math.sqrt(H))
    tokens = torch.randint(V, (T,), generator=g, device="cuda")
    lean = 2.5 * torch.rand((T, 1), generator=g, device="cuda")
    hidden.copy_(hidden + (lean * weight[tokens].float()).to(hidden.dtype))
    if case["masked"]:
        # padding: no token
        pad = _rows(T, 13, 8)
        tokens[pad] = -1
        hidden[pad[::2]] = 0.0
    s = dict(case=case, hidden=hidden, weight=weight, tokens=tokens)
    if case["kind"] == "score_train":
        s["grad_logprob"] = torch.randn(T, generator=g, device="cuda") / T
        s["grad_entropy"] = 0.1 * torch.randn(T, generator=g, device="cuda") / T
        if case["masked"]:
            s["grad_entropy"][pad] = 0.0
    return s


def _prepare_experts(case, seed):
    """Distinct experts per token, some far more popular than others, grouped
    with each expert's tokens in order; rows that nobody fills hold NaN."""
    g = _gen(seed)
    T, E, H, top = case["T"], case["E"], case["H"], case["top"]
    N = T * top
    noise = -torch.log(-torch.log(torch.rand((T, E), generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
    ids = (noise + 0.8 * torch.randn(E, generator=g, device="cuda")).topk(top, 1).indices
    if case["masked"]:
        ids[torch.rand((T, top), generator=g, device="cuda") < 0.02] = E
        ids[_rows(T, 101, 6)] = E
    e, by = ids.reshape(-1).sort(stable=True)
    load = torch.bincount(e, minlength=E + 1)
    rank = torch.arange(N, device="cuda") - (load.cumsum(0) - load)[e]
    goes = (e < E) & (rank < (case["capacity"] or N))
    kept = by[goes]
    order = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    order[:len(kept)] = kept.to(torch.int32)
    position = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    position[kept] = torch.arange(len(kept), device="cuda", dtype=torch.int32)
    rows = _matrix(g, N, H, case)
    rows[len(kept):] = float("nan")
    weights = torch.rand((T, top), generator=g, device="cuda")
    s = dict(case=case, x=_matrix(g, T, H, case), rows=rows, order=order,
             position=position.view(T, top), weights=weights / weights.sum(1, keepdim=True))
    if case["kind"] == "experts_train":
        s["grad"] = _matrix(g, T, H, case)                    # of the layer's outputs
        s["grad_grouped"] = _matrix(g, N, H, case)            # of the experts' inputs
        s["grad_grouped"][len(kept):] = float("nan")
    return s


def _prepare_embed(case, seed):
    """Tokens by a power of their rank, as in text; padding has none."""
    g = _gen(seed)
    T, V, H = case["T"], case["V"], case["H"]
    table = _matrix(g, V, H, case)
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    rank = (V ** u).long().clamp(max=V) - 1
    tokens = torch.randperm(V, generator=g, device="cuda")[rank]
    if case["masked"]:
        tokens[_rows(T, 13, 8)] = -1
    s = dict(case=case, tokens=tokens, table=table)
    if case["kind"] == "embed_train":
        s["grad"] = _matrix(g, T, H, case)
    return s


def prepare(case, seed):
    if case["kind"].startswith("score"):
        return _prepare_score(case, seed)
    return _prepare_experts(case, seed) if case["kind"].startswith("experts") else _prepare_embed(case, seed)


# ---- the operators in their plain form ---------------------------------------

def _plain_score(s):
    c, t = s["case"], s["tokens"]
    it, dt = 1.0 / c["temperature"], s["hidden"].dtype
    h, w = s["hidden"].float(), s["weight"].float()
    x = h @ w.T
    m = x.amax(1)
    d = (x - m[:, None]) * it
    e = torch.exp(d)
    total = e.sum(1)
    ls = torch.log(total)
    entropy = ls - (e * d).sum(1) / total
    has = t >= 0
    at = t.clamp(min=0)[:, None]
    lp = torch.where(has, d.gather(1, at)[:, 0] - ls, 0.0)
    out = dict(logprob=lp, entropy=entropy, stats=torch.stack([m, ls], 1))
    if c["kind"] == "score_train":
        gl, gh = torch.where(has, s["grad_logprob"], 0.0), s["grad_entropy"]
        d.sub_(ls[:, None])
        e.div_(total[:, None])
        g = e.mul_(-gl[:, None] - gh[:, None] * (d + entropy[:, None]))
        g.scatter_add_(1, at, gl[:, None])
        g.mul_(it)
        out["grad_hidden"] = (g @ w).to(dt)
        out["grad_weight"] = (g.T @ h).to(dt)
    return out


def _plain_experts(s):
    c = s["case"]
    dt, T, top, N = s["x"].dtype, c["T"], c["top"], c["T"] * c["top"]
    order, position = s["order"].long(), s["position"].long()
    filled, there = order >= 0, position >= 0
    owner = order.clamp(min=0) // top
    grouped = torch.where(filled[:, None], s["x"][owner], 0.0).to(dt)

    def back(rows, weights):
        total = torch.zeros((T, c["H"]), device=rows.device)
        for k in range(top):
            row = rows[position[:, k].clamp(min=0)].float()
            on = there[:, k:k + 1]
            total += torch.where(on, row if weights is None else weights[:, k:k + 1] * row, 0.0)
        return total

    out = dict(grouped=grouped, combined=back(s["rows"], s["weights"]).to(dt))
    if c["kind"] == "experts_train":
        w = s["weights"].reshape(-1)[order.clamp(min=0)]
        g = s["grad"].float()
        out["grad_rows"] = torch.where(filled[:, None], w[:, None] * g[owner], 0.0).to(dt)
        dots = [(g * s["rows"][position[:, k].clamp(min=0)].float()).sum(1) for k in range(top)]
        out["grad_weights"] = torch.where(there, torch.stack(dots, 1), 0.0)
        out["grad_x"] = back(s["grad_grouped"], None).to(dt)
    return out


def _plain_embed(s):
    c, t = s["case"], s["tokens"]
    has = (t >= 0)[:, None]
    rows = torch.where(has, c["scale"] * s["table"][t.clamp(min=0)].float(), 0.0)
    out = dict(rows=rows.to(s["table"].dtype))
    if c["kind"] == "embed_train":
        g = torch.zeros((c["V"] + 1, c["H"]), device=t.device)
        g.index_add_(0, torch.where(t >= 0, t, c["V"]), s["grad"].float())
        out["grad_table"] = (c["scale"] * g[:c["V"]]).to(s["table"].dtype)
    return out


def _plain(s):
    kind = s["case"]["kind"]
    if kind.startswith("score"):
        return _plain_score(s)
    return _plain_experts(s) if kind.startswith("experts") else _plain_embed(s)


# ---- the framework's operators -------------------------------------------------

def _own(s):
    import paper_2602_10729_amd as bo
    c = s["case"]
    if c["kind"].startswith("score"):
        it = 1.0 / c["temperature"]
        r = bo.linear_logprobs(s["hidden"], s["weight"], s["tokens"], inv_temperature=it)
        out = dict(logprob=r.logprob, entropy=r.entropy, stats=r.stats)
        if c["kind"] == "score_train":
            g = bo.linear_logprobs_grad(s["hidden"], s["weight"], s["tokens"], r.stats, r.entropy,
                                        s["grad_logprob"], s["grad_entropy"], inv_temperature=it)
            out.update(grad_hidden=g.hidden, grad_weight=g.weight)
        return out
    if c["kind"].startswith("experts"):
        out = dict(grouped=bo.expert_gather(s["x"], s["order"], s["position"]),
                   combined=bo.expert_combine(s["rows"], s["position"], s["weights"]))
        if c["kind"] == "experts_train":
            g = bo.expert_combine_grad(s["grad"], s["rows"], s["order"], s["position"], s["weights"])
            out.update(grad_rows=g.rows, grad_weights=g.weights,
                       grad_x=bo.expert_combine(s["grad_grouped"], s["position"]))
        return out
    out = dict(rows=bo.embed(s["tokens"], s["table"], scale=c["scale"]))
    if c["kind"] == "embed_train":
        out["grad_table"] = bo.embed_grad(s["tokens"], s["grad"], c["V"], scale=c["scale"])
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------

def work(case):
    T, H = case["T"], case["H"]
    es = 4 if case["type"] == "f32" else 2
    train = case["kind"].endswith("train")
    if case["kind"].startswith("score"):
        V = case["V"]
        b = (T + V) * H * es + T * 24
        if train:
            b += (T + V) * H * es + T * 8
        return {"bytes": b, "flops": T * V * (2 * H + 8) + (T * V * (4 * H + 6) if train else 0)}
    if case["kind"].startswith("experts"):
        N = T * case["top"]
        b = 2 * (T + N) * H * es + 12 * N
        if train:
            b += (T + 2 * N) * H * es + (N + T) * H * es + 12 * N
        return {"bytes": b, "flops": (2 + (4 if train else 0)) * N * H}
    b = T * (8 + 2 * H * es)
    if train:
        b += T * H * es + case["V"] * H * es
    return {"bytes": b, "flops": T * H * (2 if train else 1)}


# ---- 64 bits ----------------------------------------------------------------------

def _exact_score(case, s):
    """Row blocks in float64; the gradients by differentiating the definition."""
    T, V, it = case["T"], case["V"], 1.0 / case["temperature"]
    train = case["kind"] == "score_train"
    weight = s["weight"].double().requires_grad_(train)
    parts = {n: [] for n in ("logprob", "entropy", "stats") + (("grad_hidden",) if train else ())}
    block = max(1, 250_000_000 // V)
    for a in range(0, T, block):
        h = s["hidden"][a:a + block].double().requires_grad_(train)
        tok = s["tokens"][a:a + block]
        logits = h @ weight.t()
        lsm = torch.log_softmax(logits * it, 1)
        given = lsm[torch.arange(len(tok), device="cuda"), tok.clamp(min=0)].masked_fill(tok < 0, 0.0)
        entropy = -(lsm.exp() * lsm).sum(1)
        m = logits.detach().amax(1)
        parts["logprob"].append(given.detach())
        parts["entropy"].append(entropy.detach())
        parts["stats"].append(torch.stack([m, torch.logsumexp(logits.detach() * it, 1) - m * it], 1))
        if train:
            ((given * s["grad_logprob"][a:a + block].double()).sum()
             + (entropy * s["grad_entropy"][a:a + block].double()).sum()).backward()
            parts["grad_hidden"].append(h.grad)
        del h, logits, lsm, given, entropy
    out = {n: torch.cat(v) for n, v in parts.items()}
    if train:
        out["grad_weight"] = weight.grad
    return out


def _exact_experts(case, s):
    """The layer as one function of its inputs, differentiated: a token's rows
    by the pairs that were taken."""
    T, H, top = case["T"], case["H"], case["top"]
    train = case["kind"] == "experts_train"
    taken = int((s["order"] >= 0).sum())
    pair = s["order"][:taken].long()
    x = s["x"].double().requires_grad_(train)
    rows = s["rows"][:taken].double().requires_grad_(train)
    weights = s["weights"].double().requires_grad_(train)

    def whole(t):
        return torch.cat([t, t.new_zeros((T * top - taken, H))])

    grouped = x.index_select(0, pair.div(top, rounding_mode="floor"))
    weighted = rows * weights.reshape(-1).index_select(0, pair)[:, None]
    combined = torch.zeros((T, H), dtype=torch.float64, device="cuda").index_add(
        0, pair.div(top, rounding_mode="floor"), weighted)
    out = dict(grouped=whole(grouped.detach()), combined=combined.detach())
    if train:
        combined.backward(s["grad"].double())
        grouped.backward(s["grad_grouped"][:taken].double())
        out.update(grad_rows=whole(rows.grad), grad_weights=weights.grad, grad_x=x.grad)
    return out


def _exact_embed(case, s):
    train = case["kind"] == "embed_train"
    table = s["table"].double()
    live = (s["tokens"] >= 0).nonzero()[:, 0]
    rows = torch.zeros((case["T"], case["H"]), dtype=torch.float64, device="cuda")
    rows[live] = table[s["tokens"][live]] * case["scale"]
    out = dict(rows=rows)
    if train:
        grad = torch.zeros_like(table)
        grad.index_put_((s["tokens"][live],), s["grad"][live].double() * case["scale"], accumulate=True)
        out["grad_table"] = grad
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("score"):
        return _exact_score(case, s)
    return _exact_experts(case, s) if case["kind"].startswith("experts") else _exact_embed(case, s)
