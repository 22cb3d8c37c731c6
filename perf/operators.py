"""What turns a served model's outputs into assignments, as cases that can be
timed and compared.

A search over routing thresholds works on scores and loads: the log
probabilities of an answer's tokens score it, a router sends each query (or
each token of an expert model) to its best models under a bias that balances
their loads, and the assignments are grouped by model. Each case is a dict of
plain values:

kind    "logprobs"   log probability, rank, entropy and top alternatives of the
                     given tokens
        "logprobs_train"  the same, then the gradient of the logits
        "route"      scores to experts: the chosen ones and their weights
        "route_train"  the same, then the gradient of the router's logits
        "dispatch"   the chosen pairs grouped by expert
type    "bf16", "f16" or "f32"
T       rows (tokens or queries)
V, pad  vocabulary, and unused columns behind it
E       experts
top     alternatives returned, or experts chosen per row

Rows that a mask leaves nothing, masks of minus infinity and of the type's
lowest value, rows without a token and experts withdrawn by an infinite bias
stand among the inputs where "masked" is set.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
INF = float("inf")


def _lp(kind, T, V, type, top, pad=0, temperature=1.0, masked=True, name=None):
    c = dict(kind=kind, T=T, V=V, type=type, top=top, pad=pad, temperature=temperature, masked=masked)
    return dict(c, name=name) if name else c


def _rt(kind, T, E, top, type, score, bias=False, groups=1, top_groups=1, group_best=1,
        renormalise=True, scale=1.0, masked=True, name=None):
    c = dict(kind=kind, T=T, E=E, top=top, type=type, score=score, bias=bias, groups=groups,
             top_groups=top_groups, group_best=group_best, renormalise=renormalise, scale=scale,
             masked=masked)
    return dict(c, name=name) if name else c


def _dp(T, top, E, capacity=0, masked=True, name=None):
    c = dict(kind="dispatch", T=T, top=top, E=E, capacity=capacity, masked=masked)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step of one sequence: latency is what counts
        _lp("logprobs", 1, 32000, "bf16", 5, masked=False, name="logprobs_one_token"),
        # one decoding step of a batch, at a temperature, alternatives asked for
        _lp("logprobs", 64, 128000, "bf16", 20, temperature=0.7, name="logprobs_decode_batch"),
        # prompts scored in single precision, an odd vocabulary in padded rows
        _lp("logprobs", 2049, 50001, "f32", 8, pad=15, name="logprobs_ragged"),
        # a whole trace's answers scored at once: past 2^31 logits
        _lp("logprobs", 16897, 128000, "bf16", 1, name="logprobs_trace"),
        # a training step on an ordinary batch of tokens
        _lp("logprobs_train", 8192, 32000, "bf16", 0, name="logprobs_train"),
        # distillation onto the alternatives, odd sizes, half precision
        _lp("logprobs_train", 1023, 100003, "f16", 4, pad=5, temperature=2.0,
            name="logprobs_train_ragged"),
        # one decoding step through an expert layer
        _rt("route", 16, 64, 6, "f32", "softmax", masked=False, name="route_decode"),
        # a prompt through an expert layer: balance bias, groups, sigmoid scores
        _rt("route", 32768, 256, 8, "bf16", "sigmoid", bias=True, groups=8, top_groups=4,
            group_best=2, scale=2.5, name="route_prompt_groups"),
        # training a router over an odd number of experts
        _rt("route_train", 65537, 61, 4, "f32", "softmax", renormalise=False,
            name="route_train_ragged"),
        # training a router of queries over three served models
        _rt("route_train", 500000, 3, 2, "f32", "sigmoid", bias=True, masked=False,
            name="route_train_models"),
        # grouping one decoding step's choices
        _dp(32, 8, 256, name="dispatch_decode"),
        # grouping a long trace's choices, with a capacity per expert
        _dp(262144, 8, 256, capacity=10000, name="dispatch_trace"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprobs", "logprobs", "logprobs_train", "route", "route_train", "dispatch"])
    if kind.startswith("logprobs"):
        V = _log_int(rng, 1000, 200000)
        T = _log_int(rng, 1, min(30000, 6e8 / V))
        return _lp(kind, T, V, rng.choice(["bf16", "f16", "f32"]), rng.choice([0, 1, 5, 20, 33]),
                   pad=rng.choice([0, 0, 1, 8, 64]), temperature=rng.choice([1.0, 0.7, 1.5]),
                   masked=rng.random() < 0.7)
    E = _log_int(rng, 2, 512)
    top = min(E, rng.choice([1, 2, 4, 6, 8, 10]))
    T = _log_int(rng, 1, min(500000, 3e7 / E))
    if kind == "dispatch":
        return _dp(T, top, E, capacity=rng.choice([0, 0, max(1, T * top // E)]),
                   masked=rng.random() < 0.7)
    groups = rng.choice([g for g in (1, 1, 2, 4, 8) if E % g == 0 and E // g >= 2] or [1])
    top_groups = rng.randint(1, groups)
    return _rt(kind, T, E, min(top, top_groups * (E // groups)), rng.choice(["bf16", "f16", "f32"]),
               rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.6, groups=groups,
               top_groups=top_groups, group_best=rng.choice([1, 2]) if E // groups >= 2 else 1,
               renormalise=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]),
               masked=rng.random() < 0.7)


# ---- inputs -----------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(T, every, at):
    """Rows at, at + every, .. (none where T has no such row)."""
    return torch.arange(min(at, T), T, every, device="cuda")


def _prepare_logprobs(case, seed):
    """Logits as a language model gives them: a spread of a few units and, in
    each row, one token that stands out by up to 12; the given token is that
    one more often than not."""
    g = _gen(seed)
    T, V, dt = case["T"], case["V"], TYPES[case["type"]]
    buf = torch.empty((T, V + case["pad"]), dtype=dt, device="cuda")
    buf.normal_(generator=g).mul_(2.0)
    buf[:, V:] = float("nan")
    x = buf[:, :V]
    rows = torch.arange(T, device="cuda")
    best = torch.randint(V, (T,), generator=g, device="cuda")
    x[rows, best] = x[rows, best] + (12.0 * torch.rand(T, generator=g, device="cuda")).to(dt)
    tokens = torch.where(torch.rand(T, generator=g, device="cuda") < 0.6, best,
                         torch.randint(V, (T,), generator=g, device="cuda"))
    if case["masked"]:
        # constrained decoding: most tokens masked in every fourth row, now and
        # then by the type's lowest value; padding rows have no token, and some
        # rows nothing at all
        cut = torch.rand((len(range(3, T, 4)), V), generator=g, device="cuda") < 0.9
        x[3::4].masked_fill_(cut, -INF)
        cut = torch.rand((len(range(5, T, 64)), V), generator=g, device="cuda") < 0.5
        x[5::64].masked_fill_(cut, torch.finfo(dt).min)
        r = _rows(T, 64, 5)
        x[r, best[r]] = 6.0
        tokens[r] = best[r]
        x[_rows(T, 97, 9)] = -INF
        tokens[_rows(T, 13, 8)] = -1
    s = dict(case=case, logits=x, tokens=tokens)
    if case["kind"] == "logprobs_train":
        s["grad_logprob"] = torch.randn(T, generator=g, device="cuda")
        s["grad_entropy"] = 0.1 * torch.randn(T, generator=g, device="cuda")
        s["grad_top"] = torch.randn((T, case["top"]), generator=g, device="cuda")
    return s


def _choice_gaps(case, logits, bias):
    """Per row, the smallest distance above zero between two values that the
    choice of groups and experts compares, over the largest of them (64 bits)."""
    T, E, G = case["T"], case["E"], case["groups"]
    l = logits.double()
    if case["score"] == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-l))
    else:
        s = torch.exp(l - l.amax(1, keepdim=True).clamp_min(-1e30))
        s = s / s.sum(1, keepdim=True).clamp_min(1e-300)
    v = s if bias is None else s + bias.double()
    v = torch.where(l == -INF, -INF, v)
    size = v.abs().masked_fill(v == -INF, 0.0).amax(1, keepdim=True).clamp_min(1e-300)

    def least(u):
        if u.shape[1] < 2:
            return torch.full((T,), INF, device="cuda", dtype=torch.float64)
        d = u[:, :-1] - u[:, 1:]
        return torch.where(d > 0, d / size, INF).amin(1)

    gap = torch.full((T,), INF, device="cuda", dtype=torch.float64)
    if G > 1:
        gv = v.view(T, G, E // G).sort(2, descending=True).values[:, :, :case["group_best"]].sum(2)
        gv, at = gv.sort(dim=1, descending=True, stable=True)
        gap = least(gv)
        keep = torch.zeros((T, G), dtype=torch.bool, device="cuda")
        keep.scatter_(1, at[:, :case["top_groups"]], True)
        v = torch.where(keep.repeat_interleave(E // G, 1), v, -INF)
    if bias is not None:
        gap = torch.minimum(gap, least(v.sort(1, descending=True).values[:, :case["top"] + 1]))
    return gap


def _prepare_route(case, seed):
    """A router's logits: experts of unequal popularity, a bias that balances
    them. Which expert comes first must not hang on the last bits of a score:
    a row where it does is given another row's logits."""
    g = _gen(seed)
    T, E, dt = case["T"], case["E"], TYPES[case["type"]]
    l = torch.randn((T, E), generator=g, device="cuda")
    l = (l + 0.5 * torch.randn(E, generator=g, device="cuda")).to(dt)
    bias = None
    if case["bias"]:
        spread = 0.05 if case["score"] == "sigmoid" else 0.25 / E
        bias = spread * torch.randn(E, generator=g, device="cuda")
        if case["masked"] and E > 4:
            bias[E // 3] = -INF
    if case["masked"]:
        cut = torch.rand((len(range(2, T, 7)), E), generator=g, device="cuda") < 0.4
        l[2::7] = l[2::7].masked_fill(cut, -INF)
    if bias is not None or case["groups"] > 1:
        ok = _choice_gaps(case, l, bias) > 4e-6
        if not bool(ok.any()):
            l[0] = torch.linspace(2.0, -2.0, E, device="cuda").to(dt)
            ok[0] = True
        other = ok.nonzero()[:, 0]
        take = other[torch.arange(T, device="cuda") % len(other)]
        l = torch.where(ok[:, None], l, l[take])
    if case["masked"]:
        l[_rows(T, 101, 6)] = -INF
    s = dict(case=case, logits=l.contiguous(), bias=bias)
    if case["kind"] == "route_train":
        s["grad_weights"] = torch.randn((T, case["top"]), generator=g, device="cuda")
    return s


def _prepare_dispatch(case, seed):
    """Distinct experts per token, some far more popular than others; tokens
    that were routed nowhere hold -1."""
    g = _gen(seed)
    T, E = case["T"], case["E"]
    noise = -torch.log(-torch.log(torch.rand((T, E), generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
    ids = (noise + 0.8 * torch.randn(E, generator=g, device="cuda")).topk(case["top"], 1).indices
    ids = ids.to(torch.int32)
    if case["masked"]:
        ids[torch.rand((T, case["top"]), generator=g, device="cuda") < 0.02] = -1
        ids[_rows(T, 101, 6)] = -1
    return dict(case=case, ids=ids.contiguous())


def prepare(case, seed):
    if case["kind"].startswith("logprobs"):
        return _prepare_logprobs(case, seed)
    if case["kind"].startswith("route"):
        return _prepare_route(case, seed)
    return _prepare_dispatch(case, seed)


# ---- the operators in their plain form ---------------------------------------

def _plain_logprobs(s):
    c, t = s["case"], s["tokens"]
    k, it, V = c["top"], 1.0 / c["temperature"], c["V"]
    x = s["logits"].float()
    m = x.amax(1)
    dead = x == -INF
    d = torch.where(dead, 0.0, (x - m[:, None]) * it)
    e = torch.where(dead, 0.0, torch.exp(d))
    total = e.sum(1)
    ls = torch.log(total)
    entropy = torch.where(m == -INF, 0.0, ls - torch.where(e == 0, 0.0, e * d).sum(1) / total)
    has = t >= 0
    xt = x.gather(1, t.clamp(min=0)[:, None])
    lp = torch.where(xt[:, 0] == -INF, -INF, (xt[:, 0] - m) * it - ls)
    col = torch.arange(V, device=x.device)
    ahead = (x > xt).sum(1) + ((x == xt) & (col < t[:, None])).sum(1)
    out = dict(logprob=torch.where(has, lp, 0.0), entropy=entropy,
               rank=torch.where(has & (xt[:, 0] > -INF), ahead + 1, 0).to(torch.int32),
               stats=torch.stack([m, ls], 1))
    ids = None
    if k > 0:
        # order by (value, lowest index): the value's bits above the index's
        b = (x + 0.0).view(torch.int32).long()
        key = torch.where(b < 0, b ^ 0x7FFFFFFF, b) * (1 << 32) + ((1 << 32) - 1 - col)
        ids = (1 << 32) - 1 - (key.topk(k, 1).values & ((1 << 32) - 1))
        xk = x.gather(1, ids)
        ids = torch.where(xk > -INF, ids, -1)
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprobs"] = torch.where(xk > -INF, (xk - m[:, None]) * it - ls[:, None], -INF)
    if c["kind"] == "logprobs_train":
        gl = torch.where(has, s["grad_logprob"], 0.0)
        gh = s["grad_entropy"]
        g = torch.zeros((c["T"], V + 1), device=x.device)
        g.scatter_add_(1, torch.where(has, t, V)[:, None], gl[:, None])
        gsum = gl
        if k > 0:
            gt = torch.where(ids >= 0, s["grad_top"], 0.0)
            g.scatter_add_(1, torch.where(ids >= 0, ids, V), gt)
            gsum = gl + gt.sum(1)
        u = d - ls[:, None]
        p = torch.where(dead, 0.0, e / total[:, None])
        dense = torch.where(p == 0, 0.0, p * (-gsum[:, None] - gh[:, None] * (u + entropy[:, None])))
        grad = it * (g[:, :V] + dense)
        out["grad_logits"] = torch.where(m[:, None] == -INF, 0.0, grad).to(s["logits"].dtype)
    return out


def _plain_route(s):
    c, bias = s["case"], s["bias"]
    T, E, k, G = c["T"], c["E"], c["top"], c["groups"]
    l = s["logits"].float()
    dead = l == -INF
    if c["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-l))
    else:
        m = l.amax(1, keepdim=True)
        e = torch.where(dead, 0.0, torch.exp(l - m))
        score = torch.where(m == -INF, 0.0, e / e.sum(1, keepdim=True))
    biased = score if bias is None else score + bias
    biased = torch.where(dead, -INF, biased)
    value = l if bias is None else biased
    if G > 1:
        gv = biased.view(T, G, E // G).sort(2, descending=True).values[:, :, :c["group_best"]].sum(2)
        at = gv.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device=l.device).scatter_(1, at, True)
        value = torch.where(keep.repeat_interleave(E // G, 1), value, -INF)
    value, ids = value.sort(dim=1, descending=True, stable=True)
    value, ids = value[:, :k], ids[:, :k]
    there = value > -INF
    chosen = torch.where(there, score.gather(1, ids), 0.0)
    total = chosen.sum(1, keepdim=True)
    w = chosen
    if c["renormalise"]:
        w = torch.where(there, chosen / torch.where(total > 0, total, 1.0), 0.0)
    out = dict(ids=torch.where(there, ids, -1).to(torch.int32), weights=c["scale"] * w)
    if c["kind"] == "route_train":
        g = torch.where(there, s["grad_weights"], 0.0) * c["scale"]
        if c["renormalise"]:
            ds = (g - (g * w).sum(1, keepdim=True)) / torch.where(total > 0, total, 1.0)
        else:
            ds = g
        if c["score"] == "sigmoid":
            dl = torch.where(there, ds * chosen * (1.0 - chosen), 0.0)
            grad = torch.zeros_like(l).scatter_add_(1, ids, dl)
        else:
            inner = 0.0 if c["renormalise"] else (ds * chosen).sum(1, keepdim=True)
            grad = -score * inner
            grad = grad.scatter_add(1, ids, torch.where(there, ds * chosen, 0.0))
        out["grad_logits"] = grad.to(s["logits"].dtype)
    return out


def _plain_dispatch(s):
    c = s["case"]
    E, N = c["E"], c["T"] * c["top"]
    flat = s["ids"].reshape(-1).long()
    flat = torch.where((flat >= 0) & (flat < E), flat, E)
    load = torch.zeros(E + 1, dtype=torch.int64, device=flat.device)
    load.scatter_add_(0, flat, torch.ones_like(flat))
    e, order = flat.sort(stable=True)
    rank = torch.arange(N, device=flat.device) - (load.cumsum(0) - load)[e]
    kept = load[:E].clamp(max=c["capacity"]) if c["capacity"] else load[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=flat.device)
    offsets[1:] = kept.cumsum(0)
    goes = (e < E) & (rank < c["capacity"]) if c["capacity"] else e < E
    place = offsets[e] + rank
    grouped = torch.full((N + 1,), -1, dtype=torch.int64, device=flat.device)
    grouped.scatter_(0, torch.where(goes, place, N), torch.where(goes, order, -1))
    position = torch.empty(N, dtype=torch.int64, device=flat.device)
    position.scatter_(0, order, torch.where(goes, place, -1))
    i32 = torch.int32
    return dict(load=load[:E].to(i32), offsets=offsets.to(i32), order=grouped[:N].to(i32),
                position=position.view(c["T"], c["top"]).to(i32))


def _plain(s):
    kind = s["case"]["kind"]
    if kind.startswith("logprobs"):
        return _plain_logprobs(s)
    return _plain_route(s) if kind.startswith("route") else _plain_dispatch(s)


# ---- the framework's operators -------------------------------------------------

def _own(s):
    import paper_2602_10729_amd as bo
    c = s["case"]
    if c["kind"].startswith("logprobs"):
        it = 1.0 / c["temperature"]
        r = bo.token_logprobs(s["logits"], s["tokens"], top=c["top"], inv_temperature=it)
        out = dict(logprob=r.logprob, entropy=r.entropy, rank=r.rank, stats=r.stats)
        if c["top"]:
            out.update(top_ids=r.top_ids, top_logprobs=r.top_logprobs)
        if c["kind"] == "logprobs_train":
            out["grad_logits"] = bo.token_logprobs_grad(
                s["logits"], s["tokens"], r.stats, r.entropy, s["grad_logprob"], s["grad_entropy"],
                top_ids=r.top_ids if c["top"] else None,
                grad_top=s["grad_top"] if c["top"] else None, inv_temperature=it)
        return out
    if c["kind"].startswith("route"):
        how = dict(score=c["score"], renormalise=c["renormalise"], scale=c["scale"])
        r = bo.route(s["logits"], c["top"], bias=s["bias"], groups=c["groups"],
                     top_groups=c["top_groups"], group_best=c["group_best"], **how)
        out = dict(ids=r.ids, weights=r.weights)
        if c["kind"] == "route_train":
            out["grad_logits"] = bo.route_grad(s["logits"], r.ids, s["grad_weights"], **how)
        return out
    r = bo.dispatch(s["ids"], c["E"], capacity=c["capacity"])
    return dict(load=r.load, offsets=r.offsets, order=r.order, position=r.position)


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------

def work(case):
    T, k = case["T"], case["top"]
    if case["kind"] == "dispatch":
        N = T * k
        return {"bytes": 12 * N + 8 * case["E"], "flops": 2 * N}
    es = 4 if case["type"] == "f32" else 2
    train = case["kind"].endswith("train")
    if case["kind"].startswith("logprobs"):
        n = T * case["V"]
        b = n * es + T * (8 + 20 + 8 * k)
        if train:
            b += n * es + T * (8 + 4 * k)
        return {"bytes": b, "flops": n * (14 if train else 8)}
    n = T * case["E"]
    b = n * es + 8 * T * k + (4 * case["E"] if case["bias"] else 0)
    if train:
        b += n * es + 4 * T * k
    return {"bytes": b, "flops": n * (12 if train else 8)}


# ---- 64 bits ----------------------------------------------------------------------

def _exact_logprobs(case, s):
    """Row blocks in float64; the gradient by differentiating the definition.
    Masked logits take a value so low that their probability is exactly 0."""
    T, V, k, it = case["T"], case["V"], case["top"], 1.0 / case["temperature"]
    names = ["logprob", "entropy", "stats"] + (["top_logprobs"] if k else [])
    train = case["kind"] == "logprobs_train"
    parts = {n: [] for n in names + (["grad_logits"] if train else [])}
    block = max(1, 40_000_000 // V)
    for a in range(0, T, block):
        raw = s["logits"][a:a + block].double()
        tok = s["tokens"][a:a + block]
        n = raw.shape[0]
        empty = (raw == -INF).all(1)
        low = raw.masked_fill(raw == -INF, -1e30).requires_grad_(train)
        lsm = torch.log_softmax(low * it, 1)
        given = lsm[torch.arange(n, device="cuda"), tok.clamp(min=0)]
        entropy = -(lsm.exp() * lsm).sum(1)
        given_ok = tok >= 0
        masked = raw[torch.arange(n, device="cuda"), tok.clamp(min=0)] == -INF
        lp = given.detach().masked_fill(masked, -INF).masked_fill(~given_ok, 0.0)
        m = raw.amax(1)
        ls = torch.logsumexp(low.detach() * it, 1) - m * it
        parts["logprob"].append(lp)
        parts["entropy"].append(entropy.detach().masked_fill(empty, 0.0))
        parts["stats"].append(torch.stack([m, ls.masked_fill(empty, -INF)], 1))
        if k:
            val, at = raw.sort(dim=1, descending=True, stable=True)
            val, at = val[:, :k], at[:, :k]
            alt = lsm.gather(1, at)
            parts["top_logprobs"].append(alt.detach().masked_fill(val == -INF, -INF))
        if train:
            total = (given * s["grad_logprob"][a:a + block].double()).masked_fill(~given_ok, 0.0).sum()
            total = total + (entropy * s["grad_entropy"][a:a + block].double()).sum()
            if k:
                total = total + (alt * s["grad_top"][a:a + block].double()).masked_fill(
                    val == -INF, 0.0).sum()
            total.backward()
            parts["grad_logits"].append(low.grad.masked_fill(empty[:, None], 0.0))
    out = {n: torch.cat(v) for n, v in parts.items()}
    out["rank"] = None
    if k:
        out["top_ids"] = None
    return out


def _exact_route(case, s):
    T, E, k, G = case["T"], case["E"], case["top"], case["groups"]
    raw, bias = s["logits"].double(), s["bias"]
    train = case["kind"] == "route_train"
    low = raw.masked_fill(raw == -INF, -1e30).requires_grad_(train)
    score = torch.sigmoid(low) if case["score"] == "sigmoid" else torch.softmax(low, 1)
    v = score.detach() + (0.0 if bias is None else bias.double())
    v = v.masked_fill(raw == -INF, -INF)
    rank_by = raw if bias is None else v
    if G > 1:
        gv = v.view(T, G, E // G).topk(case["group_best"], 2).values.sum(2)
        at = gv.argsort(dim=1, descending=True, stable=True)
        place = torch.empty_like(at).scatter_(1, at, torch.arange(G, device="cuda").expand(T, G))
        out_of = (place >= case["top_groups"]).repeat_interleave(E // G, 1)
        rank_by = rank_by.masked_fill(out_of, -INF)
    val, ids = rank_by.sort(dim=1, descending=True, stable=True)
    there = val[:, :k] > -INF
    w = score.gather(1, ids[:, :k]) * there
    if case["renormalise"]:
        w = w / (w.sum(1, keepdim=True) + (~there.any(1, keepdim=True)).double())
    w = w * case["scale"]
    out = dict(ids=None, weights=w.detach())
    if train:
        (w * s["grad_weights"].double()).sum().backward()
        out["grad_logits"] = low.grad.masked_fill((raw == -INF).all(1, keepdim=True), 0.0)
    return out


def exact(case, seed):
    if case["kind"] == "dispatch":
        return None
    s = prepare(case, seed)
    return _exact_logprobs(case, s) if case["kind"].startswith("logprobs") else _exact_route(case, s)
