"""fp64 references of the served-output operators: log probabilities of given
tokens (from logits, or from hidden rows and an output matrix), routing to
experts, the grouping of choices by expert, the experts' rows, and embeddings.

Written row by row from the definitions; logits come in whatever precision the
caller has and are taken at their exact values. -inf masks a logit; a row whose
every logit is masked has no distribution (log probability -inf, rank 0,
entropy 0, gradient 0).
"""
from __future__ import annotations

import numpy as np

INF = np.inf


def _live(x):
    return x[x != -INF]


def token_logprobs(logits, tokens, top=0, inv_temperature=1.0):
    """dict(logprob, rank, entropy, stats, top_ids, top_logprobs, spread):
    spread is the mean distance of a logit from the largest (scaled), the
    factor by which the entropy's rounding grows."""
    l = np.asarray(logits, dtype=np.float64)
    T, V = l.shape
    it = float(np.float32(inv_temperature))
    out = dict(logprob=np.zeros(T), rank=np.zeros(T, np.int64), entropy=np.zeros(T),
               stats=np.full((T, 2), -INF), top_ids=np.full((T, top), -1, np.int64),
               top_logprobs=np.full((T, top), -INF), spread=np.zeros(T))
    for r in range(T):
        row, tok = l[r], int(tokens[r]) if tokens is not None else -1
        bad = bool(np.isnan(row).any() or (row == INF).any())
        live = _live(row)
        live = live[~np.isnan(live)]
        has = 0 <= tok < V
        order = np.lexsort((np.arange(V), -np.where(np.isnan(row), -INF, row)))
        order = [j for j in order[:top] if row[j] > -INF]
        out["top_ids"][r, :len(order)] = order
        if has and row[tok] > -INF:
            out["rank"][r] = 1 + np.sum(row > row[tok]) + np.sum(row[:tok] == row[tok])
        if bad:
            out["stats"][r] = (live.max() if live.size else -INF, np.nan)
            out["entropy"][r] = np.nan
            out["top_logprobs"][r, :len(order)] = np.nan
            out["logprob"][r] = np.nan if tok >= 0 else 0.0
            continue
        if live.size:
            m = live.max()
            d = (live - m) * it
            e = np.exp(d)
            s = e.sum()
            ls = np.log(s)
            dp = np.where(e > 0, d, 0.0)
            out["stats"][r] = (m, ls)
            out["entropy"][r] = ls - (e * dp).sum() / s
            out["spread"][r] = -(e * dp).sum() / s
            out["top_logprobs"][r, :len(order)] = (row[order] - m) * it - ls
        if has:
            out["logprob"][r] = (row[tok] - m) * it - ls if row[tok] > -INF else -INF
        elif tok >= V:
            out["logprob"][r] = np.nan
    return out


def token_logprobs_grad(logits, tokens, g_logprob=None, g_entropy=None, top_ids=None, g_top=None,
                        inv_temperature=1.0):
    """Gradient of sum(g_logprob logprob + g_entropy entropy + g_top
    top_logprobs) with respect to the logits, the ids held fixed."""
    l = np.asarray(logits, dtype=np.float64)
    T, V = l.shape
    it = float(np.float32(inv_temperature))
    f = token_logprobs(l, tokens, 0, inv_temperature)
    grad = np.zeros((T, V))
    for r in range(T):
        m, ls = f["stats"][r]
        if m == -INF and not np.isnan(ls):
            continue
        tok = int(tokens[r]) if tokens is not None else -1
        u = (l[r] - m) * it - ls
        p = np.exp(u)
        lin = np.where(p == 0, 0.0, u)
        gh = 0.0 if g_entropy is None else float(g_entropy[r])
        gl = 0.0 if g_logprob is None or tok < 0 else float(g_logprob[r])
        hot = np.zeros(V)
        total = gl
        if 0 <= tok < V:
            hot[tok] += gl
        if top_ids is not None:
            for i, j in enumerate(top_ids[r]):
                if 0 <= j < V:
                    hot[j] += float(g_top[r, i])
                    total += float(g_top[r, i])
        grad[r] = it * (hot - p * total - gh * p * (lin + f["entropy"][r]))
        if tok >= V:
            grad[r] = np.nan
    return grad


def _scores(row, score):
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-row))
    if np.isnan(row).any() or (row == INF).any():
        return np.full(row.shape, np.nan)
    m = row.max()
    if m == -INF:
        return np.zeros(row.shape)
    e = np.exp(row - m)
    return e / e.sum()


def route(logits, top, bias=None, score="softmax", groups=1, top_groups=1, group_best=1,
          renormalise=True, scale=1.0):
    """dict(ids, weights, gap): gap is, per row, the least distance above zero
    between two values whose order decides the choice (over the largest of
    them), inf where only exact comparisons decide."""
    l = np.asarray(logits, dtype=np.float64)
    T, E = l.shape
    ids = np.full((T, top), -1, np.int64)
    weights = np.zeros((T, top))
    gaps = np.full(T, INF)
    for r in range(T):
        s = _scores(l[r], score)
        v = s if bias is None else s + np.asarray(bias, dtype=np.float64)
        off = ~(l[r] > -INF) | np.isnan(v) | ~(v > -INF)
        v = np.where(off, -INF, v)
        by = np.where(off, -INF, l[r]) if bias is None else v
        fin = np.abs(v[np.isfinite(v)])
        size = max(fin.max() if fin.size else 1.0, 1e-300)

        def note(sorted_values):
            a = np.asarray(sorted_values)
            with np.errstate(invalid="ignore"):
                d = a[:-1] - a[1:]
            d = d[d > 0]
            if d.size:
                gaps[r] = min(gaps[r], d.min() / size)

        if groups > 1:
            per = E // groups
            gv = np.array([np.sort(v[g * per:(g + 1) * per])[::-1][:group_best].sum()
                           for g in range(groups)])
            best = np.lexsort((np.arange(groups), -gv))
            note(gv[best][top_groups - 1:top_groups + 1])
            out = np.ones(E, bool)
            for g in best[:top_groups]:
                out[g * per:(g + 1) * per] = False
            by = np.where(out, -INF, by)
        order = np.lexsort((np.arange(E), -by))
        if bias is not None:
            note(by[order][:top + 1])
        chosen = [j for j in order[:top] if by[j] > -INF]
        ids[r, :len(chosen)] = chosen
        w = s[chosen]
        if renormalise and chosen:
            c = l[r][chosen]
            c = c if score == "softmax" else -np.logaddexp(0.0, -c)
            w = np.exp(c - c.max())
            w = w / w.sum()
        weights[r, :len(chosen)] = scale * w
    return dict(ids=ids, weights=weights, gap=gaps)


def route_weights(logits, ids, score="softmax", renormalise=True, scale=1.0):
    """The weights of given choices."""
    l = np.asarray(logits, dtype=np.float64)
    w = np.zeros(ids.shape)
    for r in range(l.shape[0]):
        on = (ids[r] >= 0) & (ids[r] < l.shape[1])
        c = l[r][ids[r][on]]
        s = _scores(l[r], score)[ids[r][on]]
        if renormalise and s.size:
            c = c if score == "softmax" else -np.logaddexp(0.0, -c)
            s = np.exp(c - c.max())
            s = s / s.sum()
        w[r, on] = scale * s
    return w


def route_grad(logits, ids, g, score="softmax", renormalise=True, scale=1.0):
    """Gradient of sum(g weights) with respect to the logits, by the chain rule
    through the scores."""
    l = np.asarray(logits, dtype=np.float64)
    grad = np.zeros(l.shape)
    for r in range(l.shape[0]):
        on = (ids[r] >= 0) & (ids[r] < l.shape[1])
        c = ids[r][on]
        if not c.size:
            continue
        s = _scores(l[r], score)
        gr = scale * np.asarray(g[r], dtype=np.float64)[on]
        ds = np.zeros(l.shape[1])
        if renormalise:
            t = s[c].sum()
            ds[c] = gr / t - (gr * s[c]).sum() / t ** 2
        else:
            ds[c] = gr
        # renormalised weights do not change with the scores' size: sum(ds s) is 0
        inner = 0.0 if renormalise else (ds * s).sum()
        grad[r] = ds * s * (1.0 - s) if score == "sigmoid" else s * (ds - inner)
    return grad


def dispatch(ids, experts, capacity=0):
    """dict(load, offsets, order, position) of int64 arrays."""
    flat = np.asarray(ids).reshape(-1)
    N = flat.size
    lists = [[] for _ in range(experts)]
    load = np.zeros(experts, np.int64)
    for p, e in enumerate(flat):
        if 0 <= e < experts:
            load[e] += 1
            if capacity == 0 or len(lists[e]) < capacity:
                lists[e].append(p)
    offsets = np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int64)
    order = np.full(N, -1, np.int64)
    position = np.full(N, -1, np.int64)
    kept = [p for x in lists for p in x]
    order[:len(kept)] = kept
    position[kept] = np.arange(len(kept))
    return dict(load=load, offsets=offsets, order=order, position=position.reshape(np.shape(ids)))


def linear_logprobs(hidden, weight, tokens, inv_temperature=1.0):
    """token_logprobs' dict for the logits hidden weight^T, which it holds too."""
    logits = np.asarray(hidden, dtype=np.float64) @ np.asarray(weight, dtype=np.float64).T
    return dict(token_logprobs(logits, tokens, 0, inv_temperature), logits=logits)


def linear_logprobs_grad(hidden, weight, tokens, g_logprob=None, g_entropy=None, inv_temperature=1.0):
    """(gradient of hidden, of weight, of the logits) of sum(g_logprob logprob +
    g_entropy entropy): a row whose incoming gradients are both 0 takes no part."""
    h, w = np.asarray(hidden, dtype=np.float64), np.asarray(weight, dtype=np.float64)
    T, V = h.shape[0], w.shape[0]
    tok = np.full(T, -1) if tokens is None else np.asarray(tokens)
    gl = np.zeros(T) if g_logprob is None else np.where(tok >= 0, np.asarray(g_logprob, dtype=np.float64), 0.0)
    gh = np.zeros(T) if g_entropy is None else np.asarray(g_entropy, dtype=np.float64)
    live = (gl != 0) | (gh != 0)
    d = np.zeros((T, V))
    d[live] = token_logprobs_grad(h[live] @ w.T, tok[live], gl[live], gh[live],
                                  inv_temperature=inv_temperature)
    grad_h = np.zeros_like(h)
    grad_h[live] = d[live] @ w
    return grad_h, d[live].T @ h[live], d


def expert_gather(x, order, top):
    x = np.asarray(x, dtype=np.float64)
    out = np.zeros((len(order), x.shape[1]))
    for i, p in enumerate(order):
        if p >= 0:
            out[i] = x[p // top]
    return out


def expert_combine(rows, position, weights=None):
    """(sum, sum of the terms' sizes)."""
    rows, position = np.asarray(rows, dtype=np.float64), np.asarray(position)
    T, top = position.shape
    out, size = np.zeros((T, rows.shape[1])), np.zeros((T, rows.shape[1]))
    for t in range(T):
        for k in range(top):
            i = position[t, k]
            if 0 <= i < len(rows):
                term = rows[i] * (1.0 if weights is None else float(weights[t, k]))
                out[t] += term
                size[t] += np.abs(term)
    return out, size


def expert_combine_grad(grad, rows, order, position, weights=None):
    """(gradient of rows, of weights, sizes of the terms of the latter)."""
    grad, rows = np.asarray(grad, dtype=np.float64), np.asarray(rows, dtype=np.float64)
    T, top = np.shape(position)
    g_rows, g_w, size = np.zeros_like(rows), np.zeros((T, top)), np.zeros((T, top))
    for i, p in enumerate(order):
        if p >= 0:
            g_rows[i] = grad[p // top] * (1.0 if weights is None else float(weights[p // top, p % top]))
    for t in range(T):
        for k in range(top):
            i = position[t, k]
            if 0 <= i < len(rows):
                g_w[t, k] = grad[t] @ rows[i]
                size[t, k] = np.abs(grad[t]) @ np.abs(rows[i])
    return g_rows, g_w, size


def embed(tokens, table, scale=1.0):
    table = np.asarray(table, dtype=np.float64)
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if v >= 0:
            out[t] = float(np.float32(scale)) * table[v] if v < len(table) else np.nan
    return out


def embed_grad(tokens, grad, vocab, scale=1.0):
    """(gradient of the table, sums of the terms' sizes, tokens per row)."""
    grad = np.asarray(grad, dtype=np.float64)
    out, size, count = np.zeros((vocab, grad.shape[1])), np.zeros((vocab, grad.shape[1])), np.zeros(vocab, int)
    s = float(np.float32(scale))
    for t, v in enumerate(tokens):
        if 0 <= v < vocab:
            out[v] += s * grad[t]
            size[v] += np.abs(s * grad[t])
            count[v] += 1
    return out, size, count
