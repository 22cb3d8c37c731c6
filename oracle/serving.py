"""fp64 references of the served-output operators: log probabilities of given
tokens, routing to experts, and the grouping of choices by expert.

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
