"""The fp64 references of the log probabilities from hidden rows, the experts'
rows and the embeddings against brute force and central differences."""
import numpy as np
import pytest

from oracle import serving as R


@pytest.mark.parametrize("it", [1.0, 0.5])
def test_linear_gradients_against_differences(it):
    rng = np.random.default_rng(3)
    h, w = rng.normal(size=(5, 4)), rng.normal(size=(7, 4))
    tok = np.array([2, 5, -1, 6, -1])
    gl, gh = rng.normal(size=5), rng.normal(size=5)
    gh[4] = 0.0                                       # takes no part

    def total(h, w):
        f = R.linear_logprobs(h, w, tok, it)
        return (np.where(tok >= 0, gl * f["logprob"], 0) + gh * f["entropy"]).sum()

    grads = R.linear_logprobs_grad(h, w, tok, gl, gh, it)
    assert np.all(grads[0][4] == 0)
    e = 1e-6
    for which, x in enumerate((h, w)):
        for at in np.ndindex(x.shape):
            a, b = [h.copy(), w.copy()], [h.copy(), w.copy()]
            a[which][at] += e
            b[which][at] -= e
            assert abs((total(*a) - total(*b)) / (2 * e) - grads[which][at]) < 1e-7


def test_row_without_gradient_takes_no_part():
    rng = np.random.default_rng(4)
    h, w = rng.normal(size=(3, 4)), rng.normal(size=(6, 4))
    h[1] = np.nan
    g = R.linear_logprobs_grad(h, w, [0, -1, 5], [1.0, 1.0, 1.0])
    few = R.linear_logprobs_grad(h[[0, 2]], w, [0, 5], [1.0, 1.0])
    assert np.all(g[0][1] == 0) and np.allclose(g[1], few[1])


def _placed(rng, T, top, E, capacity):
    ids = np.array([rng.choice(E + 1, top, replace=False) for _ in range(T)])
    return R.dispatch(np.where(ids == E, -1, ids), E, capacity)


@pytest.mark.parametrize("capacity", [0, 3])
def test_expert_rows_against_brute_force(capacity):
    rng = np.random.default_rng(5)
    T, top, E, H = 9, 2, 4, 3
    d = _placed(rng, T, top, E, capacity)
    order, position = d["order"], d["position"]
    x, w = rng.normal(size=(T, H)), rng.random((T, top))
    g = R.expert_gather(x, order, top)
    for t in range(T):
        for k in range(top):
            if position[t, k] >= 0:
                assert np.array_equal(g[position[t, k]], x[t])
    assert np.all(g[d["offsets"][-1]:] == 0)
    # back without weights: a token times the places it has
    back, _ = R.expert_combine(g, position)
    assert np.allclose(back, x * (position >= 0).sum(1, keepdims=True))
    # gradients of sum(c combine) by differences
    rows, c = rng.normal(size=(T * top, H)), rng.normal(size=(T, H))
    g_rows, g_w, _ = R.expert_combine_grad(c, rows, order, position, w)
    f = lambda r, v: (c * R.expert_combine(r, position, v)[0]).sum()
    for at in np.ndindex(rows.shape):
        e = np.zeros_like(rows)
        e[at] = 1e-6
        assert abs((f(rows + e, w) - f(rows - e, w)) / 2e-6 - g_rows[at]) < 1e-8
    for at in np.ndindex(w.shape):
        e = np.zeros_like(w)
        e[at] = 1e-6
        assert abs((f(rows, w + e) - f(rows, w - e)) / 2e-6 - g_w[at]) < 1e-8
    # the gather's gradient is the combination without weights
    c = rng.normal(size=(T * top, H))
    want, _ = R.expert_combine(c, position)
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at] = 1e-6
        num = ((R.expert_gather(x + e, order, top) - R.expert_gather(x - e, order, top)) * c).sum() / 2e-6
        assert abs(num - want[at]) < 1e-8


def test_embedding_against_differences():
    rng = np.random.default_rng(6)
    tok, table = np.array([3, -1, 0, 3, 3, 1]), rng.normal(size=(5, 2))
    assert np.all(R.embed(tok, table, 0.5)[1] == 0) and np.isnan(R.embed([5], table)).all()
    c = rng.normal(size=(6, 2))
    g, _, count = R.embed_grad(tok, c, 5, 0.5)
    assert list(count) == [1, 1, 0, 3, 0] and np.all(g[[2, 4]] == 0)
    for at in np.ndindex(table.shape):
        e = np.zeros_like(table)
        e[at] = 1e-6
        num = ((R.embed(tok, table + e, 0.5) - R.embed(tok, table - e, 0.5)) * c).sum() / 2e-6
        assert abs(num - g[at]) < 1e-8
