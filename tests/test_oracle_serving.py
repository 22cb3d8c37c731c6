"""The fp64 references of the served-output operators against brute force,
invariants and central differences."""
import numpy as np
import pytest

from oracle import serving as R

INF = np.inf


def test_uniform_row_has_log_v():
    f = R.token_logprobs(np.zeros((1, 7)), [3], top=3)
    assert np.allclose(f["logprob"], -np.log(7)) and np.allclose(f["entropy"], np.log(7))
    assert f["rank"][0] == 4 and list(f["top_ids"][0]) == [0, 1, 2]


def test_masked_rows():
    l = np.array([[-INF, -INF, -INF], [-INF, 1.0, -INF]])
    f = R.token_logprobs(l, [1, 1], top=2)
    assert f["logprob"][0] == -INF and f["rank"][0] == 0 and f["entropy"][0] == 0
    assert list(f["top_ids"][0]) == [-1, -1]
    assert f["logprob"][1] == 0 and f["rank"][1] == 1 and list(f["top_ids"][1]) == [1, -1]
    assert np.all(R.token_logprobs_grad(l, [1, 1], [1.0, 1.0])[0] == 0)


@pytest.mark.parametrize("it", [1.0, 0.5])
def test_logprob_gradient_against_differences(it):
    rng = np.random.default_rng(3)
    l = rng.normal(size=(4, 9))
    l[1, 2] = -INF
    tok = np.array([2, 5, -1, 8])
    ids = np.array([[1, 2], [0, 5], [3, -1], [8, 8]])
    gl, gh, gt = rng.normal(size=4), rng.normal(size=4), rng.normal(size=(4, 2))

    def total(x):
        f = R.token_logprobs(x, tok, 0, it)
        v = np.where(tok >= 0, gl * f["logprob"], 0) + gh * f["entropy"]
        for i in range(2):
            g = R.token_logprobs(x, ids[:, i], 0, it)["logprob"]
            v = v + np.where(ids[:, i] >= 0, gt[:, i] * g, 0)
        return v

    grad = R.token_logprobs_grad(l, tok, gl, gh, ids, gt, it)
    h = 1e-6
    for j in range(9):
        a, b = l.copy(), l.copy()
        a[:, j] += h
        b[:, j] -= h
        assert np.allclose((total(a) - total(b)) / (2 * h), grad[:, j], atol=1e-7)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_gradient_against_differences(score, renorm):
    rng = np.random.default_rng(4)
    l = rng.normal(size=(5, 8))
    ids = np.argsort(-l, 1)[:, :3]
    ids[1, 2] = -1
    ids[2] = -1
    g = rng.normal(size=(5, 3))
    grad = R.route_grad(l, ids, g, score, renorm, 2.5)
    h = 1e-6
    for j in range(8):
        a, b = l.copy(), l.copy()
        a[:, j] += h
        b[:, j] -= h
        d = ((R.route_weights(a, ids, score, renorm, 2.5) -
              R.route_weights(b, ids, score, renorm, 2.5)) * np.where(ids >= 0, g, 0)).sum(1) / (2 * h)
        assert np.allclose(d, grad[:, j], atol=1e-7)


def test_route_groups_and_withdrawn_experts():
    l = np.array([[5.0, 0.0, 4.0, 3.9, 1.0, 1.0]])
    r = R.route(l, 2, groups=3, top_groups=1, group_best=2, score="sigmoid")
    assert list(r["ids"][0]) == [2, 3]          # 4.0 and 3.9 together outweigh 5.0 and 0.0
    bias = np.array([0, 0, -INF, 0, 0, 0.0])
    r = R.route(l, 3, bias=bias, score="sigmoid")
    assert 2 not in r["ids"][0] and np.isclose(r["weights"][0].sum(), 1)
    r = R.route(np.full((1, 4), -INF), 2)
    assert list(r["ids"][0]) == [-1, -1] and not r["weights"].any()


def test_dispatch_is_a_stable_sort():
    rng = np.random.default_rng(5)
    ids = rng.integers(-1, 7, size=(50, 3))
    d = R.dispatch(ids, 7)
    flat = ids.reshape(-1)
    want = [p for p in np.argsort(flat, kind="stable") if flat[p] >= 0]
    assert list(d["order"][:len(want)]) == want and np.all(d["order"][len(want):] == -1)
    assert np.array_equal(d["load"], np.bincount(flat[flat >= 0], minlength=7))
    c = R.dispatch(ids, 7, capacity=5)
    assert np.array_equal(np.diff(c["offsets"]), np.minimum(d["load"], 5))
    kept = c["position"].reshape(-1) >= 0
    assert np.array_equal(c["order"][c["position"].reshape(-1)[kept]], np.nonzero(kept)[0])
