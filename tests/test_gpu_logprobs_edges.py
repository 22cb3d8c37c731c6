"""Log probabilities where the arithmetic and the bookkeeping of a row are at
their edges, against the fp64 reference.

Tolerances are those of the other served-output tests (see there): they follow
from the number of roundings and hold for every value of the logits.
"""
import numpy as np
import pytest

from oracle import serving as R
from test_gpu_serving import INF, _announce, _check_grad, _check_logprobs, _dtype, _logits, _np, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,V,top", [
    ("f32", 10001, 12), ("f32", 10003, 64), ("f32", 20001, 12), ("f32", 50001, 8), ("f32", 4095, 64),
    ("bf16", 8191, 64), ("bf16", 15001, 12), ("bf16", 32003, 20), ("bf16", 50001, 8), ("bf16", 128259, 33),
    ("f16", 8191, 64), ("f16", 16367, 40), ("f16", 50005, 12)])
def test_alternatives_of_a_full_last_chunk(kind, V, top):
    """More candidates in a row's last chunk than there is room for, with logits
    behind its whole vectors: every alternative once."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("alternatives of a full last chunk", kind, V, top)
    rng = np.random.default_rng(V)
    T = 24
    x = _logits(rng, T, V, kind)
    x[0] = torch.linspace(-4, 4, V, device="cuda")         # rising: the last chunk holds the best
    x[1] = x[0].flip(0)
    x[2, : V - 900] = -INF                                 # live at the end only
    x[3, : V - 900] = -INF
    x[3, V - 1] = 30.0                                     # the very last is the likeliest
    x[4, : V - 900] = -20.0
    x[5] = 0.25                                            # all equal
    x[6, : V - 5] = -INF
    x[7, -9:] += 50.0
    tok = rng.integers(0, V, T)
    r = bo.token_logprobs(x, _tokens(tok), top=top)
    _check_logprobs(r, x, tok, top, 1.0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("base", [0, 512, 1000, 8192, 40960])
def test_rank_of_tied_tokens_past_the_vectors(kind, base):
    """Equal logits before a token count once each, wherever in the row it stands:
    every length of what is left past the whole vectors, every place in it."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("rank of tied tokens", kind, base)
    rng = np.random.default_rng(base)
    for rest in range(1, 9):
        V = base + rest
        T = 2 * min(V, 12)
        x = torch.full((T, V), 0.5, device="cuda").to(_dtype(kind))
        x[T // 2:] = torch.from_numpy(rng.integers(0, 3, (T - T // 2, V)).astype(np.float32)).cuda().to(x.dtype)
        tok = V - 1 - np.arange(T) % (T // 2)
        r = bo.token_logprobs(x, _tokens(tok))
        _check_logprobs(r, x, tok, 0, 1.0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [700, 9000, 50003])
def test_rank_beside_signalling_nans(kind, V):
    """A logit above the token's counts, also where a NaN of any kind stands
    beside it and nothing else in reach is above the token."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("rank beside NaN", kind, V)
    rng = np.random.default_rng(31)
    word, bits = {"f32": (torch.int32, [0x7F800001, 0x7FC00000, -0x7FFFFF, -1]),
                  "bf16": (torch.int16, [0x7F81, 0x7FC0, -0x7F, -1]),
                  "f16": (torch.int16, [0x7C01, 0x7E00, -0x3FF, -1])}[kind]
    T = 32
    x = _logits(rng, T, V, kind)
    tok = rng.integers(0, V, T)
    for t in range(T):
        at = 16 * int(rng.integers(0, (V - 16) // 16)) + t % 8      # a vector's every place
        x[t, tok[t]] = 20.0
        nan = 16 * (at // 16) + (t // 4) % 8
        if tok[t] // 16 == at // 16:
            tok[t] = (tok[t] + 32) % (V - 16)
            x[t, tok[t]] = 20.0
        x[t, at] = 30.0
        if nan == at:
            nan = at ^ 1
        x[t].view(word)[nan] = bits[t % 4]
    o = R.token_logprobs(_np(x), tok, 2)
    for top in (0, 2):
        r = bo.token_logprobs(x, _tokens(tok), top=top)
        assert np.array_equal(r.rank.cpu().numpy(), o["rank"])
        assert bool(r.logprob.isnan().all()) and np.array_equal(_np(r.stats[:, 0]), o["stats"][:, 0])
    assert np.array_equal(r.top_ids.cpu().numpy(), o["top_ids"])


# 131077 = 16 * 8192 + 5: a row's last share is what is left past the vectors
@pytest.mark.parametrize("V", [40, 3001, 50003, 131077])
@pytest.mark.parametrize("kind,mask", [("f32", -1e10), ("f32", -1e20), ("f32", -1e30), ("f32", -1e35), ("f32", "lowest"),
                                       ("bf16", -1e10), ("bf16", -1e20), ("bf16", -1e30), ("bf16", "lowest"),
                                       ("f16", -6e4), ("f16", "lowest")])
def test_logprobs_finite_masks(V, kind, mask):
    """Masks that are large finite values: in part of a row, in whole shares of
    it, in all of it, beside -inf, and as the given token."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs finite masks", V, kind, mask)
    rng = np.random.default_rng(V)
    T, top = 9, 12
    x = _logits(rng, T, V, kind)
    value = torch.finfo(x.dtype).min if mask == "lowest" else mask
    cut = torch.from_numpy(rng.random(V) < 0.9).cuda()
    x[0, cut] = value
    x[1] = value                                   # uniform over the mask
    x[2] = value
    x[2, V - 1] = 1.5                              # one live, at the end
    x[3, : V // 2] = value
    x[4, 5:] = value
    x[5, cut] = value
    x[5, ::3] = -INF
    x[6] = x[6] * (-value / 16)                     # as far apart as the mask is far
    x[7, V // 2] = -value                          # one above all others
    x[8] = -INF
    x[8, ::2] = value
    tok = rng.integers(0, V, T)
    tok[0], tok[2], tok[3], tok[7] = int(cut.nonzero()[0]), V - 1, 0, V // 2
    for it in (0.5, 2 / 3, 1.0, 2.0):
        r = bo.token_logprobs(x, _tokens(tok), top=top, inv_temperature=it)
        _check_logprobs(r, x, tok, top, it)
        _check_grad(x, tok, r, rng, it, top, kind)


@pytest.mark.parametrize("V", [3001, 50003])
def test_logprobs_offsets_of_every_size(V):
    """Rows that lie around every power of four from 1 to 2^62, and around the
    place where a scaled logit stops being exact to a unit (2^24)."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs offsets of every size", V)
    rng = np.random.default_rng(V + 1)
    centres = [s * 4.0 ** k for k in range(32) for s in (1, -1)] + [s * 11629080.0 for s in (1, -1)]
    x = _logits(rng, len(centres), V, "f32", spread=3.0)
    x += torch.tensor(centres, dtype=torch.float32, device="cuda")[:, None]
    tok = rng.integers(0, V, len(centres))
    for it in (1.0, 1 / 0.7):
        r = bo.token_logprobs(x, _tokens(tok), top=3, inv_temperature=it)
        _check_logprobs(r, x, tok, 3, it)
        _check_grad(x, tok, r, rng, it, 3, "f32")


@pytest.mark.parametrize("V", [700, 40003])
@pytest.mark.parametrize("kind,it", [("f32", 1e9), ("f32", 1e30), ("bf16", 1e9), ("bf16", 1e30), ("f16", 1e4),
                                     ("f32", 1e-20), ("f32", 1e-38), ("f32", 1e-40), ("bf16", 1e-38)])
def test_logprobs_extreme_temperatures(V, kind, it):
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs extreme temperatures", V, kind, it)
    rng = np.random.default_rng(V + 2)
    x = _logits(rng, 6, V, kind)
    low = torch.finfo(x.dtype).min
    x[1, ::2] = low
    x[2, ::2] = low
    x[2, 1::4] = -low                              # apart by more than the type's largest value
    x[3, : V // 2] = -INF
    x[4] = low
    x[5] = -INF
    tok = rng.integers(0, V, 6)
    r = bo.token_logprobs(x, _tokens(tok), top=5, inv_temperature=it)
    _check_logprobs(r, x, tok, 5, it)
    if it < 1e29:                                  # (beyond, terms of a gradient leave fp32)
        _check_grad(x, tok, r, rng, it, 5, kind, use=(True, it < 1, True))


@pytest.mark.parametrize("kind,it,size", [("f32", 1.0, 1e9), ("f32", 1e9, 1.0), ("f32", 1e30, 1.0), ("f32", 1e30, 1e6),
                                          ("bf16", 1.0, 1e9), ("bf16", 1e9, 1.0), ("f32", 1.0, 3e38)])
def test_gradient_of_impossible_tokens_is_zero(kind, it, size):
    """Masked logits, and those whose probability is 0 in fp32, have gradient 0
    however large the incoming gradients are; NaN still reaches the whole row."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("gradient of impossible tokens", kind, it, size)
    rng = np.random.default_rng(4)
    T, V = 4, 9003
    x = _logits(rng, T, V, kind)
    x[1, ::2] = -INF
    x[2, ::2] = -1e30
    x[3, 1:] = -1e4
    x[3, 0] = 0.0
    tok = np.array([7, 1, 3, 0])
    r = bo.token_logprobs(x, _tokens(tok), inv_temperature=it)
    sized = torch.full((T,), size, device="cuda")
    l = _np(x)
    off = torch.from_numpy((l - l.max(1, keepdims=True)) * float(np.float32(it)) < -200.0).cuda()
    off[torch.arange(T), _tokens(tok)] = False     # (a token has its own term)
    for gl, gh in ((None, sized), (sized, None), (sized, sized), (sized, -sized)):
        g = bo.token_logprobs_grad(x, _tokens(tok), r.stats, r.entropy, gl, gh, inv_temperature=it)
        assert bool((g[off] == 0).all())
    nan = torch.full((T,), float("nan"), device="cuda")
    for gl, gh in ((nan, None), (None, nan)):
        g = bo.token_logprobs_grad(x, _tokens(tok), r.stats, r.entropy, gl, gh, inv_temperature=it)
        assert bool(g.isnan().all())
    past = bo.token_logprobs_grad(x, _tokens([V, V, V, V]), r.stats, r.entropy, sized, inv_temperature=it)
    assert bool(past.isnan().all())


@pytest.mark.parametrize("V,top", [(40001, 12), (81923, 64), (131077, 5), (131077, 64)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_logprobs_joined_shares(V, top, kind):
    """Rows shared out over workgroups: shares with no live logit, with NaN or an
    infinity, with the only live ones, and a last one that holds only what is
    left past the vectors."""
    import torch
    import paper_2602_10729_amd as bo
    _announce("logprobs joined shares", V, top, kind)
    rng = np.random.default_rng(V + top)
    T, S = 16, 8192
    x = _logits(rng, T, V, kind)
    low = torch.finfo(x.dtype).min
    tok = rng.integers(0, V, T)
    x[0] = -INF                                    # nothing left
    x[1, :S] = -INF                                # a share masked
    x[2, S:] = -INF                                # all but a share
    x[3] = -INF
    x[3, V - 1] = -7.0                             # one left, at the very end
    x[4] = -INF
    x[4, S - 1] = 3.0                              # one left, at a share's end
    x[5] = low
    x[6, : 2 * S] = low
    x[7, S + 5] = float("nan")
    x[8, 2 * S + 9] = INF
    x[9] = 0.5
    x[10] = torch.linspace(-8, 8, V, device="cuda")        # each share above the one before
    x[11] = x[10].flip(0)
    x[12, : V - 3] = -INF                          # fewer than top
    x[13, S: 3 * S] = low
    x[13, 3 * S:] = -INF
    x[14, V - 2] = 50.0
    tok[2], tok[3], tok[4], tok[12], tok[14], tok[15] = S - 1, V - 1, S - 1, V - 2, V - 2, -1
    for it in (1.0, 0.5):
        r = bo.token_logprobs(x, _tokens(tok), top=top, inv_temperature=it)
        _check_logprobs(r, x, tok, top, it)
        _check_grad(x, tok, r, rng, it, top, kind)
