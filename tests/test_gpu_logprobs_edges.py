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
