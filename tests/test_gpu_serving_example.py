"""The routing search of examples/, from log probabilities to the next
configuration: it runs, its router learns, and its front never shrinks."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_search_improves():
    import routing_search as S
    print("[case] routing search", flush=True)
    h = S.main(queries=512, tokens=8, vocab=1000, iterations=4, seed=1, verbose=False)
    assert len(h) == 5 and np.all(np.diff(h) >= -1e-9) and np.isfinite(h).all()


def test_router_learns_where_quality_is():
    import torch
    import paper_2602_10729_amd as bo
    import routing_search as S
    print("[case] router training", flush=True)
    logits, answer, quality = S.trace(512, 8, 1000, 2)
    x = S.features(logits, answer, 512, S.calibrate(logits, answer))
    w = S.train_router(x, quality)
    value = quality - 0.02 * S.COST.cuda()
    r = bo.route((x @ w).contiguous(), 1)
    chosen = value.gather(1, r.ids.long()).mean()
    assert float(chosen) > float(value.mean(0).max())     # better than any one model for all
    assert torch.isfinite(w).all()
