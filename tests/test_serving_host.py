"""The served-output entry points without a GPU: sizes and arguments are
checked before any device work, and the workspace sizes are consistent."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def L():
    import os
    import paper_2602_10729_amd as bo
    if not os.path.exists(bo.lib_path()):
        from paper_2602_10729_amd import build
        build.build()
    return bo.lib()


P = ctypes.c_void_p(0x1000)
INVALID, CAPACITY = 1, 3


def _lp(L, type=0, T=2, V=10, stride=10, it=1.0, top=2, logits=P, ws=P, wb=1 << 30):
    return L.bo_token_logprobs(logits, type, T, V, stride, P, it, top, P, P, P, P, P, P, ws, wb, None)


def test_logprob_refusals(L):
    assert _lp(L, type=3) == INVALID and _lp(L, T=-1) == INVALID and _lp(L, V=0) == INVALID
    assert _lp(L, it=0.0) == INVALID and _lp(L, it=float("inf")) == INVALID
    assert _lp(L, it=1.1e30) == INVALID
    assert _lp(L, it=float("nan")) == INVALID and _lp(L, top=-1) == INVALID
    assert _lp(L, top=11) == INVALID and _lp(L, V=100, stride=100, top=65) == CAPACITY
    assert _lp(L, V=2 ** 31, stride=2 ** 31) == CAPACITY and _lp(L, T=2 ** 62) == CAPACITY
    assert _lp(L, T=2 ** 40, stride=2 ** 40) == CAPACITY       # the extent overflows
    assert _lp(L, stride=9) == INVALID and _lp(L, logits=None) == INVALID
    assert _lp(L, logits=ctypes.c_void_p(0x1002)) == INVALID   # not aligned to fp32
    assert _lp(L, T=0, logits=None) == 0


def test_logprob_grad_refusals(L):
    def call(type=0, T=2, V=10, stride=10, it=1.0, top=0, out=P, ostride=10):
        return L.bo_token_logprobs_grad(P, type, T, V, stride, P, it, P, P, P, P, top, P, P, out,
                                        ostride, None)
    assert call(type=-1) == INVALID and call(T=-2) == INVALID and call(it=-1.0) == INVALID
    assert call(top=65) == CAPACITY and call(stride=3) == INVALID
    assert call(T=0, out=None) == 0


def test_route_refusals(L):
    def call(type=0, T=2, E=12, score=0, top=2, groups=1, tg=1, gb=1, scale=1.0, stride=12):
        return L.bo_route(P, type, T, E, stride, P, score, top, groups, tg, gb, 1, scale, P, P, None)
    assert call(type=9) == INVALID and call(E=0) == INVALID and call(score=2) == INVALID
    assert call(top=0) == INVALID and call(top=33, E=64, stride=64) == CAPACITY
    assert call(E=1025, stride=1025) == CAPACITY and call(groups=5) == INVALID
    assert call(groups=0) == INVALID and call(groups=4, tg=5) == INVALID and call(groups=4, tg=0) == INVALID
    assert call(groups=12, tg=2, gb=2) == INVALID and call(gb=3) == INVALID
    assert call(groups=4, tg=1, top=4) == INVALID and call(scale=float("nan")) == INVALID
    assert call(T=0) == 0

    def grad(type=0, T=2, E=12, top=2):
        return L.bo_route_grad(P, type, T, E, 12, 0, top, 1, 1.0, P, P, P, 12, None)
    assert grad(type=9) == INVALID and grad(top=13) == INVALID and grad(T=-1) == INVALID
    assert grad(T=0) == 0


def test_dispatch_refusals(L):
    def call(N=4, E=3, cap=0):
        return L.bo_dispatch(P, N, E, cap, P, P, P, P, P, 1 << 30, None)
    assert call(N=-1) == INVALID and call(E=0) == INVALID and call(cap=-1) == INVALID
    assert call(E=1025) == CAPACITY and call(N=2 ** 31 - 1) == CAPACITY


def test_workspaces(L):
    assert L.bo_token_logprobs_workspace(0, 10, 0) == 0
    for T, V, top in ((1, 128000, 20), (3, 1000, 64), (10 ** 6, 10 ** 5, 5), (1, 2 ** 31 - 1, 64)):
        n = L.bo_token_logprobs_workspace(T, V, top)
        assert 0 <= n < 1 << 34
    assert L.bo_dispatch_workspace(0, 4) == 0 and L.bo_dispatch_workspace(5, 0) == 0
    assert 0 <= L.bo_dispatch_workspace(2 ** 31 - 65537, 1024) < 1 << 34
