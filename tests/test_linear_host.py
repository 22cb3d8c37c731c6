"""The entry points of the log probabilities from hidden rows, the experts' rows
and the embeddings without a GPU: sizes and arguments are checked before any
device work, and the workspace sizes are consistent."""
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


def test_linear_refusals(L):
    def call(type=0, T=2, V=10, H=8, it=1.0, hs=8, ws=8, hidden=P, wb=1 << 30):
        return L.bo_linear_logprobs(hidden, hs, P, ws, type, T, V, H, P, it, P, P, P, P, wb, None)
    assert call(type=3) == INVALID and call(T=-1) == INVALID and call(V=0) == INVALID and call(H=0) == INVALID
    for it in (0.0, -1.0, float("nan"), float("inf"), 1.1e30):
        assert call(it=it) == INVALID
    assert call(hs=7) == INVALID and call(hidden=None) == INVALID
    assert call(hidden=ctypes.c_void_p(0x1002)) == INVALID            # not aligned to fp32
    assert call(H=(1 << 20) + 1, hs=1 << 21, ws=1 << 21) == CAPACITY and call(T=2 ** 28 + 1) == CAPACITY
    assert call(V=2 ** 29 + 1) == CAPACITY and call(T=2 ** 20, V=2 ** 19) == CAPACITY
    assert call(T=2 ** 28, V=1, H=1 << 20, hs=2 ** 40) == CAPACITY    # the extent overflows
    assert call(T=0, hidden=None) == 0

    def grad(type=0, T=2, V=10, H=8, it=1.0, hs=8, gw=None):
        return L.bo_linear_logprobs_grad(P, hs, P, 8, type, T, V, H, P, it, P, P, P, P, P, 8, gw, 8, P,
                                         1 << 30, None)
    assert grad(type=-1) == INVALID and grad(T=-2) == INVALID and grad(it=0.0) == INVALID
    assert grad(hs=3) == INVALID and grad(H=(1 << 20) + 1) == CAPACITY
    assert grad(T=0) == 0                                            # nothing to write


def test_linear_workspaces(L):
    f, g = L.bo_linear_logprobs_workspace, L.bo_linear_logprobs_grad_workspace
    for w in (f, g):
        assert w(P, 8, P, 8, 0, 0, 10, 8) == 0 and w(P, 8, P, 8, 5, 2, 10, 8) == 0
        assert w(P, 8, P, 8, 0, 2, 10, 0) == 0 and w(P, 8, P, 8, 0, 2 ** 29, 2 ** 29, 8) == 0
    # far less than the logits, for a large batch
    T, V, H = 16384, 128000, 4096
    assert f(P, H, P, H, 1, T, V, H) < T * V * 4 / 16
    assert g(P, H, P, H, 1, T, V, H) < T * V * 4 / 8
    # rows at odd 2-byte places are copied, rows at 4-byte places are not
    even, odd = f(P, 1002, P, 1002, 1, 100, 50000, 1001), f(P, 1001, P, 1001, 1, 100, 50000, 1001)
    assert odd - even >= 2 * 50000 * 1001 and even < 10 ** 8
    assert f(ctypes.c_void_p(0x1002), 1002, P, 1002, 1, 100, 50000, 1001) > even


def test_expert_refusals(L):
    def gather(type=0, T=3, H=4, stride=4, top=2, R=6, x=P):
        return L.bo_expert_gather(x, type, T, H, stride, top, P, R, P, P, 4, None)
    assert gather(type=7) == INVALID and gather(T=-1) == INVALID and gather(H=0) == INVALID
    assert gather(top=0) == INVALID and gather(top=33, R=9) == CAPACITY and gather(R=7) == INVALID
    assert gather(R=-1) == INVALID and gather(stride=3) == INVALID and gather(T=2 ** 30, R=0) == CAPACITY
    assert gather(x=None) == INVALID and gather(T=0, R=0, x=None) == 0 and gather(R=0, x=None) == 0

    def combine(type=0, T=3, H=4, stride=4, top=2, R=6):
        return L.bo_expert_combine(P, type, R, H, stride, P, T, top, P, P, 4, None)
    assert combine(type=-1) == INVALID and combine(R=7) == INVALID and combine(stride=1) == INVALID
    assert combine(top=33) == CAPACITY and combine(T=0, R=0) == 0

    def grad(type=0, T=3, H=4, gs=4, top=2, R=6):
        return L.bo_expert_combine_grad(P, type, T, H, gs, P, R, 4, top, P, P, P, P, 4, P, None)
    assert grad(type=3) == INVALID and grad(R=9) == INVALID and grad(gs=2) == INVALID
    assert grad(top=40, R=2) == CAPACITY and grad(T=0, R=0) == 0


def test_embed_refusals(L):
    def embed(type=0, T=3, V=5, H=4, stride=4, scale=1.0):
        return L.bo_embed(P, T, P, type, V, H, stride, scale, P, 4, None)
    assert embed(type=3) == INVALID and embed(T=-1) == INVALID and embed(V=0) == INVALID
    assert embed(H=0) == INVALID and embed(scale=float("nan")) == INVALID
    assert embed(T=2 ** 31 - 1) == CAPACITY and embed(V=2 ** 31) == CAPACITY and embed(T=0) == 0

    def grad(type=0, T=3, V=5, H=4, scale=1.0):
        return L.bo_embed_grad(P, T, P, type, H, 4, scale, V, P, 4, P, 1 << 30, None)
    assert grad(type=3) == INVALID and grad(V=0) == INVALID and grad(scale=float("inf")) == INVALID
    assert grad(T=2 ** 31 - 1) == CAPACITY
    assert L.bo_embed_grad_workspace(0, 5, 4) == 0 and L.bo_embed_grad_workspace(5, 0, 4) == 0
    assert 0 < L.bo_embed_grad_workspace(1, 1, 1) < 1 << 20
    assert 0 < L.bo_embed_grad_workspace(2 ** 31 - 65537, 2 ** 31 - 1, 4) < 1 << 37
