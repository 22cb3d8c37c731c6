"""Python binding of libbo, the MI355X batch acquisition scorer.

Argument marshalling only: every step of fitting, scoring and the argmax runs
in the HIP kernels of ``libbo.so``; torch tensors supply device memory and the
current stream. There is no CPU fallback: if the library is missing or a
tensor is not on the GPU, the call raises.

Functions mirror the C ABI in ``include/bo.h``:
``fit`` (``bo_fit``), ``fit_composite`` (``bo_fit_composite``), ``mll``
(``bo_mll``), ``score`` (``bo_score``, or ``bo_score_constrained`` when feasibility
thresholds are given), ``nehvi_prepare`` / ``score_nehvi`` / ``Model.nehvi_front``
(``bo_nehvi_prepare``, ``bo_score_nehvi``, ``bo_nehvi_front``), ``argmax``,
``cholesky_test`` (device), ``token_logprobs`` / ``token_logprobs_grad``, ``route``
/ ``route_grad`` and ``dispatch`` (``bo_token_logprobs`` and so on) and
``pareto_front``, ``box_decomposition`` (host geometry, no GPU needed).
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional

import numpy as np

__all__ = ["BoError", "Model", "lib", "lib_path", "fit", "fit_composite", "mll", "score", "score_noalloc", "nehvi_prepare", "score_nehvi", "argmax",
           "cholesky_test", "draw_fronts3_test", "profile_enable", "profile_read", "measure_peak", "pareto_front", "box_decomposition", "STATUS",
           "TokenLogprobs", "token_logprobs", "token_logprobs_grad", "Routing", "route", "route_grad",
           "Dispatch", "dispatch", "MAX_ALTERNATIVES", "MAX_EXPERTS", "MAX_CHOICES",
           "MAX_N", "MAX_D", "MAX_S", "MAX_BOXES"]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libbo.so")
_lib = None

STATUS = {
    0: "BO_OK", 1: "BO_ERR_INVALID_ARGUMENT", 2: "BO_ERR_NOT_POSITIVE_DEFINITE",
    3: "BO_ERR_CAPACITY", 4: "BO_ERR_DEVICE", 5: "BO_ERR_OUT_OF_MEMORY",
    6: "BO_ERR_NONFINITE_INPUT", 7: "BO_ERR_ILL_CONDITIONED",
}
MAX_N, MAX_D, MAX_S, MAX_BOXES = 2048, 32, 4096, 4096
MAX_ALTERNATIVES, MAX_EXPERTS, MAX_CHOICES = 64, 1024, 32


class BoError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        self.status = status
        self.name = STATUS.get(status, str(status))
        super().__init__(f"{where}: {self.name}: {detail}")


def lib_path() -> str:
    return _LIB_PATH


def lib() -> ctypes.CDLL:
    """Load libbo.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2602_10729_amd.build`")
    L = ctypes.CDLL(_LIB_PATH)
    vp, i64, i32, fp = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
    L.bo_fit.argtypes = [vp, vp, i64, i32, i32, fp, fp, fp, vp, ctypes.POINTER(vp)]
    L.bo_fit.restype = ctypes.c_int
    L.bo_fit_composite.argtypes = [vp, vp, i64, i32, i32, i32, fp, fp, fp, fp, fp, fp, vp,
                                   ctypes.POINTER(vp)]
    L.bo_fit_f64.argtypes = L.bo_fit.argtypes
    L.bo_fit_f64.restype = ctypes.c_int
    L.bo_fit_composite_f64.argtypes = L.bo_fit_composite.argtypes
    L.bo_fit_composite_f64.restype = ctypes.c_int
    L.bo_fit_composite.restype = ctypes.c_int
    L.bo_mll.argtypes = [vp, vp, i64, i32, i32, fp, fp, fp, vp, vp, vp]
    L.bo_mll.restype = ctypes.c_int
    L.bo_score.argtypes = [vp, vp, i64, i32, fp, vp, i32, vp, vp, vp, vp]
    L.bo_score.restype = ctypes.c_int
    L.bo_score_constrained.argtypes = [vp, vp, i64, i32, fp, fp, vp, i32, vp, vp, vp, vp]
    L.bo_score_constrained.restype = ctypes.c_int
    L.bo_score_noalloc.argtypes = [vp, vp, i64, i32, fp, vp, i32, vp, vp]
    L.bo_score_noalloc.restype = ctypes.c_int
    L.bo_nehvi_prepare.argtypes = [vp, vp, i32, fp, fp, vp]
    L.bo_nehvi_prepare.restype = ctypes.c_int
    L.bo_score_nehvi.argtypes = [vp, vp, i64, i32, vp, i32, vp, vp]
    L.bo_score_nehvi.restype = ctypes.c_int
    L.bo_nehvi_front.argtypes = [vp, i32, vp, i32, ctypes.POINTER(i32)]
    L.bo_nehvi_front.restype = ctypes.c_int
    L.bo_argmax.argtypes = [vp, i64, vp, vp, vp]
    L.bo_argmax.restype = ctypes.c_int
    L.bo_model_front_size.argtypes = [vp]
    L.bo_model_front_size.restype = i32
    L.bo_model_front_indices.argtypes = [vp, vp, i32]
    L.bo_model_front_indices.restype = ctypes.c_int
    L.bo_cholesky_test.argtypes = [vp, i64, vp, vp]
    L.bo_cholesky_test.restype = ctypes.c_int
    L.bo_draw_fronts3_test.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp, vp]
    L.bo_draw_fronts3_test.restype = ctypes.c_int
    L.bo_pareto_front.argtypes = [vp, i64, i32, vp, vp, i32, ctypes.POINTER(i32)]
    L.bo_pareto_front.restype = ctypes.c_int
    L.bo_box_decomposition.argtypes = [vp, i32, i32, vp, vp, vp, i32, ctypes.POINTER(i32)]
    L.bo_box_decomposition.restype = ctypes.c_int
    L.bo_profile_enable.argtypes = [i32]
    L.bo_profile_enable.restype = ctypes.c_int
    L.bo_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double),
                                  ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.bo_profile_read.restype = ctypes.c_int
    L.bo_measure_peak.argtypes = [i32, i64, ctypes.POINTER(ctypes.c_double), vp]
    L.bo_measure_peak.restype = ctypes.c_int
    f32 = ctypes.c_float
    L.bo_token_logprobs_workspace.argtypes = [i64, i64, i32]
    L.bo_token_logprobs_workspace.restype = i64
    L.bo_token_logprobs.argtypes = [vp, i32, i64, i64, i64, vp, f32, i32, vp, vp, vp, vp, vp, vp,
                                    vp, i64, vp]
    L.bo_token_logprobs.restype = ctypes.c_int
    L.bo_token_logprobs_grad.argtypes = [vp, i32, i64, i64, i64, vp, f32, vp, vp, vp, vp, i32, vp,
                                         vp, vp, i64, vp]
    L.bo_token_logprobs_grad.restype = ctypes.c_int
    L.bo_route.argtypes = [vp, i32, i64, i32, i64, vp, i32, i32, i32, i32, i32, i32, f32, vp, vp, vp]
    L.bo_route.restype = ctypes.c_int
    L.bo_route_grad.argtypes = [vp, i32, i64, i32, i64, i32, i32, i32, f32, vp, vp, vp, i64, vp]
    L.bo_route_grad.restype = ctypes.c_int
    L.bo_dispatch_workspace.argtypes = [i64, i32]
    L.bo_dispatch_workspace.restype = i64
    L.bo_dispatch.argtypes = [vp, i64, i32, i64, vp, vp, vp, vp, vp, i64, vp]
    L.bo_dispatch.restype = ctypes.c_int
    L.bo_free.argtypes = [vp]
    L.bo_free.restype = None
    L.bo_status_string.argtypes = [ctypes.c_int]
    L.bo_status_string.restype = ctypes.c_char_p
    L.bo_last_error_message.argtypes = []
    L.bo_last_error_message.restype = ctypes.c_char_p
    _lib = L
    return L


def _check(status: int, where: str):
    if status != 0:
        detail = lib().bo_last_error_message().decode(errors="replace")
        raise BoError(status, where, detail)


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(int(stream.cuda_stream))


_raw_stream = None


def _stream_of(t, stream):
    """The stream's handle for a call on tensor t: torch's current stream of its
    device, read without building a stream object (0.1 us instead of 3) where
    this torch can."""
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _raw_stream(t.get_device())


def _dev(t, name, dtype=None):
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor on the GPU")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must live on a GPU (got {t.device})")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _host_f32(a, shape, name):
    a = np.ascontiguousarray(np.asarray(a, dtype=np.float32))
    if a.size != int(np.prod(shape)):
        raise ValueError(f"{name} must have {int(np.prod(shape))} elements")
    return a


class Model:
    """A fitted model (opaque handle owned by the library)."""

    def __init__(self, handle: int, n: int, d: int, m: int):
        self._h = ctypes.c_void_p(handle)
        self.n, self.d, self.m = n, d, m

    @property
    def handle(self):
        return self._h

    def front_indices(self) -> np.ndarray:
        L = lib()
        P = L.bo_model_front_size(self._h)
        out = np.zeros(max(P, 0), dtype=np.int32)
        _check(L.bo_model_front_indices(self._h, out.ctypes.data_as(ctypes.c_void_p), P),
               "bo_model_front_indices")
        return out

    def nehvi_front(self, sample: int) -> np.ndarray:
        """Front of one prepared in-sample draw (bo_nehvi_front): indices into
        the observations, sorted by objective 0 ascending."""
        L = lib()
        cnt = ctypes.c_int32(0)
        _check(L.bo_nehvi_front(self._h, int(sample), None, 0, ctypes.byref(cnt)), "bo_nehvi_front")
        out = np.zeros(cnt.value, dtype=np.int32)
        _check(L.bo_nehvi_front(self._h, int(sample), out.ctypes.data_as(ctypes.c_void_p),
                                cnt.value, ctypes.byref(cnt)), "bo_nehvi_front")
        return out

    def close(self):
        if self._h is not None and self._h.value:
            lib().bo_free(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def fit(X, Y, lengthscale, outputscale, noise, stream=None, f64=False) -> Model:
    """bo_fit (bo_fit_f64 when f64: scoring in double precision): X [n, d],
    Y [n, m] fp32 GPU tensors; hyperparameters on host."""
    import torch
    n, d = X.shape
    m = Y.shape[1]
    ls = _host_f32(lengthscale, (m, d), "lengthscale")
    os_ = _host_f32(outputscale, (m,), "outputscale")
    nz = _host_f32(noise, (m,), "noise")
    h = ctypes.c_void_p()
    fn = lib().bo_fit_f64 if f64 else lib().bo_fit
    st = fn(_dev(X, "X", torch.float32), _dev(Y, "Y", torch.float32), n, d, m,
            ls.ctypes.data_as(ctypes.c_void_p), os_.ctypes.data_as(ctypes.c_void_p),
            nz.ctypes.data_as(ctypes.c_void_p), _stream(stream), ctypes.byref(h))
    _check(st, "bo_fit_f64" if f64 else "bo_fit")
    return Model(h.value, n, d, m)


def fit_composite(X, Y, d_route, lengthscale, scale_route, scale_dep, scale_int, pref, noise,
                  stream=None, f64=False) -> Model:
    """bo_fit_composite (bo_fit_composite_f64 when f64): the composite kernel
    (routing Matern-5/2 + preference-weighted deployment Matern-3/2 +
    interaction). X [n, d], Y [n, m] fp32 GPU tensors; hyperparameters on host
    (pref [m, d - d_route])."""
    import torch
    n, d = X.shape
    m = Y.shape[1]
    ls = _host_f32(lengthscale, (m, d), "lengthscale")
    sr = _host_f32(scale_route, (m,), "scale_route")
    sd = _host_f32(scale_dep, (m,), "scale_dep")
    si = _host_f32(scale_int, (m,), "scale_int")
    pf = _host_f32(pref, (m, max(d - int(d_route), 0)), "pref")
    nz = _host_f32(noise, (m,), "noise")
    h = ctypes.c_void_p()
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    fn = lib().bo_fit_composite_f64 if f64 else lib().bo_fit_composite
    st = fn(_dev(X, "X", torch.float32), _dev(Y, "Y", torch.float32), n, d,
            m, int(d_route), p(ls), p(sr), p(sd), p(si), p(pf), p(nz),
            _stream(stream), ctypes.byref(h))
    _check(st, "bo_fit_composite_f64" if f64 else "bo_fit_composite")
    return Model(h.value, n, d, m)


def mll(X, Y, lengthscale, outputscale, noise, stream=None):
    """bo_mll: (value [m], gradient [m, d + 2]) of the exact log marginal
    likelihood with respect to (log lengthscales, log outputscale, log noise)."""
    import torch
    n, d = X.shape
    m = Y.shape[1]
    ls = _host_f32(lengthscale, (m, d), "lengthscale")
    os_ = _host_f32(outputscale, (m,), "outputscale")
    nz = _host_f32(noise, (m,), "noise")
    val = np.zeros(m, dtype=np.float64)
    grad = np.zeros((m, d + 2), dtype=np.float64)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    st = lib().bo_mll(_dev(X, "X", torch.float32), _dev(Y, "Y", torch.float32), n, d, m, p(ls),
                      p(os_), p(nz), _stream(stream), p(val), p(grad))
    _check(st, "bo_mll")
    return val, grad


def score(model: Model, cand, ref, Z, ehvi=None, mu=None, sigma=None, stream=None,
          lower=None):
    """bo_score: cand [M, q, d], Z [S, q, m] fp32 GPU tensors; ref host [m].

    Returns the ehvi tensor [M] (allocated if not given). mu/sigma
    [M, q, m] are written only when passed. ``lower`` (host [m], optional)
    selects bo_score_constrained with these feasibility thresholds.
    """
    import torch
    M, q, d = cand.shape
    S = Z.shape[0]
    r = _host_f32(ref, (model.m,), "ref")
    if ehvi is None:
        ehvi = torch.empty(M, dtype=torch.float32, device=cand.device)
    mu_p = _dev(mu, "mu", torch.float32) if mu is not None else ctypes.c_void_p(0)
    sg_p = _dev(sigma, "sigma", torch.float32) if sigma is not None else ctypes.c_void_p(0)
    args = (_dev(cand, "cand", torch.float32), M, q, r.ctypes.data_as(ctypes.c_void_p))
    tail = (_dev(Z, "Z", torch.float32), S, _dev(ehvi, "ehvi", torch.float32), mu_p, sg_p,
            _stream(stream))
    if lower is None:
        st = lib().bo_score(model.handle, *args, *tail)
        _check(st, "bo_score")
    else:
        lw = _host_f32(lower, (model.m,), "lower")
        st = lib().bo_score_constrained(model.handle, *args, lw.ctypes.data_as(ctypes.c_void_p),
                                        *tail)
        _check(st, "bo_score_constrained")
    return ehvi


def score_noalloc(model: Model, cand, ref, Z, ehvi, stream=None):
    """bo_score_noalloc: bo_score without mu/sigma outputs that allocates no
    device memory (its workspace is the library's fixed per-device scratch).
    cand [M, q, d], Z [S, q, m], ehvi [M] fp32 GPU tensors (ehvi must be
    given: this call allocates nothing, the binding neither); ref host [m]."""
    import torch
    M, q, d = cand.shape
    S = Z.shape[0]
    r = _host_f32(ref, (model.m,), "ref")
    st = lib().bo_score_noalloc(model.handle, _dev(cand, "cand", torch.float32), M, q,
                                r.ctypes.data_as(ctypes.c_void_p), _dev(Z, "Z", torch.float32), S,
                                _dev(ehvi, "ehvi", torch.float32), _stream(stream))
    _check(st, "bo_score_noalloc")
    return ehvi


def nehvi_prepare(model: Model, ZX, ref, lower=None, stream=None):
    """bo_nehvi_prepare: ZX [S, n, m] fp32 GPU tensor (in-sample base
    samples); ref host [m]; lower host [m] or None. Synchronous."""
    import torch
    S = ZX.shape[0]
    r = _host_f32(ref, (model.m,), "ref")
    lw = None if lower is None else _host_f32(lower, (model.m,), "lower")
    st = lib().bo_nehvi_prepare(model.handle, _dev(ZX, "ZX", torch.float32), S,
                                r.ctypes.data_as(ctypes.c_void_p),
                                lw.ctypes.data_as(ctypes.c_void_p) if lw is not None else None,
                                _stream(stream))
    _check(st, "bo_nehvi_prepare")


def score_nehvi(model: Model, cand, Z, ehvi=None, stream=None):
    """bo_score_nehvi: cand [M, d] or [M, q, d] and Z [S, m] or [S, q, m] fp32
    GPU tensors. Returns the ehvi tensor [M] (allocated if not given)."""
    import torch
    M = cand.shape[0]
    q = cand.shape[1] if cand.dim() == 3 else 1
    S = Z.shape[0]
    if ehvi is None:
        ehvi = torch.empty(M, dtype=torch.float32, device=cand.device)
    st = lib().bo_score_nehvi(model.handle, _dev(cand, "cand", torch.float32), M, q,
                              _dev(Z, "Z", torch.float32), S, _dev(ehvi, "ehvi", torch.float32),
                              _stream(stream))
    _check(st, "bo_score_nehvi")
    return ehvi


def argmax(values, index=None, value=None, stream=None):
    """bo_argmax into device scalars (int64 index, float32 value)."""
    import torch
    dev = values.device
    if index is None:
        index = torch.empty(1, dtype=torch.int64, device=dev)
    if value is None:
        value = torch.empty(1, dtype=torch.float32, device=dev)
    st = lib().bo_argmax(_dev(values, "values", torch.float32), values.numel(),
                         _dev(index, "index", torch.int64), _dev(value, "value", torch.float32),
                         _stream(stream))
    _check(st, "bo_argmax")
    return index, value


def profile_enable(on: bool = True):
    """Start (or stop) per-phase event timing of bo_score calls."""
    _check(lib().bo_profile_enable(1 if on else 0), "bo_profile_enable")


def profile_read():
    """(posterior_ms, ehvi_ms, calls, posterior_launches) since the last read."""
    a, b = ctypes.c_double(), ctypes.c_double()
    c, n = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().bo_profile_read(ctypes.byref(a), ctypes.byref(b), ctypes.byref(c),
                                 ctypes.byref(n)), "bo_profile_read")
    return a.value, b.value, c.value, n.value


PEAK_VALU_FMA, PEAK_VALU_CLAMP, PEAK_MFMA_F32, PEAK_HBM_COPY, PEAK_MFMA_F16 = 0, 1, 2, 3, 4


def measure_peak(what: int, iters: int = 4096, stream=None) -> float:
    """Achieved rate of a synthetic probe (see bo_measure_peak in bo.h)."""
    r = ctypes.c_double()
    _check(lib().bo_measure_peak(what, iters, ctypes.byref(r), _stream(stream)), "bo_measure_peak")
    return r.value


def cholesky_test(A, L=None, stream=None):
    """bo_cholesky_test: lower factor of a symmetric fp32 GPU matrix."""
    import torch
    n = A.shape[0]
    if L is None:
        L = torch.empty_like(A)
    st = lib().bo_cholesky_test(_dev(A, "A", torch.float32), n, _dev(L, "L", torch.float32),
                                _stream(stream))
    _check(st, "bo_cholesky_test")
    return L


def draw_fronts3_test(F, ref, lower=None, stream=None):
    """bo_draw_fronts3_test: per-draw fronts and boxes of three-objective
    values F (fp64 GPU tensor [S][n][3]). Returns (fronts, boxes): per draw the
    front's indices (objective 0 ascending) and its boxes [nb][6]
    (lo0, lo1, lo2, w0, w1, w2)."""
    import torch
    S, n, m = F.shape
    if m != 3:
        raise ValueError("F must be [S][n][3]")
    front = torch.empty((S, n), dtype=torch.int32, device=F.device)
    boxes = torch.empty((S, 3 * n + 1, 6), dtype=torch.float32, device=F.device)
    counts = torch.empty(2 * S, dtype=torch.int32, device=F.device)
    r = np.ascontiguousarray(np.asarray(ref, dtype=np.float32))
    lo = None if lower is None else np.ascontiguousarray(np.asarray(lower, dtype=np.float32))
    st = lib().bo_draw_fronts3_test(
        _dev(F, "F", torch.float64), n, S, r.ctypes.data_as(ctypes.c_void_p),
        None if lo is None else lo.ctypes.data_as(ctypes.c_void_p),
        _dev(front, "front"), _dev(boxes, "boxes"), _dev(counts, "counts"), _stream(stream))
    _check(st, "bo_draw_fronts3_test")
    c = counts.cpu().numpy()
    fr, bx = front.cpu().numpy(), boxes.cpu().numpy()
    return ([fr[s, :c[S + s]].copy() for s in range(S)],
            [bx[s, :c[s]].copy() for s in range(S)])


# ---- served outputs: log probabilities, routing, dispatch ----------------------
#
# None of these calls takes part in torch's autograd: what they return requires no
# gradient, whatever their inputs do. Gradients come from the _grad calls.

class TokenLogprobs(NamedTuple):
    """What token_logprobs returns, row by row: fp32 ``logprob``, ``entropy``
    and ``stats`` [T, 2] (largest logit, log of the sum relative to it), int32
    ``rank``, and the alternatives' int32 ``top_ids`` and fp32
    ``top_logprobs`` [T, top]."""
    logprob: object
    rank: object
    entropy: object
    stats: object
    top_ids: object
    top_logprobs: object


class Routing(NamedTuple):
    """The chosen experts of each row, best first: int32 ``ids`` and fp32
    ``weights`` [T, top] (id -1, weight 0 where a row has no more)."""
    ids: object
    weights: object


class Dispatch(NamedTuple):
    """Choices grouped by expert, all int32: ``load`` [E] asked for, ``offsets``
    [E + 1] into ``order`` [N] (pair indices, -1 past offsets[E]), and
    ``position`` (the shape of ids): each pair's place in order, or -1."""
    load: object
    offsets: object
    order: object
    position: object


_TYPES = None
_f32 = _i32 = _i64 = None


def _torch_types():
    global _TYPES, _f32, _i32, _i64
    import torch
    _f32, _i32, _i64 = torch.float32, torch.int32, torch.int64
    _TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _rows(t, name):
    """(pointer, type, T, columns, row stride) of a matrix whose rows are
    contiguous and any distance apart."""
    if _TYPES is None:
        _torch_types()
    kind = _TYPES.get(getattr(t, "dtype", None))
    if kind is None:
        _dev(t, name)                  # no tensor, or not on a GPU
        raise TypeError(f"{name} must be float32, bfloat16 or float16 (got {t.dtype})")
    if not t.is_cuda:
        raise ValueError(f"{name} must live on a GPU (got {t.device})")
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix (got {t.dim()} dimensions)")
    T, C = t.shape
    rs, cs = t.stride()
    if cs != 1 and C > 1:
        raise ValueError(f"{name} must have contiguous rows")
    if T > 1 and rs < C:
        raise ValueError(f"{name} must have rows that do not overlap")
    return t.data_ptr(), kind, T, C, rs if T > 1 else C


def _vec(t, name, dtype, shape):
    """Pointer of a contiguous GPU tensor of this type and shape."""
    try:
        if t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _dev(t, name, dtype)
    raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")


def _new(t, stream, *specs):
    """Uninitialised tensors beside t, of the given (shape, type)s; they belong to
    the stream that the work runs on."""
    if stream is None:
        return [t.new_empty(shape, dtype=dtype) for shape, dtype in specs]
    import torch
    with torch.cuda.stream(stream):
        return [t.new_empty(shape, dtype=dtype) for shape, dtype in specs]


def _workspace(t, stream, nbytes):
    """(tensor to hold, pointer) of a call's workspace."""
    if nbytes == 0:
        return None, None
    w, = _new(t, stream, ((nbytes + 3) // 4, _i32))
    return w, w.data_ptr()


def token_logprobs(logits, tokens=None, top=0, inv_temperature=1.0, out=None, stream=None):
    """bo_token_logprobs: logits [T, V] (fp32, bf16 or fp16 GPU tensor, rows
    any distance apart), tokens int64 [T] (negative: none) or None. Returns a
    TokenLogprobs; ``out`` takes one of the same shapes to write into. Outside
    autograd: the logits' gradient is token_logprobs_grad's."""
    lp, kind, T, V, stride = _rows(logits, "logits")
    top = int(top)
    if top < 0:
        raise ValueError("top must not be negative")
    tp = None if tokens is None else _vec(tokens, "tokens", _i64, (T,))
    specs = (((T,), _f32), ((T,), _i32), ((T,), _f32), ((T, 2), _f32), ((T, top), _i32),
             ((T, top), _f32))
    if out is None:
        out = TokenLogprobs(*_new(logits, stream, *specs))
        ptrs = [t.data_ptr() for t in out]
    else:
        ptrs = [_vec(t, n, d, s) for t, n, (s, d) in zip(out, TokenLogprobs._fields, specs)]
    L = _lib or lib()
    need = L.bo_token_logprobs_workspace(T, V, top)
    ws, wp = _workspace(logits, stream, need)
    st = L.bo_token_logprobs(lp, kind, T, V, stride, tp, inv_temperature, top, *ptrs, wp, need,
                             _stream_of(logits, stream))
    if st:
        _check(st, "bo_token_logprobs")
    return out


def token_logprobs_grad(logits, tokens, stats, entropy, grad_logprob=None, grad_entropy=None,
                        top_ids=None, grad_top=None, inv_temperature=1.0, out=None, stream=None):
    """bo_token_logprobs_grad: the gradient of the logits ([T, V], their type)
    from those of token_logprobs' outputs; ``stats`` and ``entropy`` as it
    returned them. ``out`` may be ``logits`` itself."""
    lp, kind, T, V, stride = _rows(logits, "logits")
    tp = None if tokens is None else _vec(tokens, "tokens", _i64, (T,))
    sp, ep = _vec(stats, "stats", _f32, (T, 2)), _vec(entropy, "entropy", _f32, (T,))
    gl = None if grad_logprob is None else _vec(grad_logprob, "grad_logprob", _f32, (T,))
    gh = None if grad_entropy is None else _vec(grad_entropy, "grad_entropy", _f32, (T,))
    if (top_ids is None) != (grad_top is None):
        raise ValueError("top_ids and grad_top go together")
    top, ip, gp = 0, None, None
    if top_ids is not None:
        top = top_ids.shape[-1]
        ip, gp = _vec(top_ids, "top_ids", _i32, (T, top)), _vec(grad_top, "grad_top", _f32, (T, top))
    if out is None:
        out, = _new(logits, stream, ((T, V), logits.dtype))
    op, okind, oT, oV, ostride = _rows(out, "out")
    if (okind, oT, oV) != (kind, T, V):
        raise ValueError("out must have the logits' shape and type")
    st = (_lib or lib()).bo_token_logprobs_grad(lp, kind, T, V, stride, tp, inv_temperature, sp, ep,
                                                gl, gh, top, ip, gp, op, ostride,
                                                _stream_of(logits, stream))
    if st:
        _check(st, "bo_token_logprobs_grad")
    return out


_SCORES = {"softmax": 0, "sigmoid": 1}


def _score(score):
    if score not in _SCORES:
        raise ValueError(f"score must be 'softmax' or 'sigmoid' (got {score!r})")
    return _SCORES[score]


def route(logits, top, bias=None, score="softmax", groups=1, top_groups=1, group_best=1,
          renormalise=True, scale=1.0, out=None, stream=None):
    """bo_route: each row of logits [T, E] (fp32, bf16 or fp16 GPU tensor, rows
    any distance apart) is sent to its ``top`` best experts. ``bias`` fp32 [E]
    enters the choice only (-inf withdraws an expert); with groups the choice
    is limited to the ``top_groups`` best groups, by the sum of their
    ``group_best`` largest values. Returns a Routing; ``out`` takes one of the
    same shapes to write into. Outside autograd: the logits' gradient is
    route_grad's."""
    lp, kind, T, E, stride = _rows(logits, "logits")
    top = int(top)
    if top < 1:
        raise ValueError("top must be at least 1")
    sc = _score(score)
    bp = None if bias is None else _vec(bias, "bias", _f32, (E,))
    shape = (T, top)
    if out is None:
        out = Routing(*_new(logits, stream, (shape, _i32), (shape, _f32)))
        ip, wp = out.ids.data_ptr(), out.weights.data_ptr()
    else:
        ip, wp = _vec(out[0], "ids", _i32, shape), _vec(out[1], "weights", _f32, shape)
    st = (_lib or lib()).bo_route(lp, kind, T, E, stride, bp, sc, top, groups, top_groups, group_best,
                                  1 if renormalise else 0, scale, ip, wp, _stream_of(logits, stream))
    if st:
        _check(st, "bo_route")
    return out


def route_grad(logits, ids, grad_weights, score="softmax", renormalise=True, scale=1.0, out=None,
               stream=None):
    """bo_route_grad: the gradient of route's logits ([T, E], their type) from
    that of its weights, for the ``ids`` it chose. ``out`` may be ``logits``
    itself."""
    lp, kind, T, E, stride = _rows(logits, "logits")
    if getattr(ids, "ndim", 0) != 2:
        raise TypeError("ids must be an int32 matrix on the GPU")
    top = ids.shape[1]
    ip = _vec(ids, "ids", _i32, (T, top))
    gp = _vec(grad_weights, "grad_weights", _f32, (T, top))
    sc = _score(score)
    if out is None:
        out, = _new(logits, stream, ((T, E), logits.dtype))
    op, okind, oT, oE, ostride = _rows(out, "out")
    if (okind, oT, oE) != (kind, T, E):
        raise ValueError("out must have the logits' shape and type")
    st = (_lib or lib()).bo_route_grad(lp, kind, T, E, stride, sc, top, 1 if renormalise else 0, scale,
                                       ip, gp, op, ostride, _stream_of(logits, stream))
    if st:
        _check(st, "bo_route_grad")
    return out


def dispatch(ids, experts, capacity=0, out=None, stream=None):
    """bo_dispatch: the choices ``ids`` (int32 GPU tensor of any shape, in
    row-major order) grouped by expert, at most ``capacity`` each when that is
    not 0. Returns a Dispatch; ``out`` takes one of the same shapes to write
    into."""
    if _TYPES is None:
        _torch_types()
    idp = _vec(ids, "ids", _i32, getattr(ids, "shape", ()))
    N, E = ids.numel(), int(experts)
    if E < 1:
        raise ValueError("experts must be at least 1")
    specs = (((E,), _i32), ((E + 1,), _i32), ((N,), _i32), (ids.shape, _i32))
    if out is None:
        out = Dispatch(*_new(ids, stream, *specs))
        ptrs = [t.data_ptr() for t in out]
    else:
        ptrs = [_vec(t, n, d, s) for t, n, (s, d) in zip(out, Dispatch._fields, specs)]
    L = _lib or lib()
    need = L.bo_dispatch_workspace(N, E)
    ws, wp = _workspace(ids, stream, need)
    st = L.bo_dispatch(idp, N, E, capacity, *ptrs, wp, need, _stream_of(ids, stream))
    if st:
        _check(st, "bo_dispatch")
    return out


def pareto_front(Y, ref: Optional[np.ndarray] = None) -> np.ndarray:
    """Host: front indices (sorted by objective 0) of Y [n, m] (fp32)."""
    Y = np.ascontiguousarray(np.asarray(Y, dtype=np.float32))
    n, m = Y.shape
    rp = ctypes.c_void_p(0)
    if ref is not None:
        ref = _host_f32(ref, (m,), "ref")
        rp = ref.ctypes.data_as(ctypes.c_void_p)
    idx = np.zeros(max(n, 1), dtype=np.int32)
    cnt = ctypes.c_int32(0)
    _check(lib().bo_pareto_front(Y.ctypes.data_as(ctypes.c_void_p), n, m, rp,
                                 idx.ctypes.data_as(ctypes.c_void_p), n, ctypes.byref(cnt)),
           "bo_pareto_front")
    return idx[:cnt.value].copy()


def box_decomposition(F, ref):
    """Host: disjoint boxes (lo, hi) [B, m] of the region F does not dominate."""
    F = np.ascontiguousarray(np.asarray(F, dtype=np.float32))
    m = np.asarray(ref).shape[0]
    F = F.reshape(-1, m)
    r = _host_f32(ref, (m,), "ref")
    cnt = ctypes.c_int32(0)
    L = lib()
    cap = 4 * F.shape[0] + 8
    while True:
        lo = np.zeros((cap, m), dtype=np.float32)
        hi = np.zeros((cap, m), dtype=np.float32)
        st = L.bo_box_decomposition(F.ctypes.data_as(ctypes.c_void_p), F.shape[0], m,
                                    r.ctypes.data_as(ctypes.c_void_p),
                                    lo.ctypes.data_as(ctypes.c_void_p),
                                    hi.ctypes.data_as(ctypes.c_void_p), cap, ctypes.byref(cnt))
        if st == 3 and cnt.value > cap:
            cap = cnt.value
            continue
        _check(st, "bo_box_decomposition")
        return lo[:cnt.value].copy(), hi[:cnt.value].copy()
