"""Python binding of libstagefrontier: argument marshalling only.

Each function carries the name of the C entry point it calls and forwards
torch tensors as raw device pointers plus the current CUDA stream; every step
of the computation runs in the library's CUDA kernels.  Torch is used for
device memory and streams only.  Missing output tensors are allocated here
(torch.empty) for convenience.  There is no CPU fallback: importing this
module fails if the shared library cannot be loaded.
"""
from __future__ import annotations

import ctypes
import os
from array import array
from dataclasses import dataclass
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libstagefrontier.so")

SF_OK, SF_EINVAL, SF_EINVAL_ALIGN, SF_EUNSUPPORTED, SF_ECUDA, SF_EWORKSPACE = 0, -1, -2, -3, -4, -5
SF_ST_NEGATIVE, SF_ST_RANGE, SF_ST_TIMEOUT, SF_ST_INDEX = 1, 2, 4, 8
SF_ST_NONFINITE = 16
SF_F32, SF_BF16, SF_F16 = 0, 1, 2
SF_SCORE_SOFTMAX, SF_SCORE_SIGMOID = 0, 1
SF_POLICY_DIRECT_ROWS = 1024
SF_ACT_SILU, SF_ACT_GELU, SF_ACT_GELU_TANH, SF_ACT_RELU = 0, 1, 2, 3
SF_VERIFY_MAX_DRAFT = 64
SF_STEP_CONFIDENT = 0x80
LABEL_NAMES = ("frontier_accounting", "direct_exposure", "sync_wait_dependent", "co_critical",
               "role_aware_needed", "telemetry_limited", "raw_only")


class SFError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {_lib.sf_status_str(code).decode()} ({code})")
        self.code = code


class Ratio(ctypes.Structure):
    _fields_ = [("num", ctypes.c_int64), ("den", ctypes.c_int64)]


class LabelConfig(ctypes.Structure):
    _fields_ = [(n, Ratio) for n in ("gamma_A", "gamma_G", "eta_A", "eta_G", "tau_C", "eta_Q",
                                     "gamma_switch", "gamma_elig", "closure_max", "overlap_max")] + \
               [("denom_floor_ns", ctypes.c_int64), ("max_missing_ranks", ctypes.c_int32),
                ("model_fit_mask", ctypes.c_uint32)]


class PolicyConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in ("clip_low", "clip_high", "kl_coef", "inv_temperature")]


class RouteConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("k", "score", "groups", "top_groups", "group_top", "renorm")] + \
               [("scale", ctypes.c_float)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libstagefrontier.so not built at {LIB_PATH}; run "
                          "`python -m paper_2606_06751_gb300.build`")
    L = ctypes.CDLL(LIB_PATH)
    P, I, I32, S = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
    sigs = {
        "sf_frontier": [P, I, I, I, P, P, P, P, S],
        "sf_frontier_ties": [P, I, I, I, P, P, P, S],
        "sf_window_aggregate": [P, I, I, I, I, I, P, P, P, P, P, I32, P, S],
        "sf_topk_suspects": [P, P, I, I, I, I32, P, P, P, P, S],
        "sf_window_baselines": [P, I, I, I, I, I, P, P, P, P, I32, P, S],
        "sf_rank_lag": [P, I, I, I, P, P, P, P, ctypes.c_size_t, P, S],
        "sf_rank_lag_windows": [P, I, I, I, I, I, P, P, I32, P, ctypes.c_size_t, P, S],
        "sf_group_aggregate": [P, I, I, I, P, I, I, I, P, P, I32, P, S],
        "sf_stage_group_sum": [P, I, I, P, I, P, S],
        "sf_raw_spread": [P, I, I, I, I, I, P, I32, P, ctypes.c_size_t, P, S],
        "sf_window_median": [P, I, I, I, I, P, P, S],
        "sf_direct_gain": [P, I, I, I, I, P, P, I32, Ratio, P, P, P, P, P, P, P, P, S],
        "sf_label_gates": [I, I, I, I, P, P, P, P, P, P, P, ctypes.POINTER(LabelConfig), P, P, P, P,
                           P, P, P, S],
        "sf_label_windows": [P, I, I, I, I, P, P, P, I32, ctypes.POINTER(LabelConfig), P,
                             ctypes.c_size_t, P, P, P, P, P, P, P, P, P, S],
        "sf_label_windows_noalloc": [P, I, I, I, I, P, P, P, I32, ctypes.POINTER(LabelConfig), P, P, P,
                                     P, P, P, P, P, P, S],
        "sf_stream_windows": [P, I, I, I, I, I32, I, ctypes.POINTER(LabelConfig), P, ctypes.c_size_t, P,
                              ctypes.c_size_t, P, P, P, P, P, P, P, P, P, P, P, P, P, P, S, S],
        "sf_stream_gathered_windows": [P, I, I, I, I, I32, I, ctypes.POINTER(LabelConfig), P, ctypes.c_size_t, P,
                                       ctypes.c_size_t, P, P, P, P, P, P, P, P, P, P, P, P, P, P, S, S],
        "sf_gathered_to_steps": [P, I, I, I, I, P, S],
        "sf_policy_loss": [P, I32, I, I, I, P, P, P, P, P, ctypes.POINTER(PolicyConfig), P, P, P, P, P, I, P,
                           ctypes.c_size_t, P, S],
        "sf_route_experts": [P, I32, I, I, I, P, ctypes.POINTER(RouteConfig), P, P, P, I32, P, S],
        "sf_route_experts_grad": [P, I32, I, I, I, P, P, ctypes.POINTER(RouteConfig), P, I, P, S],
        "sf_grad_norm": [P, P, P, I, P, P, P, ctypes.c_size_t, P, S],
        "sf_grad_clip": [P, P, P, P, I, ctypes.c_float, ctypes.c_float, P, P, P, P, ctypes.c_size_t, P, S],
        "sf_gated_ffn": [P, I32, I, I, I, P, P, I, I, I32, P, I, P, ctypes.c_size_t, P, S],
        "sf_gated_ffn_grad": [P, I32, I, I, I, P, P, I, I, I32, P, I, P, I, P, P, I32, I, I32, P, I, P,
                              ctypes.c_size_t, P, S],
        "sf_dropout": [P, I32, I, I, I, ctypes.c_float, P, P, I, P, I, S],
        "sf_verify_draft": [P, I32, I, I, I, I, P, I, P, P, P, P, ctypes.c_float, P, P, P, P, S],
    }
    for name, argt in sigs.items():
        f = getattr(L, name)
        f.argtypes = argt
        f.restype = ctypes.c_int
    L.sf_status_str.argtypes = [ctypes.c_int]
    L.sf_status_str.restype = ctypes.c_char_p
    L.sf_num_windows.argtypes = [I, I, I]
    L.sf_num_windows.restype = I
    L.sf_selftest_bounded_wait.argtypes = [ctypes.c_uint64, P, S]
    L.sf_selftest_bounded_wait.restype = ctypes.c_int
    L.sf_launch_count.argtypes = []
    L.sf_launch_count.restype = ctypes.c_uint64
    L.sf_label_config_default.argtypes = [ctypes.POINTER(LabelConfig)]
    L.sf_label_config_default.restype = None
    L.sf_label_windows_workspace_size.argtypes = [I, I, I, I]
    L.sf_label_windows_workspace_size.restype = ctypes.c_size_t
    L.sf_rank_workspace_size.argtypes = [I, I, I]
    L.sf_rank_workspace_size.restype = ctypes.c_size_t
    L.sf_grad_needs_workspace.argtypes = [P, P, I]
    L.sf_grad_needs_workspace.restype = I32
    L.sf_grad_workspace_size.argtypes = [I]
    L.sf_grad_workspace_size.restype = ctypes.c_size_t
    L.sf_policy_loss_workspace_size.argtypes = [I, I]
    L.sf_policy_loss_workspace_size.restype = ctypes.c_size_t
    L.sf_gated_ffn_workspace_size.argtypes = [I32, I, I, I, I32, I32]
    L.sf_gated_ffn_workspace_size.restype = ctypes.c_size_t
    for name in ("sf_stream_windows_staging_size", "sf_stream_gathered_staging_size"):
        getattr(L, name).argtypes = [I, I, I, I]
        getattr(L, name).restype = ctypes.c_size_t
    return L


_lib = _load()


def lib():
    return _lib


def _p(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# the current stream's handle without a Stream object around it (3 us), where torch has that
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _new(shape, dtype, device, stream) -> torch.Tensor:
    """Memory for a result of work on `stream` (None: the current one).  It comes from
    that stream's pool, so that the work follows whatever used the memory before, and
    stays until the current stream, where the caller reads the result, is done with it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    t = _scratch(shape, dtype, device, stream)
    here = torch.cuda.current_stream()
    if stream != here:
        t.record_stream(here)
    return t


def _scratch(shape, dtype, device, stream) -> torch.Tensor:
    """Memory that only work on `stream` uses, from that stream's pool: freed when the
    call returns, it goes to later work on the same stream."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _hold(tensors, stream):
    """Tensors of the caller's that work on `stream` uses: their memory stays until that work is done."""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def _check(rc: int, where: str):
    if rc != SF_OK:
        raise SFError(rc, where)


def _dev(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA tensor of {dtype}")
    return t


def _d3(d: torch.Tensor):
    _dev(d, torch.int64, "d")
    if d.dim() != 3:
        raise ValueError("d must be [T][R][S]")
    return d.shape


def _empty(shape, dtype, like: torch.Tensor, stream):
    return _new(shape, dtype, like.device, stream)


def num_windows(t0: int, T: int, W: int) -> int:
    return int(_lib.sf_num_windows(t0, T, W))


def launch_count() -> int:
    return int(_lib.sf_launch_count())


def default_config() -> LabelConfig:
    c = LabelConfig()
    _lib.sf_label_config_default(ctypes.byref(c))
    return c


def new_status(device) -> torch.Tensor:
    return torch.zeros(1, dtype=torch.int32, device=device)


@dataclass
class Frontier:
    a: Optional[torch.Tensor]
    lead: Optional[torch.Tensor]
    makespan: Optional[torch.Tensor]


def sf_frontier(d, a=None, lead=None, makespan=None, status=None, stream=None, outputs=("a", "lead", "makespan")):
    T, R, S = _d3(d)
    if a is None and "a" in outputs:
        a = _empty((T, S), torch.int64, d, stream)
    if lead is None and "lead" in outputs:
        lead = _empty((T, S), torch.int32, d, stream)
    if makespan is None and "makespan" in outputs:
        makespan = _empty((T,), torch.int64, d, stream)
    _check(_lib.sf_frontier(_p(d), T, R, S, _p(a), _p(lead), _p(makespan), _p(status), _stream(stream)),
           "sf_frontier")
    return Frontier(a, lead, makespan)


def sf_frontier_ties(d, a=None, ties=None, status=None, stream=None):
    """ties[t, s]: how many ranks reach the frontier F[t, s] (Sec. 4's tie set);
    `a` are sf_frontier's increments on the same d (computed here when absent)."""
    T, R, S = _d3(d)
    if a is None:
        a = sf_frontier(d, status=status, stream=stream, outputs=("a",)).a
    ties = ties if ties is not None else _empty((T, S), torch.int32, d, stream)
    _check(_lib.sf_frontier_ties(_p(d), T, R, S, _p(a), _p(ties), _p(status), _stream(stream)),
           "sf_frontier_ties")
    return ties


@dataclass
class Windows:
    X: torch.Tensor
    D: torch.Tensor
    E: Optional[torch.Tensor]
    C: Optional[torch.Tensor]
    step_lead: Optional[torch.Tensor]


def sf_window_aggregate(d, W: int, t0: int = 0, X=None, D=None, E=None, C=None, step_lead=None,
                        accumulate: bool = False, want=("E", "C", "step_lead"), status=None, stream=None):
    T, R, S = _d3(d)
    nW = num_windows(t0, T, W)
    X = X if X is not None else _empty((nW, S), torch.int64, d, stream)
    D = D if D is not None else _empty((nW,), torch.int64, d, stream)
    if E is None and "E" in want:
        E = _empty((nW, S, R), torch.int64, d, stream)
    if C is None and "C" in want:
        C = _empty((nW, S, R), torch.int32, d, stream)
    if step_lead is None and "step_lead" in want:
        step_lead = _empty((T,), torch.uint8, d, stream)
    _check(_lib.sf_window_aggregate(_p(d), T, R, S, t0, W, _p(X), _p(D), _p(E), _p(C), _p(step_lead),
                                    1 if accumulate else 0, _p(status), _stream(stream)),
           "sf_window_aggregate")
    return Windows(X, D, E, C, step_lead)


@dataclass
class TopK:
    stage: torch.Tensor
    stage_value: torch.Tensor
    pair: Optional[torch.Tensor]
    pair_value: Optional[torch.Tensor]


def sf_topk_suspects(X, E, k: int, stream=None, out: Optional[TopK] = None):
    _dev(X, torch.int64, "X")
    nW, S = X.shape
    R = E.shape[2] if E is not None else 1
    if out is None:
        out = TopK(_empty((nW, k), torch.int32, X, stream), _empty((nW, k), torch.int64, X, stream),
                   None if E is None else _empty((nW, k, 2), torch.int32, X, stream),
                   None if E is None else _empty((nW, k), torch.int64, X, stream))
    _check(_lib.sf_topk_suspects(_p(X), _p(E), nW, S, R, k, _p(out.stage), _p(out.stage_value),
                                 _p(out.pair), _p(out.pair_value), _stream(stream)), "sf_topk_suspects")
    return out


def sf_window_median(d, W: int, m=None, status=None, stream=None):
    T, R, S = _d3(d)
    nW = (T + W - 1) // W
    m = m if m is not None else _empty((nW, R, S), torch.int64, d, stream)
    _check(_lib.sf_window_median(_p(d), T, R, S, W, _p(m), _p(status), _stream(stream)), "sf_window_median")
    return m


@dataclass
class Evidence:
    X: torch.Tensor
    Y: torch.Tensor
    D: torch.Tensor
    step_lead: torch.Tensor
    quality: Optional[torch.Tensor]
    E: Optional[torch.Tensor] = None
    C: Optional[torch.Tensor] = None


def sf_direct_gain(d, W: int, m, wall=None, other_stage: int = -1, eta_Q=(1, 20), out: Optional[Evidence] = None,
                   lead_credit: bool = False, status=None, stream=None):
    T, R, S = _d3(d)
    nW = (T + W - 1) // W
    if out is None:
        q = _empty((nW, 6), torch.uint64, d, stream) if (wall is not None or other_stage >= 0) else None
        out = Evidence(_empty((nW, S), torch.int64, d, stream), _empty((nW, S), torch.int64, d, stream),
                       _empty((nW,), torch.int64, d, stream), _empty((T,), torch.uint8, d, stream), q)
        if lead_credit:
            out.E = _empty((nW, S, R), torch.int64, d, stream)
            out.C = _empty((nW, S, R), torch.int32, d, stream)
    _check(_lib.sf_direct_gain(_p(d), T, R, S, W, _p(m), _p(wall), other_stage, Ratio(*eta_Q), _p(out.X),
                               _p(out.Y), _p(out.D), _p(out.E), _p(out.C), _p(out.step_lead), _p(out.quality),
                               _p(status), _stream(stream)), "sf_direct_gain")
    return out


@dataclass
class Labels:
    labels: torch.Tensor
    route_mask: torch.Tensor
    amb_mask: torch.Tensor
    share: torch.Tensor
    gain: torch.Tensor
    n_confident: Optional[torch.Tensor] = None
    n_switch: Optional[torch.Tensor] = None
    X: Optional[torch.Tensor] = None
    Y: Optional[torch.Tensor] = None
    D: Optional[torch.Tensor] = None


def _label_out(nW, S, like, stream):
    return Labels(_empty((nW,), torch.int32, like, stream), _empty((nW,), torch.int32, like, stream),
                  _empty((nW,), torch.int32, like, stream), _empty((nW, S), torch.float64, like, stream),
                  _empty((nW, S), torch.float64, like, stream))


def sf_label_gates(T: int, R: int, S: int, W: int, ev: Evidence, role=None, missing=None, cfg=None,
                   out: Optional[Labels] = None, stream=None):
    nW = (T + W - 1) // W
    cfg = cfg if cfg is not None else default_config()
    if out is None:
        out = _label_out(nW, S, ev.X, stream)
        out.n_confident = _empty((nW,), torch.int32, ev.X, stream)
        out.n_switch = _empty((nW,), torch.int32, ev.X, stream)
    _check(_lib.sf_label_gates(T, R, S, W, _p(ev.X), _p(ev.Y), _p(ev.D), _p(ev.step_lead), _p(ev.quality),
                               _p(role), _p(missing), ctypes.byref(cfg), _p(out.labels), _p(out.route_mask),
                               _p(out.amb_mask), _p(out.share), _p(out.gain), _p(out.n_confident),
                               _p(out.n_switch), _stream(stream)), "sf_label_gates")
    return out


def workspace_size(T: int, R: int, S: int, W: int) -> int:
    return int(_lib.sf_label_windows_workspace_size(T, R, S, W))


def sf_label_windows(d, W: int, role=None, missing=None, wall=None, other_stage: int = -1, cfg=None,
                     workspace=None, out: Optional[Labels] = None, evidence: bool = True, status=None,
                     stream=None):
    T, R, S = _d3(d)
    nW = (T + W - 1) // W
    cfg = cfg if cfg is not None else default_config()
    need = workspace_size(T, R, S, W)
    if workspace is None:
        workspace = _scratch(need, torch.uint8, d.device, stream)
    if out is None:
        out = _label_out(nW, S, d, stream)
        if evidence:
            out.X = _empty((nW, S), torch.int64, d, stream)
            out.Y = _empty((nW, S), torch.int64, d, stream)
            out.D = _empty((nW,), torch.int64, d, stream)
    _check(_lib.sf_label_windows(_p(d), T, R, S, W, _p(role), _p(missing), _p(wall), other_stage,
                                 ctypes.byref(cfg), _p(workspace), workspace.numel(), _p(out.labels),
                                 _p(out.route_mask), _p(out.amb_mask), _p(out.share), _p(out.gain),
                                 _p(out.X), _p(out.Y), _p(out.D), _p(status), _stream(stream)),
           "sf_label_windows")
    return out


STATIC_SCRATCH_BYTES = 16 * 1024 * 1024


def sf_label_windows_noalloc(d, W: int, role=None, missing=None, wall=None, other_stage: int = -1,
                             cfg=None, out: Labels = None, status=None, stream=None):
    """The labeler with its intermediates in the library's static device
    scratch (no workspace; the outputs are still the caller's tensors)."""
    T, R, S = _d3(d)
    cfg = cfg if cfg is not None else default_config()
    if out is None:
        raise ValueError("pass preallocated outputs (Labels with X, Y, D) to the no-allocation entry point")
    _check(_lib.sf_label_windows_noalloc(_p(d), T, R, S, W, _p(role), _p(missing), _p(wall), other_stage,
                                         ctypes.byref(cfg), _p(out.labels), _p(out.route_mask),
                                         _p(out.amb_mask), _p(out.share), _p(out.gain), _p(out.X),
                                         _p(out.Y), _p(out.D), _p(status), _stream(stream)),
           "sf_label_windows_noalloc")
    return out


@dataclass
class Streamed:
    X: torch.Tensor
    Y: torch.Tensor
    D: torch.Tensor
    E: Optional[torch.Tensor]
    C: Optional[torch.Tensor]
    top_stage: torch.Tensor
    top_pair: Optional[torch.Tensor]
    top_pair_value: Optional[torch.Tensor]
    labels: torch.Tensor
    route_mask: torch.Tensor
    amb_mask: torch.Tensor
    share: torch.Tensor
    gain: torch.Tensor


class StreamBuffers:
    """Device staging, workspace and outputs for sf_stream_windows, reusable across calls.  Calls on other
    streams than the current one follow it, or get those streams here."""

    def __init__(self, T: int, R: int, S: int, W: int, k: int, chunk_steps: int, device, lead_credit=True,
                 gathered=False, stream=None, copy_stream=None):
        nW = (T + W - 1) // W
        e = lambda shape, dt: _new(shape, dt, device, stream)  # noqa: E731
        self.shape = (T, R, S, W, k, chunk_steps)
        size = _lib.sf_stream_gathered_staging_size if gathered else _lib.sf_stream_windows_staging_size
        # copies write it first, then `stream` reads it
        self.staging = _new((int(size(T, R, S, chunk_steps)),), torch.uint8, device, copy_stream)
        if stream is not None:
            self.staging.record_stream(stream)
        self.workspace = e((workspace_size(min(chunk_steps, T), R, S, W),), torch.uint8)
        self.out = Streamed(e((nW, S), torch.int64), e((nW, S), torch.int64), e((nW,), torch.int64),
                            e((nW, S, R), torch.int64) if lead_credit else None,
                            e((nW, S, R), torch.int32) if lead_credit else None,
                            e((nW, k), torch.int32), e((nW, k, 2), torch.int32) if lead_credit else None,
                            e((nW, k), torch.int64) if lead_credit else None,
                            e((nW,), torch.int32), e((nW,), torch.int32), e((nW,), torch.int32),
                            e((nW, S), torch.float64), e((nW, S), torch.float64))


def sf_stream_windows(h_d: torch.Tensor, W: int, k: int, chunk_steps: int, bufs: StreamBuffers = None,
                      cfg=None, status=None, stream=None, copy_stream=None) -> Streamed:
    """h_d: [T][R][S] int64 CPU tensor (pin it for copy/compute overlap)."""
    if h_d.is_cuda or h_d.dtype != torch.int64 or not h_d.is_contiguous() or h_d.dim() != 3:
        raise TypeError("h_d must be a contiguous [T][R][S] int64 host tensor")
    T, R, S = h_d.shape
    cfg = cfg if cfg is not None else default_config()
    dev = torch.device("cuda", torch.cuda.current_device())
    cs = copy_stream if copy_stream is not None else (stream if stream is not None else torch.cuda.current_stream())
    if bufs is None:
        bufs = StreamBuffers(T, R, S, W, k, chunk_steps, dev, stream=stream, copy_stream=cs)
    o = bufs.out
    _check(_lib.sf_stream_windows(h_d.data_ptr(), T, R, S, W, k, chunk_steps, ctypes.byref(cfg),
                                  _p(bufs.staging), bufs.staging.numel(), _p(bufs.workspace), bufs.workspace.numel(),
                                  _p(o.X), _p(o.Y), _p(o.D), _p(o.E), _p(o.C), _p(o.top_stage), _p(o.top_pair),
                                  _p(o.top_pair_value), _p(o.labels), _p(o.route_mask), _p(o.amb_mask), _p(o.share),
                                  _p(o.gain), _p(status), _stream(stream), cs.cuda_stream), "sf_stream_windows")
    return o


def sf_selftest_bounded_wait(limit_ns: int, status: torch.Tensor, stream=None):
    _check(_lib.sf_selftest_bounded_wait(limit_ns, _p(status), _stream(stream)), "sf_selftest_bounded_wait")


@dataclass
class Baselines:
    M: torch.Tensor      # [nW][S] sum_t max_r d
    SUM: torch.Tensor    # [nW][S][2] uint64 (lo, hi) of sum_t sum_r d
    SLOW: torch.Tensor   # [nW][S] slowest-rank breakdown
    RANK0: torch.Tensor  # [nW][S] rank-0 local total


def sf_window_baselines(d, W: int, t0: int = 0, out: Optional[Baselines] = None, accumulate: bool = False,
                        status=None, stream=None) -> Baselines:
    T, R, S = _d3(d)
    nW = num_windows(t0, T, W)
    if out is None:
        out = Baselines(_empty((nW, S), torch.int64, d, stream), _empty((nW, S, 2), torch.uint64, d, stream),
                        _empty((nW, S), torch.int64, d, stream), _empty((nW, S), torch.int64, d, stream))
    _check(_lib.sf_window_baselines(_p(d), T, R, S, t0, W, _p(out.M), _p(out.SUM), _p(out.SLOW), _p(out.RANK0),
                                    1 if accumulate else 0, _p(status), _stream(stream)), "sf_window_baselines")
    return out


@dataclass
class Lag:
    L: Optional[torch.Tensor]   # [T][S] F - median_r P
    dL: Optional[torch.Tensor]  # [T][S] increment of the lag over stages
    G: Optional[torch.Tensor]   # [T][S] max-minus-second-max gap


def rank_workspace(T: int, R: int, S: int, device) -> torch.Tensor:
    """Device scratch for sf_rank_lag / sf_raw_spread (reusable across calls)."""
    return torch.empty(int(_lib.sf_rank_workspace_size(T, R, S)), dtype=torch.uint8, device=device)


def sf_rank_lag(d, out: Optional[Lag] = None, workspace=None, status=None, stream=None) -> Lag:
    T, R, S = _d3(d)
    if out is None:
        out = Lag(*(_empty((T, S), torch.int64, d, stream) for _ in range(3)))
    ws = workspace
    if ws is None:
        ws = _scratch(int(_lib.sf_rank_workspace_size(T, R, S)), torch.uint8, d.device, stream)
    _check(_lib.sf_rank_lag(_p(d), T, R, S, _p(out.L), _p(out.dL), _p(out.G), _p(ws), ws.numel(), _p(status),
                            _stream(stream)), "sf_rank_lag")
    return out


def sf_raw_spread(d, W: int, t0: int = 0, spread=None, accumulate: bool = False, workspace=None, status=None,
                  stream=None):
    T, R, S = _d3(d)
    spread = spread if spread is not None else _empty((num_windows(t0, T, W), S), torch.int64, d, stream)
    ws = workspace
    if ws is None:
        ws = _scratch(int(_lib.sf_rank_workspace_size(T, R, S)), torch.uint8, d.device, stream)
    _check(_lib.sf_raw_spread(_p(d), T, R, S, t0, W, _p(spread), 1 if accumulate else 0, _p(ws), ws.numel(),
                              _p(status), _stream(stream)), "sf_raw_spread")
    return spread


@dataclass
class GroupWindows:
    X: torch.Tensor  # [nW][G][S] sums of the group frontier's increments
    D: torch.Tensor  # [nW][G] sums of the group makespans


def sf_group_aggregate(d, group, G: int, W: int, t0: int = 0, out: Optional[GroupWindows] = None,
                       accumulate: bool = False, status=None, stream=None) -> GroupWindows:
    T, R, S = _d3(d)
    group = _dev(group, torch.int32, "group")
    nW = num_windows(t0, T, W)
    if out is None:
        out = GroupWindows(_empty((nW, G, S), torch.int64, d, stream), _empty((nW, G), torch.int64, d, stream))
    _check(_lib.sf_group_aggregate(_p(d), T, R, S, _p(group), G, t0, W, _p(out.X), _p(out.D),
                                   1 if accumulate else 0, _p(status), _stream(stream)), "sf_group_aggregate")
    return out


def sf_stage_group_sum(X, stage_group, K: int, Y=None, stream=None):
    """stage_group: a host sequence of S group ids in [0, K)."""
    nW, S = X.shape
    sg = (ctypes.c_int32 * S)(*[int(v) for v in stage_group])
    Y = Y if Y is not None else _empty((nW, K), torch.int64, X, stream)
    _check(_lib.sf_stage_group_sum(_p(X), nW, S, sg, K, _p(Y), _stream(stream)), "sf_stage_group_sum")
    return Y


def sf_stream_gathered_windows(h_g: torch.Tensor, T: int, R: int, S: int, W: int, k: int, chunk_steps: int,
                               bufs: StreamBuffers = None, cfg=None, status=None, stream=None,
                               copy_stream=None) -> Streamed:
    """h_g: int64 CPU tensor holding the windows' gathered [R][n][S] blocks one
    after another (T*R*S values; pin it for copy/compute overlap)."""
    if h_g.is_cuda or h_g.dtype != torch.int64 or not h_g.is_contiguous() or h_g.numel() != T * R * S:
        raise TypeError("h_g must be a contiguous int64 host tensor of T*R*S values")
    cfg = cfg if cfg is not None else default_config()
    dev = torch.device("cuda", torch.cuda.current_device())
    cs = copy_stream if copy_stream is not None else (stream if stream is not None else torch.cuda.current_stream())
    if bufs is None:
        bufs = StreamBuffers(T, R, S, W, k, chunk_steps, dev, gathered=True, stream=stream, copy_stream=cs)
    o = bufs.out
    _check(_lib.sf_stream_gathered_windows(h_g.data_ptr(), T, R, S, W, k, chunk_steps, ctypes.byref(cfg),
                                           _p(bufs.staging), bufs.staging.numel(), _p(bufs.workspace),
                                           bufs.workspace.numel(), _p(o.X), _p(o.Y), _p(o.D), _p(o.E), _p(o.C),
                                           _p(o.top_stage), _p(o.top_pair), _p(o.top_pair_value), _p(o.labels),
                                           _p(o.route_mask), _p(o.amb_mask), _p(o.share), _p(o.gain), _p(status),
                                           _stream(stream), cs.cuda_stream), "sf_stream_gathered_windows")
    return o


def sf_gathered_to_steps(src: torch.Tensor, T: int, R: int, S: int, N: int, dst=None, stream=None):
    """src: device int64 holding ceil(T/N) gathered [R][n][S] blocks; returns [T][R][S]."""
    if not src.is_cuda or src.dtype != torch.int64 or not src.is_contiguous() or src.numel() != T * R * S:
        raise TypeError("src must be a contiguous int64 CUDA tensor of T*R*S values")
    dst = dst if dst is not None else _empty((T, R, S), torch.int64, src, stream)
    _check(_lib.sf_gathered_to_steps(_p(src), T, R, S, N, _p(dst), _stream(stream)), "sf_gathered_to_steps")
    return dst


def sf_rank_lag_windows(d, W: int, t0: int = 0, Lw=None, Gw=None, accumulate: bool = False, workspace=None,
                        status=None, stream=None):
    """Window sums of the lag and the gap: (Lw, Gw), each [nW][S]."""
    T, R, S = _d3(d)
    nW = num_windows(t0, T, W)
    Lw = Lw if Lw is not None else _empty((nW, S), torch.int64, d, stream)
    Gw = Gw if Gw is not None else _empty((nW, S), torch.int64, d, stream)
    ws = workspace
    if ws is None:
        ws = _scratch(int(_lib.sf_rank_workspace_size(T, R, S)), torch.uint8, d.device, stream)
    _check(_lib.sf_rank_lag_windows(_p(d), T, R, S, t0, W, _p(Lw), _p(Gw), 1 if accumulate else 0, _p(ws),
                                    ws.numel(), _p(status), _stream(stream)), "sf_rank_lag_windows")
    return Lw, Gw


# ---------------------------------------------------------------- training-step operators

_DTYPES = {torch.float32: SF_F32, torch.bfloat16: SF_BF16, torch.float16: SF_F16}


def _rows(t: torch.Tensor, name: str):
    """(rows, columns, row stride) of a CUDA matrix whose rows are contiguous."""
    try:
        n, m = t.shape
        fine = t.is_cuda and t.dtype in _DTYPES
    except (AttributeError, TypeError, ValueError):
        fine = False
    if not fine:
        raise TypeError(f"{name} must be a CUDA matrix of float32, bfloat16 or float16")
    ld, one = t.stride()
    if m > 1 and one != 1:
        raise TypeError(f"{name} must have contiguous rows")
    return n, m, (ld if n > 1 else m)


def _vec(t: Optional[torch.Tensor], n: int, dtype, name: str):
    if t is not None:
        _dev(t, dtype, name)
        if t.numel() != n:
            raise ValueError(f"{name} must have {n} elements")
    return t


@dataclass
class PolicyLoss:
    logp: Optional[torch.Tensor]
    token_loss: Optional[torch.Tensor]
    stats: torch.Tensor
    dlogits: Optional[torch.Tensor]


def sf_policy_loss(logits, target, old_logp, advantage, ref_logp=None, weight=None, clip=(0.2, 0.2),
                   kl_coef: float = 0.0, inv_temperature: float = 1.0, grad: bool = False, grad_out=None, logp=None,
                   token_loss=None, stats=None, dlogits=None, want=("logp", "token_loss"), workspace=None,
                   status=None, stream=None) -> PolicyLoss:
    """Clipped policy loss with a KL term of N tokens from their logits [N][V];
    `stats` holds the weighted sums (loss, policy term, KL, clipped share).
    With `grad` (or a `dlogits` to write, which may be `logits` itself) also
    the gradient of the logits for the upstream gradient `grad_out` (a device
    scalar, 1 if absent).  Tokens of weight 0 are not read."""
    N, V, ld = _rows(logits, "logits")
    _vec(target, N, torch.int64, "target")
    _vec(old_logp, N, torch.float32, "old_logp")
    _vec(advantage, N, torch.float32, "advantage")
    _vec(ref_logp, N, torch.float32, "ref_logp")
    _vec(weight, N, torch.float32, "weight")
    _vec(grad_out, 1, torch.float32, "grad_out")
    new = lambda n, dtype=torch.float32: _new(n, dtype, logits.device, stream)  # noqa: E731
    if logp is not None:
        _vec(logp, N, torch.float32, "logp")
    elif "logp" in want:
        logp = new(N)
    if token_loss is not None:
        _vec(token_loss, N, torch.float32, "token_loss")
    elif "token_loss" in want:
        token_loss = new(N)
    stats = new(4) if stats is None else _vec(stats, 4, torch.float32, "stats")
    ldd = V
    if dlogits is not None:
        n, m, ldd = _rows(dlogits, "dlogits")
        if (n, m) != (N, V) or dlogits.dtype != logits.dtype:
            raise ValueError("dlogits must have logits' shape and type")
    elif grad:
        dlogits = new((N, V), logits.dtype)
    if workspace is None and (logp is None or N > SF_POLICY_DIRECT_ROWS):
        workspace = _scratch(_lib.sf_policy_loss_workspace_size(N, V), torch.uint8, logits.device, stream)
    cfg = PolicyConfig(clip[0], clip[1], kl_coef, inv_temperature)
    _check(_lib.sf_policy_loss(_p(logits), _DTYPES[logits.dtype], N, V, ld, _p(target), _p(old_logp), _p(ref_logp),
                               _p(advantage), _p(weight), ctypes.byref(cfg), _p(grad_out), _p(logp), _p(token_loss),
                               _p(stats), _p(dlogits), ldd, _p(workspace), 0 if workspace is None else workspace.numel(),
                               _p(status),
                               _stream(stream)), "sf_policy_loss")
    return PolicyLoss(logp, token_loss, stats, dlogits)


_SCORES = {"softmax": SF_SCORE_SOFTMAX, "sigmoid": SF_SCORE_SIGMOID}


@dataclass
class Routing:
    index: torch.Tensor
    weight: torch.Tensor
    load: Optional[torch.Tensor]


def _score(score: str) -> int:
    if score not in _SCORES:
        raise ValueError(f"score must be one of {', '.join(_SCORES)}")
    return _SCORES[score]


def sf_route_experts(logits, k: int, bias=None, score: str = "softmax", groups: int = 1, top_groups: int = 1,
                     group_top: int = 2, renorm: bool = True, scale: float = 1.0, index=None, weight=None, load=None,
                     accumulate: bool = False, want=("load",), status=None, stream=None) -> Routing:
    """Tokens' k experts from router logits [T][E]: index and weight [T][k] by
    falling choice value, and the experts' loads [E] (added to `load` with
    `accumulate`).  `bias` [E] takes part in the choice only."""
    T, E, ld = _rows(logits, "logits")
    _vec(bias, E, torch.float32, "bias")
    if accumulate and load is None:
        raise ValueError("accumulate adds to a load that the caller gives")
    new = lambda shape, dtype: _new(shape, dtype, logits.device, stream)  # noqa: E731
    slots = T * k if k > 0 else 0  # a bad k is the library's to refuse
    index = new((T, max(k, 0)), torch.int32) if index is None else _vec(index, slots, torch.int32, "index")
    weight = new((T, max(k, 0)), torch.float32) if weight is None else _vec(weight, slots, torch.float32, "weight")
    if load is not None:
        _vec(load, E, torch.int32, "load")
    elif "load" in want:
        load = new(E, torch.int32)
    cfg = RouteConfig(k, _score(score), groups, top_groups, group_top, 1 if renorm else 0, scale)
    _check(_lib.sf_route_experts(_p(logits), _DTYPES[logits.dtype], T, E, ld, _p(bias), ctypes.byref(cfg), _p(index),
                                 _p(weight), _p(load), 1 if accumulate else 0, _p(status), _stream(stream)),
           "sf_route_experts")
    return Routing(index, weight, load)


def sf_route_experts_grad(logits, index, dweight, score: str = "softmax", renorm: bool = True, scale: float = 1.0,
                          dlogits=None, status=None, stream=None) -> torch.Tensor:
    """The gradient of the router's logits from that of its weights [T][k]."""
    T, E, ld = _rows(logits, "logits")
    _dev(index, torch.int32, "index")
    if index.dim() != 2 or index.shape[0] != T:
        raise ValueError("index must be [T][k]")
    k = index.shape[1]
    _vec(dweight, T * k, torch.float32, "dweight")
    ldd = E
    if dlogits is None:
        dlogits = _empty((T, E), logits.dtype, logits, stream)
    else:
        n, m, ldd = _rows(dlogits, "dlogits")
        if (n, m) != (T, E) or dlogits.dtype != logits.dtype:
            raise ValueError("dlogits must have logits' shape and type")
    cfg = RouteConfig(k, _score(score), 1, 1, 1, 1 if renorm else 0, scale)
    _check(_lib.sf_route_experts_grad(_p(logits), _DTYPES[logits.dtype], T, E, ld, _p(index), _p(dweight),
                                      ctypes.byref(cfg), _p(dlogits), ldd, _p(status), _stream(stream)),
           "sf_route_experts_grad")
    return dlogits


@dataclass
class GradNorm:
    norm: torch.Tensor
    coef: Optional[torch.Tensor]
    tensor_norm: Optional[torch.Tensor]


# as C calls over a whole list: half the time of a loop (0.2 us a tensor)
_is_cuda, _dtype_of = torch.Tensor.is_cuda.__get__, torch.Tensor.dtype.__get__


def _tensor_list(tensors, name: str):
    """Host arrays (pointers, sizes, types) of contiguous CUDA tensors."""
    try:
        types = array("i", map(_DTYPES.__getitem__, map(_dtype_of, tensors)))
        fine = all(map(_is_cuda, tensors)) and all(map(torch.Tensor.is_contiguous, tensors))
    except (KeyError, TypeError):
        fine = False
    if not fine:
        raise TypeError(f"{name} must be contiguous CUDA tensors of float32, bfloat16 or float16")
    return array("Q", map(torch.Tensor.data_ptr, tensors)), array("q", map(torch.Tensor.numel, tensors)), types


def _grad(grads, out, max_norm, eps, norm, coef, tensor_norm, per_tensor, workspace, status, stream):
    grads = list(grads)
    n = len(grads)
    ptr, numel, dtype = _tensor_list(grads, "grads")
    device = grads[0].device if n else torch.device("cuda", torch.cuda.current_device())
    out_ptr = None
    if out is not None:
        out_ptr, out_numel, out_dtype = _tensor_list(list(out), "out")
        if out_numel != numel or out_dtype != dtype:
            raise ValueError("out must have the gradients' sizes and types")
    new = lambda m: _new(m, torch.float32, device, stream)  # noqa: E731
    norm = new(1) if norm is None else _vec(norm, 1, torch.float32, "norm")
    if tensor_norm is not None:
        _vec(tensor_norm, n, torch.float32, "tensor_norm")
    elif per_tensor:
        tensor_norm = new(n)
    at = lambda a: a.buffer_info()[0]  # noqa: E731
    if workspace is None and _lib.sf_grad_needs_workspace(at(numel), at(dtype), n):
        workspace = _scratch(_lib.sf_grad_workspace_size(n), torch.uint8, device, stream)
    size = 0 if workspace is None else workspace.numel()
    if max_norm is None:
        _check(_lib.sf_grad_norm(at(ptr), at(numel), at(dtype), n, _p(norm), _p(tensor_norm), _p(workspace), size,
                                 _p(status), _stream(stream)), "sf_grad_norm")
        return GradNorm(norm, None, tensor_norm)
    coef = new(1) if coef is None else _vec(coef, 1, torch.float32, "coef")
    _check(_lib.sf_grad_clip(at(ptr), None if out_ptr is None else at(out_ptr), at(numel), at(dtype), n, max_norm, eps,
                             _p(norm), _p(coef), _p(tensor_norm), _p(workspace), size, _p(status), _stream(stream)),
           "sf_grad_clip")
    return GradNorm(norm, coef, tensor_norm)


def sf_grad_norm(grads, per_tensor: bool = False, norm=None, tensor_norm=None, workspace=None, status=None,
                 stream=None) -> GradNorm:
    """The 2-norm over a sequence of gradient tensors and, with `per_tensor`, of each."""
    return _grad(grads, None, None, 0.0, norm, None, tensor_norm, per_tensor, workspace, status, stream)


def sf_grad_clip(grads, max_norm: float, out=None, eps: float = 1e-6, per_tensor: bool = False, norm=None, coef=None,
                 tensor_norm=None, workspace=None, status=None, stream=None) -> GradNorm:
    """sf_grad_norm, then the gradients times coef = min(1, max_norm / (norm + eps)):
    in place, or into the tensors of `out`.  Where the norm is not finite, coef is
    NaN and the gradients stay as they are."""
    return _grad(grads, out, max_norm, eps, norm, coef, tensor_norm, per_tensor, workspace, status, stream)


# ---------------------------------------------------------------- the operators around a policy's layers

_ACTS = {"silu": SF_ACT_SILU, "gelu": SF_ACT_GELU, "gelu_tanh": SF_ACT_GELU_TANH, "relu": SF_ACT_RELU}


# the current device without torch's initialisation around it, where torch has that
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _here(tensors) -> int:
    """The current device, which the launches go to and the tensors given have to be on."""
    d = _device()
    for t in tensors:
        if t is not None and t.get_device() != d:
            raise ValueError("tensors must be on the current CUDA device")
    return d


def _on(stream, d: int) -> int:
    return _raw_stream(d) if stream is None and _raw_stream is not None else _stream(stream)


def _like_rows(t, shape, dtypes, name: str):
    """The row stride of an output matrix that has to be of this shape and type."""
    n, m, ld = _rows(t, name)
    if (n, m) != shape or t.dtype not in dtypes:
        raise ValueError(f"{name} must be {list(shape)} of {' or '.join(map(str, dtypes))}")
    return ld


def _ffn_inputs(x, w_gate, w_up, act: str):
    """(T, H, F, ldx, ldw, activation, whether all rows start on 16 bytes, the three pointers)"""
    T, H, ldx = _rows(x, "x")
    F, h, ldw = _rows(w_gate, "w_gate")
    if h != H or w_gate.dtype != x.dtype:
        raise ValueError("w_gate must be [F][H] of x's type")
    if _like_rows(w_up, (F, H), (x.dtype,), "w_up") != ldw:
        raise ValueError("w_gate and w_up must have one row spacing")
    number = _ACTS.get(act)
    if number is None:
        raise ValueError(f"act must be one of {', '.join(_ACTS)}")
    size = 4 if x.dtype == torch.float32 else 2
    px, pg, pu = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr()
    even = (px | pg | pu | (ldx * size if T > 1 else 0) | (ldw * size if F > 1 else 0)) % 16 == 0
    return T, H, F, ldx, ldw, number, even, px, pg, pu


def _ffn_workspace(x, T, H, F, even, grad, stream):
    n = _lib.sf_gated_ffn_workspace_size(_DTYPES[x.dtype], T, H, F, 1 if even else 0, grad)
    return None if n == 0 else _scratch(n, torch.uint8, x.device, stream)


def sf_gated_ffn(x, w_gate, w_up, act: str = "silu", h=None, workspace=None, status=None, stream=None) -> torch.Tensor:
    """The gated feed-forward product act(x w_gate^T) * (x w_up^T) [T][F] of x [T][H]
    and weights [F][H], all of one type."""
    T, H, F, ldx, ldw, number, even, px, pg, pu = _ffn_inputs(x, w_gate, w_up, act)
    d = _here((x, w_gate, w_up, h, workspace, status))
    if h is None:
        h, ldh = _new((T, F), x.dtype, x.device, stream), F
    else:
        ldh = _like_rows(h, (T, F), (x.dtype,), "h")
    if workspace is None:
        workspace = _ffn_workspace(x, T, H, F, even, 0, stream)
    if stream is not None:
        _hold((h, workspace), stream)
    _check(_lib.sf_gated_ffn(px, _DTYPES[x.dtype], T, H, ldx, pg, pu, F, ldw, number, h.data_ptr(), ldh, _p(workspace),
                             0 if workspace is None else workspace.numel(), _p(status), _on(stream, d)), "sf_gated_ffn")
    return h


@dataclass
class GatedFfnGrad:
    dx: Optional[torch.Tensor]
    dw_gate: Optional[torch.Tensor]
    dw_up: Optional[torch.Tensor]
    h: Optional[torch.Tensor]


def sf_gated_ffn_grad(x, w_gate, w_up, dh, act: str = "silu", dx=None, dw_gate=None, dw_up=None, h=None,
                      accumulate: bool = False, want=("dx", "dw"), dw_dtype=None, workspace=None, status=None,
                      stream=None) -> GatedFfnGrad:
    """The gradients of sf_gated_ffn's inputs from that of its result, dh [T][F]: of
    x, and of both weights (of x's type or float32; added to the tensors given with
    `accumulate`).  With "h" in `want` the product itself once more."""
    T, H, F, ldx, ldw, number, even, px, pg, pu = _ffn_inputs(x, w_gate, w_up, act)
    dtype, device = x.dtype, x.device
    lddh = _like_rows(dh, (T, F), (dtype,), "dh")
    d = _here((x, w_gate, w_up, dh, dx, dw_gate, dw_up, h, workspace, status))
    if (dw_gate is None) != (dw_up is None):
        raise ValueError("dw_gate and dw_up go together")
    lddx, lddw, ldh = H, H, F
    if dx is not None:
        lddx = _like_rows(dx, (T, H), (dtype,), "dx")
    elif "dx" in want:
        dx = _new((T, H), dtype, device, stream)
    if dw_gate is not None:
        lddw = _like_rows(dw_gate, (F, H), (dtype, torch.float32), "dw_gate")
        if _like_rows(dw_up, (F, H), (dw_gate.dtype,), "dw_up") != lddw:
            raise ValueError("dw_gate and dw_up must have one row spacing")
    elif accumulate:
        raise ValueError("accumulate adds to gradients that the caller gives")
    elif "dw" in want:
        if dw_dtype is None:
            dw_dtype = dtype
        elif dw_dtype is not dtype and dw_dtype is not torch.float32:
            raise ValueError("dw_dtype must be x's type or float32")
        dw_gate = _new((F, H), dw_dtype, device, stream)
        dw_up = _new((F, H), dw_dtype, device, stream)
    if h is not None:
        ldh = _like_rows(h, (T, F), (dtype,), "h")
    elif "h" in want:
        h = _new((T, F), dtype, device, stream)
    if workspace is None:
        workspace = _ffn_workspace(x, T, H, F, even, 1, stream)
    if stream is not None:
        _hold((dx, dw_gate, dw_up, h, workspace), stream)
    _check(_lib.sf_gated_ffn_grad(px, _DTYPES[dtype], T, H, ldx, pg, pu, F, ldw, number, dh.data_ptr(), lddh, _p(dx), lddx,
                                  _p(dw_gate), _p(dw_up), SF_F32 if dw_gate is None else _DTYPES[dw_gate.dtype], lddw,
                                  1 if accumulate else 0, _p(h), ldh, _p(workspace),
                                  0 if workspace is None else workspace.numel(), _p(status), _on(stream, d)),
           "sf_gated_ffn_grad")
    return GatedFfnGrad(dx, dw_gate, dw_up, h)


def sf_dropout(x, p: float, key, residual=None, out=None, stream=None) -> torch.Tensor:
    """residual + x [N][D], each value of x kept with probability 1 - p and scaled.
    The mask comes from `key` (int64 [2] on the device: seed and offset) and is not
    stored; the same call on the gradient, without residual, is the backward pass.
    `out` may be x or residual itself."""
    N, D, ldx = _rows(x, "x")
    _vec(key, 2, torch.int64, "key")
    d = _here((x, key, residual, out))
    dtype = x.dtype
    ldr = ldo = D
    if residual is not None:
        ldr = _like_rows(residual, (N, D), (dtype,), "residual")
    if out is None:
        out = _new((N, D), dtype, x.device, stream)
    else:
        ldo = _like_rows(out, (N, D), (dtype,), "out")
    _check(_lib.sf_dropout(x.data_ptr(), _DTYPES[dtype], N, D, ldx, p, key.data_ptr(), _p(residual), ldr, out.data_ptr(),
                           ldo, _on(stream, d)), "sf_dropout")
    return out


@dataclass
class Verified:
    token: torch.Tensor
    accepted: torch.Tensor
    logp: Optional[torch.Tensor]


def _row_stack(t, shape, dtype, name: str):
    """The row stride of a [B][n][V] tensor whose rows are evenly spaced."""
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name} must be {list(shape)} of {dtype}")
    B, n, V = shape
    far, ld, one = t.stride()
    if V > 1 and one != 1:
        raise TypeError(f"{name} must have contiguous rows")
    if n > 1 and B > 1 and far != n * ld:
        raise TypeError(f"{name}'s rows must be evenly spaced")
    return ld if n > 1 else far if B > 1 and n > 0 else V


def sf_verify_draft(target, token, draft=None, lengths=None, uniform=None, noise=None, inv_temperature: float = 1.0,
                    out_token=None, accepted=None, logp=None, want=("logp",), status=None, stream=None) -> Verified:
    """Drafted tokens [B][L] against the policy's logits [B][L + 1][V]: the tokens
    that are kept with the next one, then -1 ([B][L + 1]), how many drafted ones
    were accepted [B], and the log-probabilities of the tokens (the old_logp of
    sf_policy_loss).  `draft` [B][L][V] are the logits that the tokens were drawn
    from (absent: they were looked up), `lengths` [B] the drafted tokens of each
    sequence, `uniform` [B][L] and `noise` [B][V] (exponential) the random numbers;
    without them the choice is greedy."""
    _dev(token, torch.int64, "token")
    if token.dim() != 2:
        raise ValueError("token must be [B][L]")
    B, L = token.shape
    for t in (target, draft):
        if t is not None and not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in _DTYPES and t.dim() == 3):
            raise TypeError("target and draft must be CUDA tensors [B][rows][V] of float32, bfloat16 or float16")
    dtype, device = target.dtype, target.device
    V = target.shape[2]
    ldt = _row_stack(target, (B, L + 1, V), dtype, "target")
    ldq = V if draft is None else _row_stack(draft, (B, L, V), dtype, "draft")
    _vec(lengths, B, torch.int32, "lengths")
    _vec(uniform, B * L, torch.float32, "uniform")
    _vec(noise, B * V, torch.float32, "noise")
    if (uniform is None) != (noise is None):
        raise ValueError("uniform and noise go together")
    d = _here((target, token, draft, lengths, uniform, noise, out_token, accepted, logp, status))
    if out_token is None:
        out_token = _new((B, L + 1), torch.int64, device, stream)
    else:
        _vec(out_token, B * (L + 1), torch.int64, "out_token")
    if accepted is None:
        accepted = _new(B, torch.int32, device, stream)
    else:
        _vec(accepted, B, torch.int32, "accepted")
    if logp is not None:
        _vec(logp, B * (L + 1), torch.float32, "logp")
    elif "logp" in want:
        logp = _new((B, L + 1), torch.float32, device, stream)
    if stream is not None:
        _hold((out_token, accepted, logp), stream)
    _check(_lib.sf_verify_draft(target.data_ptr(), _DTYPES[dtype], B, L, V, ldt, _p(draft), ldq, token.data_ptr(),
                                _p(lengths), _p(uniform), _p(noise), inv_temperature, out_token.data_ptr(),
                                accepted.data_ptr(), _p(logp), _p(status), _on(stream, d)), "sf_verify_draft")
    return Verified(out_token, accepted, logp)
