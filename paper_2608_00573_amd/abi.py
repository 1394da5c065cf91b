"""ctypes binding of libtrimmoe (include/trimmoe.h): marshalling only.

Every step of the adaptive-depth MoE layer runs inside the HIP library;
this module only mirrors the C structs, passes device pointers taken from
torch tensors (torch provides device memory and streams) and turns status
codes into exceptions.  There is no fallback: if the library is missing
the import of ``lib()`` raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import NamedTuple

import numpy as np

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtrimmoe.so")

ABI_VERSION = 6   # TRIMMOE_ABI_VERSION this binding is written for
STATIC_SCRATCH_BYTES = 64 << 20  # TRIMMOE_STATIC_SCRATCH_BYTES
N_COUNTERS = 16   # per-layer trace counters (row stride of trimmoe_trace.counters)
TRIMMOE_OK = 0
TRIMMOE_ERR_SHAPE = -2
STATUS = {0: "OK", -1: "ERR_NULL", -2: "ERR_SHAPE", -3: "ERR_DTYPE", -4: "ERR_POLICY",
          -5: "ERR_LAYER", -6: "ERR_WORKSPACE", -7: "ERR_HIP"}
F32, BF16 = 0, 1
ACT_RELU, ACT_SWIGLU = 0, 1
CONF_SOFTMAX, CONF_SIGMOID = 0, 1
MAX_EXPERTS, MAX_TOPK = 256, 8


class Layer(C.Structure):
    _fields_ = [("w_router", C.c_void_p), ("b_router", C.c_void_p),
                ("w_up", C.c_void_p), ("w_gate", C.c_void_p), ("w_down", C.c_void_p),
                ("ws_up", C.c_void_p), ("ws_gate", C.c_void_p), ("ws_down", C.c_void_p),
                ("w_exit", C.c_void_p), ("b_exit", C.c_void_p),
                ("local_mask", C.c_void_p), ("sim", C.c_void_p),
                ("theta", C.c_float), ("skip_slope", C.c_float),
                ("trans_to", C.c_void_p), ("trans_p", C.c_void_p)]


class Model(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_experts", C.c_int32),
                ("top_k", C.c_int32), ("d_ff", C.c_int32), ("d_ff_shared", C.c_int32),
                ("vocab_exit", C.c_int32), ("dtype", C.c_int32), ("act", C.c_int32),
                ("conf_mode", C.c_int32), ("normalize_topk", C.c_int32),
                ("layers", C.POINTER(Layer)), ("trans_b", C.c_int32)]


class Policy(C.Structure):
    _fields_ = [("p_exit", C.c_float), ("budget", C.c_float), ("omega_t", C.c_float),
                ("t_local", C.c_float), ("t_remote", C.c_float), ("phi_scale", C.c_float),
                ("sim_min", C.c_float), ("p_exit_tok", C.c_void_p),
                ("budget_tok", C.c_void_p), ("horizon", C.c_int32), ("la_subs", C.c_int32)]


class State(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("h", C.c_void_p), ("d_acc", C.c_void_p),
                ("active_idx", C.c_void_p), ("n_active", C.c_void_p),
                ("exit_layer", C.c_void_p), ("xi", C.c_void_p)]


class Trace(C.Structure):
    _fields_ = [("action", C.c_void_p), ("target", C.c_void_p), ("exec", C.c_void_p),
                ("kind", C.c_void_p), ("gate", C.c_void_p), ("importance", C.c_void_p),
                ("xi", C.c_void_p), ("d_acc", C.c_void_p), ("counters", C.c_void_p)]


EXPORTS = ["trimmoe_abi_version", "trimmoe_status_str", "trimmoe_workspace_size",
           "trimmoe_state_reset", "trimmoe_layer_step", "trimmoe_stack_forward",
           "trimmoe_stack_forward_timed", "trimmoe_stack_forward_static",
           "trimmoe_set_clock_record",
           "trimmoe_window_stats", "trimmoe_feedback_update",
           "trimmoe_calib_exit_layers", "trimmoe_calib_stats", "trimmoe_calib_transitions",
           "trimmoe_place_replicas", "trimmoe_head_argmax_workspace_size",
           "trimmoe_head_argmax", "trimmoe_consistency_labels",
           "trimmoe_train_exit_head_workspace_size",
           "trimmoe_train_exit_head",
           "trimmoe_head_cross_entropy_workspace_size", "trimmoe_head_cross_entropy",
           "trimmoe_head_cross_entropy_backward_workspace_size",
           "trimmoe_head_cross_entropy_backward",
           "trimmoe_balance_loss_workspace_size", "trimmoe_balance_loss",
           "trimmoe_balance_loss_backward_workspace_size", "trimmoe_balance_loss_backward",
           "trimmoe_checkpoint_pack", "trimmoe_checkpoint_unpack",
           "trimmoe_expert_ffn_workspace_size", "trimmoe_expert_ffn",
           "trimmoe_expert_ffn_backward_workspace_size", "trimmoe_expert_ffn_backward"]
TIMED_CLASSES = ["route", "bucket", "up", "down", "shared", "combine", "exit", "gate"]

_lib = None


def lib():
    """The loaded libtrimmoe.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "paper_2608_00573_amd.build.build() (there is no fallback)")
        L = C.CDLL(LIB_PATH)
        L.trimmoe_abi_version.restype = C.c_int
        L.trimmoe_status_str.restype = C.c_char_p
        L.trimmoe_status_str.argtypes = [C.c_int]
        L.trimmoe_workspace_size.restype = C.c_int
        L.trimmoe_workspace_size.argtypes = [C.POINTER(Model), C.c_int32, C.POINTER(C.c_size_t)]
        L.trimmoe_state_reset.restype = C.c_int
        L.trimmoe_state_reset.argtypes = [C.POINTER(Model), C.POINTER(State), C.c_void_p]
        L.trimmoe_layer_step.restype = C.c_int
        L.trimmoe_layer_step.argtypes = [C.POINTER(Model), C.c_int32, C.POINTER(Policy),
                                         C.POINTER(State), C.POINTER(Trace), C.c_void_p,
                                         C.c_size_t, C.c_void_p]
        L.trimmoe_stack_forward.restype = C.c_int
        L.trimmoe_stack_forward.argtypes = [C.POINTER(Model), C.POINTER(Policy),
                                            C.POINTER(State), C.POINTER(Trace), C.c_void_p,
                                            C.c_size_t, C.c_void_p]
        L.trimmoe_stack_forward_timed.restype = C.c_int
        L.trimmoe_stack_forward_timed.argtypes = [C.POINTER(Model), C.POINTER(Policy),
                                                  C.POINTER(State), C.POINTER(Trace),
                                                  C.c_void_p, C.c_size_t, C.c_void_p,
                                                  C.POINTER(C.c_void_p), C.c_int32]
        L.trimmoe_set_clock_record.restype = C.c_int
        L.trimmoe_set_clock_record.argtypes = [C.c_void_p]
        L.trimmoe_stack_forward_static.restype = C.c_int
        L.trimmoe_stack_forward_static.argtypes = [C.POINTER(Model), C.POINTER(Policy),
                                                   C.POINTER(State), C.POINTER(Trace),
                                                   C.c_void_p]
        L.trimmoe_window_stats.restype = C.c_int
        L.trimmoe_window_stats.argtypes = [C.POINTER(Model), C.POINTER(Policy),
                                           C.POINTER(State), C.POINTER(Trace), C.c_void_p,
                                           C.c_void_p]
        L.trimmoe_feedback_update.restype = C.c_int
        L.trimmoe_feedback_update.argtypes = [C.POINTER(Policy), C.POINTER(C.c_double),
                                              C.c_double, C.c_double, C.c_double]
        i32, f32, p = C.c_int32, C.c_float, C.c_void_p
        L.trimmoe_calib_exit_layers.restype = C.c_int
        L.trimmoe_calib_exit_layers.argtypes = [i32, i32, p, f32, p]
        L.trimmoe_calib_stats.restype = C.c_int
        L.trimmoe_calib_stats.argtypes = [i32, i32, i32, i32, p, p, p, p, p, p, p, p]
        L.trimmoe_calib_transitions.restype = C.c_int
        L.trimmoe_calib_transitions.argtypes = [i32, i32, i32, i32, p, p, i32, p, p]
        L.trimmoe_place_replicas.restype = C.c_int
        L.trimmoe_place_replicas.argtypes = [i32, i32, i32, p, p, p, p, p, p, p, p,
                                             C.POINTER(C.c_int32)]
        L.trimmoe_head_argmax_workspace_size.restype = C.c_int
        L.trimmoe_head_argmax_workspace_size.argtypes = [i32, i32, i32, C.POINTER(C.c_size_t)]
        L.trimmoe_head_argmax.restype = C.c_int
        L.trimmoe_head_argmax.argtypes = [i32, i32, i32, i32, p, p, p, p, p, C.c_size_t, p]
        L.trimmoe_consistency_labels.restype = C.c_int
        L.trimmoe_consistency_labels.argtypes = [i32, p, p, p, p]
        L.trimmoe_train_exit_head_workspace_size.restype = C.c_int
        L.trimmoe_train_exit_head_workspace_size.argtypes = [i32, C.POINTER(C.c_size_t)]
        L.trimmoe_train_exit_head.restype = C.c_int
        L.trimmoe_train_exit_head.argtypes = [i32, i32, i32, p, p, i32, f32, p, p, p, p,
                                              C.c_size_t, p]
        size, out = C.c_size_t, C.POINTER(C.c_size_t)
        for name in ("trimmoe_head_cross_entropy", "trimmoe_head_cross_entropy_backward"):
            getattr(L, name + "_workspace_size").restype = C.c_int
            getattr(L, name + "_workspace_size").argtypes = [i32, i32, i32, i32, out]
        L.trimmoe_head_cross_entropy.restype = C.c_int
        L.trimmoe_head_cross_entropy.argtypes = [i32] * 4 + [p] * 7 + [size, p]
        L.trimmoe_head_cross_entropy_backward.restype = C.c_int
        L.trimmoe_head_cross_entropy_backward.argtypes = [i32] * 4 + [p] * 10 + [size, p]
        for name in ("trimmoe_balance_loss", "trimmoe_balance_loss_backward"):
            getattr(L, name + "_workspace_size").restype = C.c_int
            getattr(L, name + "_workspace_size").argtypes = [i32, i32, i32, i32, i32, out]
        L.trimmoe_balance_loss.restype = C.c_int
        L.trimmoe_balance_loss.argtypes = [i32] * 5 + [p] * 9 + [size, p]
        L.trimmoe_balance_loss_backward.restype = C.c_int
        L.trimmoe_balance_loss_backward.argtypes = [i32] * 5 + [p] * 10 + [size, p]
        for name in ("trimmoe_checkpoint_pack", "trimmoe_checkpoint_unpack"):
            getattr(L, name).restype = C.c_int
            getattr(L, name).argtypes = [i32] * 3 + [p] * 4
        for name in ("trimmoe_expert_ffn", "trimmoe_expert_ffn_backward"):
            getattr(L, name + "_workspace_size").restype = C.c_int
            getattr(L, name + "_workspace_size").argtypes = [i32] * 7 + [out]
        L.trimmoe_expert_ffn.restype = C.c_int
        L.trimmoe_expert_ffn.argtypes = [i32] * 7 + [p] * 11 + [size, p]
        L.trimmoe_expert_ffn_backward.restype = C.c_int
        L.trimmoe_expert_ffn_backward.argtypes = [i32] * 8 + [p] * 16 + [size, p]
        if L.trimmoe_abi_version() != ABI_VERSION:
            raise RuntimeError(f"{LIB_PATH} has ABI version {L.trimmoe_abi_version()}, the "
                               f"binding expects {ABI_VERSION}: rebuild it")
        _lib = L
    return _lib


class TrimmoeError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} returned {status} ({STATUS.get(status, '?')})")
        self.status = status


def _check(fn: str, rc: int):
    if rc != TRIMMOE_OK:
        raise TrimmoeError(fn, rc)


def _check_sizes(fn: str, dims):
    """The library takes sizes of 32 bits (ctypes would pass the lower ones of more)."""
    if max(dims) > 2 ** 31 - 1:
        raise TrimmoeError(fn, TRIMMOE_ERR_SHAPE)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


# handle of a device's current stream without a Stream object for it (2.9 us of a small
# call's 20), where this torch has it: the name is not among torch's documented ones
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(stream):
    if stream is None:
        if _raw_stream is not None:
            return C.c_void_p(_raw_stream(torch.cuda.current_device()))
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


# ------------------------------------------------------------- wrappers ----
def trimmoe_abi_version() -> int:
    return lib().trimmoe_abi_version()


def trimmoe_status_str(status: int) -> str:
    return lib().trimmoe_status_str(status).decode()


def trimmoe_workspace_size(model: Model, max_tokens: int) -> int:
    out = C.c_size_t(0)
    _check("trimmoe_workspace_size",
           lib().trimmoe_workspace_size(C.byref(model), max_tokens, C.byref(out)))
    return out.value


def trimmoe_state_reset(model: Model, state: State, stream=None):
    _check("trimmoe_state_reset",
           lib().trimmoe_state_reset(C.byref(model), C.byref(state), _stream_handle(stream)))


def trimmoe_layer_step(model: Model, layer: int, policy: Policy, state: State, trace,
                       workspace: torch.Tensor, stream=None):
    tr = C.byref(trace) if trace is not None else None
    _check("trimmoe_layer_step",
           lib().trimmoe_layer_step(C.byref(model), layer, C.byref(policy), C.byref(state), tr,
                                    _ptr(workspace), workspace.numel(), _stream_handle(stream)))


def trimmoe_stack_forward(model: Model, policy: Policy, state: State, trace,
                          workspace: torch.Tensor, stream=None):
    tr = C.byref(trace) if trace is not None else None
    _check("trimmoe_stack_forward",
           lib().trimmoe_stack_forward(C.byref(model), C.byref(policy), C.byref(state), tr,
                                       _ptr(workspace), workspace.numel(),
                                       _stream_handle(stream)))


def trimmoe_stack_forward_static(model: Model, policy: Policy, state: State, trace,
                                 stream=None):
    """trimmoe_stack_forward on the library's per-device scratch array: no
    workspace argument, nothing allocated."""
    tr = C.byref(trace) if trace is not None else None
    _check("trimmoe_stack_forward_static",
           lib().trimmoe_stack_forward_static(C.byref(model), C.byref(policy), C.byref(state),
                                              tr, _stream_handle(stream)))


def trimmoe_stack_forward_timed(model: Model, policy: Policy, state: State, trace,
                                workspace: torch.Tensor, events, stream=None):
    """``events``: list of N * (len(TIMED_CLASSES) + 1) torch.cuda.Event(enable_timing=True)
    already recorded once (so that their HIP events exist)."""
    arr = (C.c_void_p * len(events))(*[e.cuda_event for e in events])
    tr = C.byref(trace) if trace is not None else None
    _check("trimmoe_stack_forward_timed",
           lib().trimmoe_stack_forward_timed(C.byref(model), C.byref(policy), C.byref(state), tr,
                                             _ptr(workspace), workspace.numel(),
                                             _stream_handle(stream), arr, len(events)))


def trimmoe_set_clock_record(rec):
    """``rec``: an int64 device tensor of 2 * len(TIMED_CLASSES) zeros, or None
    to stop recording (the caller keeps the tensor alive while it is set)."""
    if rec is not None:
        assert rec.is_cuda and rec.dtype == torch.int64 and rec.is_contiguous()
        assert rec.numel() == 2 * len(TIMED_CLASSES)
    _check("trimmoe_set_clock_record", lib().trimmoe_set_clock_record(_ptr(rec)))


def clock_mhz(rec) -> dict:
    """Mean engine clock (MHz) per GEMM class from a filled record."""
    r = rec.cpu().tolist()
    return {c: 100.0 * r[2 * i] / r[2 * i + 1]
            for i, c in enumerate(TIMED_CLASSES) if r[2 * i + 1] > 0}


def trimmoe_window_stats(model: Model, policy: Policy, state: State, trace,
                         stats: torch.Tensor, stream=None):
    """Add one stack pass's observations to ``stats`` (float64 [6] on the GPU)."""
    assert stats.dtype == torch.float64 and stats.numel() == 6 and stats.is_contiguous()
    tr = C.byref(trace) if trace is not None else None
    _check("trimmoe_window_stats",
           lib().trimmoe_window_stats(C.byref(model), C.byref(policy), C.byref(state), tr,
                                      _ptr(stats), _stream_handle(stream)))


def trimmoe_feedback_update(policy: Policy, stats, eta: float, kappa: float, p_floor: float):
    """Update policy.p_exit and policy.omega_t in place from a window's stats
    (six numbers on the host)."""
    arr = (C.c_double * 6)(*[float(v) for v in stats])
    _check("trimmoe_feedback_update",
           lib().trimmoe_feedback_update(C.byref(policy), arr, eta, kappa, p_floor))


# ------------------------------------- offline statistics and placement ----
def _host(a, dtype):
    """A C-contiguous numpy copy (or view) of a host array in `dtype`."""
    if isinstance(a, torch.Tensor):
        a = a.detach().cpu().numpy()
    return np.ascontiguousarray(np.asarray(a, dtype=dtype))


def _np_ptr(a: np.ndarray):
    return C.c_void_p(a.ctypes.data)


def trimmoe_calib_exit_layers(xi, p_exit: float) -> np.ndarray:
    """Exit layer of every calibration token from per-layer confidences [N, Q]."""
    xi = _host(xi, np.float32)
    N, Q = xi.shape
    out = np.zeros(Q, dtype=np.int32)
    _check("trimmoe_calib_exit_layers",
           lib().trimmoe_calib_exit_layers(N, Q, _np_ptr(xi), float(p_exit), _np_ptr(out)))
    return out


def trimmoe_calib_stats(target, importance, exit_layer, theta, n_experts: int):
    """(pi [N], act [N, E], sigma [N, E], lambda [N, E]) of a calibration record."""
    target = _host(target, np.int16)
    importance = _host(importance, np.float32)
    exit_layer = _host(exit_layer, np.int32)
    theta = _host(theta, np.float32)
    N, Q, k = target.shape
    E = int(n_experts)
    pi = np.zeros(N)
    act, sigma, lam = np.zeros((N, E)), np.zeros((N, E)), np.zeros((N, E))
    _check("trimmoe_calib_stats",
           lib().trimmoe_calib_stats(N, Q, E, k, _np_ptr(target), _np_ptr(importance),
                                     _np_ptr(exit_layer), _np_ptr(theta), _np_ptr(pi),
                                     _np_ptr(act), _np_ptr(sigma), _np_ptr(lam)))
    return pi, act, sigma, lam


def trimmoe_calib_transitions(target, exit_layer, n_experts: int, trans_b: int):
    """Transition rows (to int16 [N-1, E, B], p float32 [N-1, E, B])."""
    target = _host(target, np.int16)
    exit_layer = _host(exit_layer, np.int32)
    N, Q, k = target.shape
    E, B = int(n_experts), int(trans_b)
    to = np.zeros((max(N - 1, 0), E, B), dtype=np.int16)
    pr = np.zeros((max(N - 1, 0), E, B), dtype=np.float32)
    _check("trimmoe_calib_transitions",
           lib().trimmoe_calib_transitions(N, Q, E, k, _np_ptr(target), _np_ptr(exit_layer), B,
                                           _np_ptr(to), _np_ptr(pr)))
    return to, pr


def trimmoe_place_replicas(lam, rho, z, nbytes, capacity, bandwidth, latency, x0):
    """Greedy replication from a baseline x0 [M, N, E]; returns (x, n_placed)."""
    x = _host(x0, np.uint8).copy()
    M, N, E = x.shape
    args = [_host(v, np.float64) for v in (lam, rho, z, nbytes, capacity, bandwidth, latency)]
    n = C.c_int32(0)
    _check("trimmoe_place_replicas",
           lib().trimmoe_place_replicas(M, N, E, *[_np_ptr(v) for v in args], _np_ptr(x),
                                        C.byref(n)))
    return x, int(n.value)


# ------------------------------------------------- exit-head training ------
def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"hidden states must be bf16 or fp32, not {t.dtype}")


def _aligned_ws(nbytes: int, device) -> torch.Tensor:
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + nbytes]


def trimmoe_head_argmax(w_head: torch.Tensor, h: torch.Tensor, b_head=None,
                        stream=None) -> torch.Tensor:
    """argmax over the rows of an output head [V, d] for each row of h [Q, d]
    (both on one GPU, same dtype); returns int32 [Q] on the GPU."""
    assert w_head.dtype == h.dtype and w_head.is_contiguous() and h.is_contiguous()
    V, d = w_head.shape
    Q = h.shape[0]
    dt = _dtype_code(h)
    n = C.c_size_t(0)
    _check("trimmoe_head_argmax_workspace_size",
           lib().trimmoe_head_argmax_workspace_size(dt, V, Q, C.byref(n)))
    ws = _aligned_ws(n.value, h.device)
    out = torch.empty(Q, dtype=torch.int32, device=h.device)
    _check("trimmoe_head_argmax",
           lib().trimmoe_head_argmax(dt, V, d, Q, _ptr(w_head), _ptr(b_head), _ptr(h), _ptr(out),
                                     _ptr(ws), ws.numel(), _stream_handle(stream)))
    return out


def trimmoe_consistency_labels(pred: torch.Tensor, ref: torch.Tensor, stream=None):
    """Eq. (22) on the GPU: uint8 [Q], 1 where pred == ref (int32 [Q] each)."""
    assert pred.dtype == torch.int32 and ref.dtype == torch.int32 and pred.shape == ref.shape
    out = torch.empty(pred.shape[0], dtype=torch.uint8, device=pred.device)
    _check("trimmoe_consistency_labels",
           lib().trimmoe_consistency_labels(pred.shape[0], _ptr(pred), _ptr(ref), _ptr(out),
                                            _stream_handle(stream)))
    return out


def trimmoe_train_exit_head(h: torch.Tensor, labels: torch.Tensor, epochs: int, lr: float,
                            w: torch.Tensor, c: torch.Tensor, loss=None, stream=None):
    """Gradient descent of the sigmoid exit head on BCE; w (fp32 [d]) and c
    (fp32 [1]) are updated in place; loss (fp32 [epochs]) if given."""
    assert w.dtype == torch.float32 and c.dtype == torch.float32 and labels.dtype == torch.uint8
    Q, d = h.shape
    n = C.c_size_t(0)
    _check("trimmoe_train_exit_head_workspace_size",
           lib().trimmoe_train_exit_head_workspace_size(Q, C.byref(n)))
    ws = _aligned_ws(n.value, h.device)
    _check("trimmoe_train_exit_head",
           lib().trimmoe_train_exit_head(_dtype_code(h), d, Q, _ptr(h), _ptr(labels), int(epochs),
                                         float(lr), _ptr(w), _ptr(c), _ptr(loss), _ptr(ws),
                                         ws.numel(), _stream_handle(stream)))


# ------------------------------------------------------- training losses ---
class _NoContext:
    def __enter__(self):
        return None

    def __exit__(self, *exc):
        return False


_NO_CONTEXT = _NoContext()


def _on_stream(t: torch.Tensor, stream):
    """Context in which outputs and workspaces belong to the stream that the
    call runs on (`stream`, or the current one of t's device)."""
    if not t.is_cuda:
        raise ValueError(f"tensors on the GPU are needed, not on {t.device}")
    if stream is not None:
        if stream.device != t.device:
            raise ValueError(f"a stream of {stream.device} for tensors on {t.device}")
        return torch.cuda.stream(stream)
    if t.device.index == torch.cuda.current_device():
        return _NO_CONTEXT
    return torch.cuda.device(t.device)


def _take(name: str, t: torch.Tensor, shape, dtype, device):
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on {device} "
                         f"is needed, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _rows_and_weights(w: torch.Tensor, h: torch.Tensor):
    code = _dtype_code(h)
    if w.dim() != 2 or h.dim() != 2:
        raise ValueError("the weights are [V, d] (or [E, d]) and the rows [n, d]")
    (n, d), v = h.shape, w.shape[0]
    _take("weights", w, (v, d), h.dtype, h.device)
    if not h.is_contiguous():
        raise ValueError("rows: a contiguous tensor is needed")
    return code, v, d, n


@functools.lru_cache(maxsize=1024)
def _loss_ws_bytes(name: str, dims) -> int:
    _check_sizes(name, dims)
    n = C.c_size_t(0)
    _check(name + "_workspace_size", getattr(lib(), name + "_workspace_size")(*dims, C.byref(n)))
    return max(n.value, 256)


def _loss_ws(name: str, dims, device) -> torch.Tensor:
    n = _loss_ws_bytes(name, dims)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    # (torch's allocator aligns its blocks further than the library asks)
    return ws if ws.data_ptr() % 256 == 0 else _aligned_ws(n, device)


def trimmoe_head_cross_entropy(w_head: torch.Tensor, h: torch.Tensor, target: torch.Tensor,
                               b_head=None, stream=None):
    """(loss fp32 [Q], lse fp32 [Q]) of the head w_head [V, d] (bias fp32 [V])
    on rows h [Q, d] against target int32 [Q]; a target outside [0, V) is
    ignored (loss 0)."""
    dt, V, d, Q = _rows_and_weights(w_head, h)
    dev = h.device
    _take("target", target, (Q,), torch.int32, dev)
    if b_head is not None:
        _take("b_head", b_head, (V,), torch.float32, dev)
    with _on_stream(h, stream):
        loss = torch.empty(Q, dtype=torch.float32, device=dev)
        lse = torch.empty(Q, dtype=torch.float32, device=dev)
        ws = _loss_ws("trimmoe_head_cross_entropy", (dt, V, d, Q), dev)
        _check("trimmoe_head_cross_entropy",
               lib().trimmoe_head_cross_entropy(dt, V, d, Q, _ptr(w_head), _ptr(b_head), _ptr(h),
                                                _ptr(target), _ptr(loss), _ptr(lse), _ptr(ws),
                                                ws.numel(), _stream_handle(None)))
    return loss, lse


def trimmoe_head_cross_entropy_backward(w_head: torch.Tensor, h: torch.Tensor,
                                        target: torch.Tensor, lse: torch.Tensor,
                                        dloss: torch.Tensor, b_head=None, want_dh=True,
                                        want_dw=True, stream=None):
    """Gradients (dh [Q, d], dw [V, d], db fp32 [V]) of sum(dloss * loss), dloss
    fp32 [Q], lse from trimmoe_head_cross_entropy; None for one that is not
    wanted (db: without a bias)."""
    dt, V, d, Q = _rows_and_weights(w_head, h)
    dev = h.device
    _take("target", target, (Q,), torch.int32, dev)
    _take("lse", lse, (Q,), torch.float32, dev)
    _take("dloss", dloss, (Q,), torch.float32, dev)
    if b_head is not None:
        _take("b_head", b_head, (V,), torch.float32, dev)
    with _on_stream(h, stream):
        dh = torch.empty_like(h) if want_dh else None
        dw = torch.empty_like(w_head) if want_dw else None
        db = None if b_head is None else torch.empty_like(b_head)
        ws = _loss_ws("trimmoe_head_cross_entropy_backward", (dt, V, d, Q), dev)
        _check("trimmoe_head_cross_entropy_backward",
               lib().trimmoe_head_cross_entropy_backward(
                   dt, V, d, Q, _ptr(w_head), _ptr(b_head), _ptr(h), _ptr(target), _ptr(lse),
                   _ptr(dloss), _ptr(dh), _ptr(dw), _ptr(db), _ptr(ws), ws.numel(),
                   _stream_handle(None)))
    return dh, dw, db


def trimmoe_balance_loss(w_router: torch.Tensor, h: torch.Tensor, target: torch.Tensor,
                         b_router=None, stream=None):
    """(loss fp32 [1], counts int32 [E + 1], prob_sum fp32 [E], prob fp32
    [Q, E]) of the router w_router [E, d] (bias fp32 [E]) on rows h [Q, d] with
    the routed experts target int16 [Q, k] (-1: none); counts[E] is the number
    of rows with a routed slot."""
    dt, E, d, Q = _rows_and_weights(w_router, h)
    dev = h.device
    k = target.shape[1] if target.dim() == 2 else 0
    _take("target", target, (Q, k), torch.int16, dev)
    if b_router is not None:
        _take("b_router", b_router, (E,), torch.float32, dev)
    with _on_stream(h, stream):
        f = dict(dtype=torch.float32, device=dev)
        loss, prob_sum = torch.empty(1, **f), torch.empty(E, **f)
        prob = torch.empty(Q, E, **f)
        counts = torch.empty(E + 1, dtype=torch.int32, device=dev)
        ws = _loss_ws("trimmoe_balance_loss", (dt, E, k, d, Q), dev)
        _check("trimmoe_balance_loss",
               lib().trimmoe_balance_loss(dt, E, k, d, Q, _ptr(w_router), _ptr(b_router), _ptr(h),
                                          _ptr(target), _ptr(loss), _ptr(counts), _ptr(prob_sum),
                                          _ptr(prob), _ptr(ws), ws.numel(), _stream_handle(None)))
    return loss, counts, prob_sum, prob


def trimmoe_balance_loss_backward(w_router: torch.Tensor, h: torch.Tensor, target: torch.Tensor,
                                  prob: torch.Tensor, counts: torch.Tensor, dloss: torch.Tensor,
                                  want_dh=True, want_dw=True, want_db=True, stream=None):
    """Gradients (dh [Q, d], dw [E, d], db fp32 [E]) of dloss * loss (dloss fp32
    [1]) with prob and counts from trimmoe_balance_loss (counts may be summed
    over ranks); None for one that is not wanted."""
    dt, E, d, Q = _rows_and_weights(w_router, h)
    dev = h.device
    k = target.shape[1] if target.dim() == 2 else 0
    _take("target", target, (Q, k), torch.int16, dev)
    _take("prob", prob, (Q, E), torch.float32, dev)
    _take("counts", counts, (E + 1,), torch.int32, dev)
    _take("dloss", dloss, (1,), torch.float32, dev)
    with _on_stream(h, stream):
        dh = torch.empty_like(h) if want_dh else None
        dw = torch.empty_like(w_router) if want_dw else None
        db = torch.empty(E, dtype=torch.float32, device=dev) if want_db else None
        ws = _loss_ws("trimmoe_balance_loss_backward", (dt, E, k, d, Q), dev)
        _check("trimmoe_balance_loss_backward",
               lib().trimmoe_balance_loss_backward(
                   dt, E, k, d, Q, _ptr(w_router), _ptr(h), _ptr(target), _ptr(prob), _ptr(counts),
                   _ptr(dloss), _ptr(dh), _ptr(dw), _ptr(db), _ptr(ws), ws.numel(),
                   _stream_handle(None)))
    return dh, dw, db


# ------------------------------------------------ activations in 8 bits ----
class Packed(NamedTuple):
    """Rows in 8 bits: codes int8 [n, c] and scale bytes uint8 [n, ceil(c / 32)],
    32 consecutive values of a row in steps of 2^(scale - 133)."""
    codes: torch.Tensor
    scale: torch.Tensor


PACK_BLOCK = 32  # values of a row that share a scale byte


def _packed_like(n: int, c: int, device) -> Packed:
    return Packed(torch.empty(n, c, dtype=torch.int8, device=device),
                  torch.empty(n, -(-c // PACK_BLOCK), dtype=torch.uint8, device=device))


def _take_packed(name: str, x, n: int, c: int, device):
    if not isinstance(x, (tuple, list)) or len(x) != 2:
        raise ValueError(f"{name}: (codes, scale) as trimmoe_checkpoint_pack gives them is needed")
    _take(name + " codes", x[0], (n, c), torch.int8, device)
    _take(name + " scale", x[1], (n, -(-c // PACK_BLOCK)), torch.uint8, device)


def trimmoe_checkpoint_pack(x: torch.Tensor, stream=None) -> Packed:
    """x [n, c] (bf16 or fp32, on the GPU) in 8 bits a value and a byte a block of
    32: off by at most 1 / 127 of the block's largest magnitude; a block that
    holds a NaN or an infinity comes back as NaN."""
    code = _dtype_code(x)
    if x.dim() != 2 or x.shape[1] < 1 or not x.is_contiguous():
        raise ValueError("a contiguous tensor [n, c] is needed")
    n, c = x.shape
    _check_sizes("trimmoe_checkpoint_pack", (n, c))
    with _on_stream(x, stream):
        out = _packed_like(n, c, x.device)
        _check("trimmoe_checkpoint_pack",
               lib().trimmoe_checkpoint_pack(code, n, c, _ptr(x), _ptr(out.codes),
                                             _ptr(out.scale), _stream_handle(None)))
    return out


def trimmoe_checkpoint_unpack(codes: torch.Tensor, scale: torch.Tensor,
                              dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """The values that codes and scale (of trimmoe_checkpoint_pack) stand for, in
    bf16 or fp32 (exact in both)."""
    if codes.dim() != 2 or codes.shape[1] < 1:
        raise ValueError("codes are [n, c]")
    n, c = codes.shape
    _check_sizes("trimmoe_checkpoint_unpack", (n, c))
    _take_packed("checkpoint", (codes, scale), n, c, codes.device)
    with _on_stream(codes, stream):
        x = torch.empty(n, c, dtype=dtype, device=codes.device)
        _check("trimmoe_checkpoint_unpack",
               lib().trimmoe_checkpoint_unpack(_dtype_code(x), n, c, _ptr(codes), _ptr(scale),
                                               _ptr(x), _stream_handle(None)))
    return x


# ---------------------------------------------- expert feed-forward block --
KEEP = {None: 0, "full": 1, "packed": 2}


def _ffn_args(w_up, w_gate, w_down, rows, offsets):
    """(dtype code, act, E, d, F, n) of the block's weights [E, F, d], [E, d, F]
    (or [F, d], [d, F]: one expert) and rows [n, d] in the weights' dtype."""
    code = _dtype_code(w_up)
    one = w_up.dim() == 2
    if w_up.dim() not in (2, 3) or rows.dim() != 2:
        raise ValueError("the weights are [E, F, d] and [E, d, F] (or of one expert), the rows [n, d]")
    E = 1 if one else w_up.shape[0]
    F, d = w_up.shape[-2:]
    dev = w_up.device
    _take("w_up", w_up, (F, d) if one else (E, F, d), w_up.dtype, dev)
    _take("w_down", w_down, (d, F) if one else (E, d, F), w_up.dtype, dev)
    if w_gate is not None:
        _take("w_gate", w_gate, tuple(w_up.shape), w_up.dtype, dev)
    if offsets is not None:
        _take("offsets", offsets, (E + 1,), torch.int32, dev)
    elif E != 1:
        raise ValueError("offsets: rows of several experts need their borders")
    return code, ACT_RELU if w_gate is None else ACT_SWIGLU, E, d, F, rows.shape[0]


def trimmoe_expert_ffn(w_up: torch.Tensor, w_gate, w_down: torch.Tensor, x: torch.Tensor,
                       offsets=None, keep=None, stream=None):
    """(y [n, d], kept) of the feed-forward block y = w_down (silu(w_gate x) *
    (w_up x)), or w_down relu(w_up x) without w_gate, on rows x [n, d] sorted by
    expert: expert e's are offsets[e] .. offsets[e + 1] - 1 (int32 [E + 1] on the
    GPU; None: one expert's).  Weights [E, F, d], [E, F, d], [E, d, F], or [F, d],
    [F, d], [d, F] of one expert.  Rows of no expert give zeros.  keep: what the
    gradient needs of w_up x and w_gate x: "full" (in x's dtype), "packed" (8
    bits) or None; kept is then (up, gate) as tensors or Packed, gate None
    without w_gate, or None."""
    if keep not in KEEP:
        raise ValueError(f"keep is one of {list(KEEP)}")
    if not isinstance(x, torch.Tensor):
        raise ValueError("x: a tensor [n, d] is needed (the gradient alone takes Packed rows)")
    dims = _ffn_args(w_up, w_gate, w_down, x, offsets)
    code, act, E, d, F, n = dims
    dev = w_up.device
    _take("x", x, (n, d), w_up.dtype, dev)
    with _on_stream(x, stream):
        y = torch.empty_like(x)
        kept = [None, None]
        if keep is not None:
            for i in range(1 if w_gate is None else 2):
                kept[i] = (_packed_like(n, F, dev) if keep == "packed"
                           else torch.empty(n, F, dtype=x.dtype, device=dev))
        flat = [t for k in kept for t in _codes_and_scale(k)]
        dims = dims + (KEEP[keep],)
        ws = _loss_ws("trimmoe_expert_ffn", dims, dev)
        _check("trimmoe_expert_ffn",
               lib().trimmoe_expert_ffn(*dims, _ptr(w_up), _ptr(w_gate), _ptr(w_down), _ptr(x),
                                        _ptr(offsets), _ptr(y), *map(_ptr, flat), _ptr(ws),
                                        ws.numel(), _stream_handle(None)))
    return y, None if keep is None else tuple(kept)


def _codes_and_scale(k):
    """(values or codes, scale or None) of a kept array."""
    return tuple(k) if isinstance(k, (tuple, list)) else (k, None)


def trimmoe_expert_ffn_backward(w_up: torch.Tensor, w_gate, w_down: torch.Tensor, x,
                                dy: torch.Tensor, kept, offsets=None, want_dx=True, want_dw=True,
                                stream=None):
    """Gradients (dx [n, d], dw_up, dw_gate, dw_down, in the weights' shapes and
    dtype) of sum(dy * y) with kept from trimmoe_expert_ffn (tensors or Packed, both
    alike); x: the rows, or their Packed form.  None for one that is not wanted
    (dw_gate: without w_gate)."""
    if not isinstance(dy, torch.Tensor):
        raise ValueError("dy: a tensor [n, d] is needed")
    code, act, E, d, F, n = _ffn_args(w_up, w_gate, w_down, dy, offsets)
    dev = w_up.device
    _take("dy", dy, (n, d), w_up.dtype, dev)
    x_packed = not isinstance(x, torch.Tensor)
    if x_packed:
        _take_packed("x", x, n, d, dev)
    else:
        _take("x", x, (n, d), w_up.dtype, dev)
    if not isinstance(kept, (tuple, list)) or len(kept) != 2 or (kept[1] is None) != (w_gate is None):
        raise ValueError("kept: (up, gate) as trimmoe_expert_ffn gives them is needed")
    packed = not isinstance(kept[0], torch.Tensor)
    for name, k in zip(("up", "gate"), kept):
        if k is None:
            continue
        if packed != (not isinstance(k, torch.Tensor)):
            raise ValueError("up and gate are kept in one form")
        if packed:
            _take_packed(name, k, n, F, dev)
        else:
            _take(name, k, (n, F), w_up.dtype, dev)
    up, up_scale = _codes_and_scale(kept[0])
    gate, gate_scale = _codes_and_scale(kept[1])
    x, x_scale = _codes_and_scale(x)
    with _on_stream(dy, stream):
        dx = torch.empty_like(dy) if want_dx else None
        dw = [None if w is None or not want_dw else torch.empty_like(w)
              for w in (w_up, w_gate, w_down)]
        ws = _loss_ws("trimmoe_expert_ffn_backward", (code, act, E, d, F, n, int(x_packed)), dev)
        _check("trimmoe_expert_ffn_backward",
               lib().trimmoe_expert_ffn_backward(
                   code, act, E, d, F, n, KEEP["packed" if packed else "full"], int(x_packed),
                   *map(_ptr, (w_up, w_gate, w_down, x, x_scale, dy, offsets, up, up_scale, gate,
                               gate_scale, dx, *dw, ws)), ws.numel(), _stream_handle(None)))
    return (dx, *dw)


# ------------------------------------------------ struct construction ------
class ModelHandle:
    """A Model struct over device tensors; keeps the tensors alive.

    ``layers`` is a list of dicts with the keys of trimmoe_layer (torch
    tensors on one GPU, or None) plus the floats ``theta`` and
    ``skip_slope``.
    """

    def __init__(self, *, n_layers, d_model, n_experts, top_k, d_ff, d_ff_shared, vocab_exit,
                 dtype, act, conf_mode, normalize_topk, layers):
        self._keep = []
        arr = (Layer * n_layers)()
        for i, L in enumerate(layers):
            for key in ("w_router", "b_router", "w_up", "w_gate", "w_down", "ws_up", "ws_gate",
                        "ws_down", "w_exit", "b_exit", "local_mask", "sim", "trans_to",
                        "trans_p"):
                t = L.get(key)
                if t is not None:
                    if not t.is_contiguous():
                        t = t.contiguous()
                    self._keep.append(t)
                setattr(arr[i], key, None if t is None else t.data_ptr())
            arr[i].theta = float(L["theta"])
            arr[i].skip_slope = float(L["skip_slope"])
        self.layers = arr
        trans_b = next((int(L["trans_to"].shape[1]) for L in layers
                        if L.get("trans_to") is not None), 0)
        self.model = Model(n_layers, d_model, n_experts, top_k, d_ff, d_ff_shared, vocab_exit,
                           dtype, act, conf_mode, normalize_topk,
                           C.cast(arr, C.POINTER(Layer)), trans_b)


def make_policy(*, p_exit, budget, omega_t, t_local, t_remote, phi_scale, sim_min,
                p_exit_tok=None, budget_tok=None, horizon=1, la_subs=4) -> Policy:
    return Policy(p_exit, budget, omega_t, t_local, t_remote, phi_scale, sim_min,
                  None if p_exit_tok is None else p_exit_tok.data_ptr(),
                  None if budget_tok is None else budget_tok.data_ptr(), int(horizon),
                  int(la_subs))


class StateBuffers:
    """Caller-owned per-token state on one GPU (h is used in place)."""

    def __init__(self, h: torch.Tensor):
        T = h.shape[0]
        dev = h.device
        self.h = h
        self.d_acc = torch.zeros(T, dtype=torch.float32, device=dev)
        self.active_idx = torch.zeros(max(T, 1), dtype=torch.int32, device=dev)
        self.n_active = torch.zeros(1, dtype=torch.int32, device=dev)
        self.exit_layer = torch.zeros(max(T, 1), dtype=torch.int32, device=dev)
        self.xi = torch.zeros(max(T, 1), dtype=torch.float32, device=dev)
        self.state = State(T, h.data_ptr(), self.d_acc.data_ptr(), self.active_idx.data_ptr(),
                           self.n_active.data_ptr(), self.exit_layer.data_ptr(),
                           self.xi.data_ptr())


class TraceBuffers:
    """Per-layer decision record on one GPU."""

    def __init__(self, n_layers: int, T: int, k: int, device):
        z = dict(device=device)
        self.action = torch.zeros(n_layers, T, dtype=torch.int8, **z)
        self.target = torch.zeros(n_layers, T, k, dtype=torch.int16, **z)
        self.exec = torch.zeros(n_layers, T, k, dtype=torch.int16, **z)
        self.kind = torch.zeros(n_layers, T, k, dtype=torch.int8, **z)
        self.gate = torch.zeros(n_layers, T, k, dtype=torch.float32, **z)
        self.importance = torch.zeros(n_layers, T, dtype=torch.float32, **z)
        self.xi = torch.zeros(n_layers, T, dtype=torch.float32, **z)
        self.d_acc = torch.zeros(n_layers, T, dtype=torch.float32, **z)
        self.counters = torch.zeros(n_layers, N_COUNTERS, dtype=torch.int32, **z)
        self.trace = Trace(*(getattr(self, n).data_ptr() for n in
                             ("action", "target", "exec", "kind", "gate", "importance", "xi",
                              "d_acc", "counters")))


class CounterTrace:
    """A trace that records only the per-layer counters (what the runtime
    feedback observations need)."""

    def __init__(self, n_layers: int, device):
        self.counters = torch.zeros(n_layers, N_COUNTERS, dtype=torch.int32, device=device)
        self.trace = Trace(None, None, None, None, None, None, None, None,
                           self.counters.data_ptr())


def alloc_workspace(model: Model, max_tokens: int, device) -> torch.Tensor:
    """A 256-byte aligned uint8 workspace of the size the library asks for."""
    n = trimmoe_workspace_size(model, max_tokens)
    ws = torch.empty(n + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + n]


def model_handle(dims: dict, layers: list) -> ModelHandle:
    """ModelHandle from a dims dict (n_layers, d_model, n_experts, top_k, d_ff,
    d_ff_shared, vocab_exit, dtype 'bf16'|'f32', act 'relu'|'swiglu',
    normalize_topk, optional conf_mode 'softmax'|'sigmoid') and per-layer
    tensor dicts keyed like trimmoe_layer."""
    return ModelHandle(
        n_layers=dims["n_layers"], d_model=dims["d_model"], n_experts=dims["n_experts"],
        top_k=dims["top_k"], d_ff=dims["d_ff"], d_ff_shared=dims["d_ff_shared"],
        vocab_exit=dims["vocab_exit"], dtype={"f32": F32, "bf16": BF16}[dims["dtype"]],
        act={"relu": ACT_RELU, "swiglu": ACT_SWIGLU}[dims["act"]],
        conf_mode={"softmax": CONF_SOFTMAX, "sigmoid": CONF_SIGMOID}[dims.get("conf_mode", "softmax")],
        normalize_topk=int(dims["normalize_topk"]), layers=layers)
