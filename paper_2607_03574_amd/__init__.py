"""Python binding of libndvm (the C ABI declared in include/ndvm.h).

Argument marshalling only: every step of the hot path (trace production,
scheduling, forward replay, reverse sweep) runs inside libndvm.so.  Torch is
used for device memory and streams.  If the library has not been built the
import fails: there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os
import sys
from typing import Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libndvm.so")

OK, E_ARG, E_BYTECODE, E_STRUCT_DIVERGE, E_TAPE, E_NOMEM, E_DEVICE, E_UNSUPPORTED, E_INTERNAL = range(9)
STATUS_NAMES = {0: "NDVM_OK", 1: "NDVM_E_ARG", 2: "NDVM_E_BYTECODE", 3: "NDVM_E_STRUCT_DIVERGE",
                4: "NDVM_E_TAPE", 5: "NDVM_E_NOMEM", 6: "NDVM_E_DEVICE", 7: "NDVM_E_UNSUPPORTED",
                8: "NDVM_E_INTERNAL"}
POLICY_SAVE = 1        # store what the reverse sweep reads, recompute nothing
POLICY_RECOMPUTE = 2   # store segment inputs, recompute inside segments
BRANCH_SKIP = 0x100    # option OR'd into the policy: waves skip branch arms none of their lanes takes
NOALLOC_SCRATCH_BYTES = 64 << 20    # NDVM_NOALLOC_SCRATCH_BYTES

# exported symbols of include/ndvm.h
EXPORTS = ["ndvm_tape_build", "ndvm_tape_upload", "ndvm_tape_upload_many", "ndvm_tape_info_get", "ndvm_workspace_bytes",
           "ndvm_forward", "ndvm_grad", "ndvm_grad_many", "ndvm_workspace_bytes_many",
           "ndvm_tape_free", "ndvm_free", "ndvm_last_error", "ndvm_adam_step", "ndvm_grad_noalloc",
           "ndvm_grad_points", "ndvm_workspace_bytes_points", "ndvm_walk_prepare", "ndvm_walk_measure", "ndvm_walk_workspace_bytes",
           "ndvm_walk_grad", "ndvm_walk_status", "ndvm_walk_free",
           "ndvm_layer_norm", "ndvm_layer_norm_workspace_bytes", "ndvm_layer_norm_grad",
           "ndvm_rms_norm", "ndvm_rms_norm_workspace_bytes", "ndvm_rms_norm_grad", "ndvm_rms_norm_8bit", "ndvm_quantize_rows",
           "ndvm_linear_attention_workspace_bytes", "ndvm_linear_attention", "ndvm_linear_attention_grad",
           "ndvm_linear_attention_step", "ndvm_delta_attention_workspace_bytes", "ndvm_delta_attention",
           "ndvm_delta_attention_grad", "ndvm_delta_attention_step", "ndvm_gated_ffn_workspace_bytes", "ndvm_gated_ffn", "ndvm_gated_ffn_grad",
           "ndvm_linear_workspace_bytes", "ndvm_linear", "ndvm_linear_grad", "ndvm_linear_8bit_workspace_bytes", "ndvm_linear_8bit"]
ACTIVATIONS = {"silu": 0, "gelu": 1, "sigmoid": 2, "relu": 3}     # NDVM_ACT_*
ACT_NONE = 4           # NDVM_ACT_NONE: no activation (linear)

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with paper_2607_03574_amd/build.py "
                      "(or __graft_entry__.build()); there is no fallback path")

_lib = ctypes.CDLL(LIB_PATH)
_vp, _i64, _sz, _int = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int


class _Info(ctypes.Structure):
    _fields_ = [("n_params", ctypes.c_uint32), ("n_obs", ctypes.c_uint32), ("n_ops", ctypes.c_uint32),
                ("n_consts", ctypes.c_uint32), ("loss_slot", ctypes.c_uint32),
                ("n_selects", ctypes.c_uint32), ("tape_bytes", ctypes.c_uint64)]


def _sig(name, res, args):
    f = getattr(_lib, name)
    f.restype = res
    f.argtypes = args
    return f


_tape_build = _sig("ndvm_tape_build", _int, [ctypes.c_char_p, _sz, ctypes.POINTER(_vp), ctypes.POINTER(_sz)])
_tape_upload = _sig("ndvm_tape_upload", _int, [ctypes.c_char_p, _sz, _int, _vp, ctypes.POINTER(_vp)])
_tape_upload_many = _sig("ndvm_tape_upload_many", _int, [ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(_sz), _int,
                                                         _int, _vp, ctypes.POINTER(_vp)])
_tape_info = _sig("ndvm_tape_info_get", _int, [_vp, ctypes.POINTER(_Info)])
_ws_bytes = _sig("ndvm_workspace_bytes", _int, [_vp, _i64, _int, ctypes.POINTER(_sz)])
_ws_bytes_many = _sig("ndvm_workspace_bytes_many", _int, [ctypes.POINTER(_vp), _int, _i64, ctypes.POINTER(_sz)])
_forward = _sig("ndvm_forward", _int, [_vp, _vp, _i64, _i64, _vp, _i64, _vp, _vp, _sz, _vp])
_grad = _sig("ndvm_grad", _int, [_vp, _vp, _i64, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _sz, _vp])
_grad_noalloc = _sig("ndvm_grad_noalloc", _int, [_vp, _vp, _i64, _i64, _vp, _i64, _vp, _vp, _i64, _vp])
_grad_points = _sig("ndvm_grad_points", _int, [_vp, _vp, _i64, _i64, _vp, _i64, _i64, ctypes.c_double, _vp, _vp,
                                                _i64, _vp, _sz, _vp])
_ws_bytes_points = _sig("ndvm_workspace_bytes_points", _int, [_vp, _i64, _i64, ctypes.POINTER(_sz)])
_grad_many = _sig("ndvm_grad_many", _int, [ctypes.POINTER(_vp), _int, _vp, _i64, _i64, _i64, _vp, _i64, _vp,
                                            _vp, _i64, _i64, _vp, _sz, _vp])
_walk_prepare = _sig("ndvm_walk_prepare", _int, [ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(_sz), _int, _vp,
                                                  ctypes.POINTER(_vp)])
_walk_ws_bytes = _sig("ndvm_walk_workspace_bytes", _int, [_vp, _i64, ctypes.POINTER(_sz)])
_walk_grad = _sig("ndvm_walk_grad", _int, [_vp, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _vp, _i64, _i64, _vp, _sz,
                                            _vp])
_walk_status = _sig("ndvm_walk_status", _int, [_vp, _vp])
_walk_free = _sig("ndvm_walk_free", None, [_vp])


class _WalkInfo(ctypes.Structure):
    _fields_ = [("n_params", ctypes.c_uint32), ("n_obs", ctypes.c_uint32), ("n_nodes", ctypes.c_uint64),
                ("depth", ctypes.c_uint32), ("n_locals", ctypes.c_uint32), ("n_frames", ctypes.c_uint32),
                ("n_loops", ctypes.c_uint32)]


_walk_measure = _sig("ndvm_walk_measure", _int, [ctypes.c_char_p, _sz, ctypes.POINTER(_WalkInfo)])
_tape_free = _sig("ndvm_tape_free", None, [_vp])
_free = _sig("ndvm_free", None, [_vp])
_last_error = _sig("ndvm_last_error", ctypes.c_char_p, [])
_f64 = ctypes.c_double
_adam = _sig("ndvm_adam_step", _int, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64, _f64, _f64, _f64, _f64,
                                      _vp])


class _AttentionShape(ctypes.Structure):
    _fields_ = [("dtype", _int), ("n_seq", _i64), ("n_tokens", _i64), ("heads", _i64), ("kv_heads", _i64),
                ("dk", _i64), ("dv", _i64), ("scale", _f64)]


class _Heads(ctypes.Structure):
    _fields_ = [("data", _vp), ("seq_stride", _i64), ("tok_stride", _i64), ("head_stride", _i64)]


_shape_p, _heads_p = ctypes.POINTER(_AttentionShape), ctypes.POINTER(_Heads)
_norm = _sig("ndvm_layer_norm", _int, [_int, _vp, _i64, _i64, _i64, _vp, _vp, _f64, _vp, _i64, _vp, _vp, _vp])
_norm_ws = _sig("ndvm_layer_norm_workspace_bytes", _int, [_i64, _i64, ctypes.POINTER(_sz)])
_norm_grad = _sig("ndvm_layer_norm_grad", _int, [_int, _vp, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _vp,
                                                 _vp, _vp, _sz, _vp])
_rms = _sig("ndvm_rms_norm", _int, [_int, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _f64, _vp, _i64, _vp, _i64, _vp, _vp])
_rms_ws = _sig("ndvm_rms_norm_workspace_bytes", _int, [_i64, _i64, ctypes.POINTER(_sz)])
_rms_grad = _sig("ndvm_rms_norm_grad", _int, [_int, _vp, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _vp,
                                              _sz, _vp])
_rms_8bit = _sig("ndvm_rms_norm_8bit", _int, [_int, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _f64, _vp, _i64, _vp, _vp, _i64, _vp])
_quantize = _sig("ndvm_quantize_rows", _int, [_int, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _vp])
_attn_ws = _sig("ndvm_linear_attention_workspace_bytes", _int, [_shape_p, _int, _int, ctypes.POINTER(_sz)])
_attn = _sig("ndvm_linear_attention", _int, [_shape_p, _heads_p, _heads_p, _heads_p, _vp, _vp, _vp, _heads_p, _vp, _vp,
                                             _sz, _vp])
_attn_grad = _sig("ndvm_linear_attention_grad", _int, [_shape_p, _heads_p, _heads_p, _heads_p, _vp, _vp, _vp, _heads_p,
                                                       _vp, _heads_p, _heads_p, _heads_p, _vp, _vp, _sz, _vp])
_attn_step = _sig("ndvm_linear_attention_step", _int, [_shape_p, _heads_p, _heads_p, _heads_p, _vp, _vp, _i64, _vp,
                                                       _heads_p, _vp])


class _DeltaShape(ctypes.Structure):
    _fields_ = [("dtype", _int), ("n_seq", _i64), ("n_tokens", _i64), ("heads", _i64), ("qk_heads", _i64),
                ("dk", _i64), ("dv", _i64), ("scale", _f64)]


_delta_p = ctypes.POINTER(_DeltaShape)
_delta_ws = _sig("ndvm_delta_attention_workspace_bytes", _int, [_delta_p, _int, _int, ctypes.POINTER(_sz)])
_delta = _sig("ndvm_delta_attention", _int, [_delta_p] + [_heads_p] * 5 + [_vp, _vp, _heads_p, _vp, _vp, _sz, _vp])
_delta_grad = _sig("ndvm_delta_attention_grad", _int, [_delta_p] + [_heads_p] * 5 + [_vp, _vp, _heads_p, _vp] + [_heads_p] * 5
                   + [_vp, _vp, _sz, _vp])
_delta_step = _sig("ndvm_delta_attention_step", _int, [_delta_p] + [_heads_p] * 5 + [_vp, _i64, _vp, _heads_p, _vp])
_ffn_ws = _sig("ndvm_gated_ffn_workspace_bytes", _int, [_int, _i64, _i64, _i64, _int, ctypes.POINTER(_sz)])
_ffn = _sig("ndvm_gated_ffn", _int, [_int, _int, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _i64, _i64, _vp, _i64, _vp, _sz,
                                     _vp])
_ffn_grad = _sig("ndvm_gated_ffn_grad", _int, [_int, _int, _vp, _i64, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _i64, _i64,
                                               _vp, _i64, _vp, _i64, _vp, _i64, _vp, _sz, _vp])

_linear_ws = _sig("ndvm_linear_workspace_bytes", _int, [_int, _int, _i64, _i64, _i64, _int, ctypes.POINTER(_sz)])
_linear = _sig("ndvm_linear", _int, [_int, _int, _vp, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _sz, _vp])
_linear_grad = _sig("ndvm_linear_grad", _int, [_int, _int, _vp, _i64, _vp, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _vp,
                                               _i64, _vp, _vp, _sz, _vp])
_linear8_ws = _sig("ndvm_linear_8bit_workspace_bytes", _int, [_i64, _i64, _i64, ctypes.POINTER(_sz)])
_linear8 = _sig("ndvm_linear_8bit", _int, [_int, _int, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _i64, _vp,
                                           _i64, _vp, _sz, _vp])


class NdvmError(RuntimeError):
    def __init__(self, status: int, where: str):
        msg = (_last_error() or b"").decode(errors="replace")
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


def _check(st: int, where: str):
    if st != OK:
        raise NdvmError(st, where)


def last_error() -> str:
    return (_last_error() or b"").decode(errors="replace")


def tape_build(bytecode: bytes) -> bytes:
    """Trace producer: stack bytecode -> serialized lane-invariant tape."""
    out, n = _vp(), _sz()
    _check(_tape_build(bytecode, len(bytecode), ctypes.byref(out), ctypes.byref(n)), "ndvm_tape_build")
    try:
        return ctypes.string_at(out, n.value)
    finally:
        _free(out)


class Tape:
    """Owner of an uploaded tape handle."""

    def __init__(self, handle: int):
        self.handle = handle

    def __del__(self, _free_fn=_tape_free, _finalizing=sys.is_finalizing):
        # at interpreter exit the device runtime may already be gone: leave
        # the handle to the process teardown then
        h, self.handle = getattr(self, "handle", None), None
        if h and not _finalizing():
            _free_fn(h)

    @property
    def info(self) -> dict:
        return tape_info(self)


def _stream_ptr(stream):
    import torch
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def _launch_stream(stream, device):
    """The torch stream a call launches on: the current stream when `stream`
    is None, else `stream` (a torch stream or a raw hipStream_t handle).
    Temporaries a call allocates (workspace, default outputs) are allocated
    and filled under this stream, so the caching allocator orders their reuse
    after the launch and a fill cannot land after the kernel's writes.  Inputs
    the caller produced on another stream are the caller's to order (as for
    any torch kernel launched on a side stream)."""
    import torch
    if stream is None:
        return torch.cuda.current_stream(device)
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream), device=device)


def tape_upload(tape_bytes: bytes, policy: int = POLICY_RECOMPUTE, stream=None) -> Tape:
    h = _vp()
    _check(_tape_upload(tape_bytes, len(tape_bytes), policy, _stream_ptr(stream), ctypes.byref(h)),
           "ndvm_tape_upload")
    return Tape(h.value)


def tape_upload_many(tapes: Sequence[bytes], policy: int = POLICY_RECOMPUTE, stream=None) -> list:
    """tape_upload for a population of tapes (one library call)."""
    n = len(tapes)
    arr = (ctypes.c_char_p * n)(*tapes)
    lens = (_sz * n)(*[len(t) for t in tapes])
    hs = (_vp * n)()
    _check(_tape_upload_many(arr, lens, n, policy, _stream_ptr(stream), hs), "ndvm_tape_upload_many")
    return [Tape(h) for h in hs]


def tape_info(tape: Tape) -> dict:
    info = _Info()
    _check(_tape_info(tape.handle, ctypes.byref(info)), "ndvm_tape_info_get")
    return {k: getattr(info, k) for k, _ in _Info._fields_}


def workspace_bytes(tape: Tape, L: int, with_grad: bool = True) -> int:
    n = _sz()
    _check(_ws_bytes(tape.handle, L, int(with_grad), ctypes.byref(n)), "ndvm_workspace_bytes")
    return n.value


def workspace_bytes_many(tapes: Sequence[Tape], L: int) -> int:
    arr = (_vp * len(tapes))(*[t.handle for t in tapes])
    n = _sz()
    _check(_ws_bytes_many(arr, len(tapes), L, ctypes.byref(n)), "ndvm_workspace_bytes_many")
    return n.value


def _dev_f64(t, name):
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float64 or not t.is_cuda:
        raise TypeError(f"{name} must be a float64 CUDA/ROCm tensor")
    return t


def _ld(t, dim=0):
    """Leading dimension of a row-major 2-D view: its row stride, or the row
    length when there is only one row (torch reports any stride for a
    dimension of size one)."""
    return t.stride(dim) if t.shape[dim] > 1 else max(t.shape[dim + 1], 1)


def _workspace(tape_or_bytes, device, workspace):
    import torch
    need = tape_or_bytes
    if workspace is None:
        return torch.empty(max(need, 8), dtype=torch.uint8, device=device), need
    if workspace.numel() * workspace.element_size() < need:
        raise ValueError("workspace too small")
    return workspace, workspace.numel() * workspace.element_size()


def forward(tape: Tape, params, obs, loss=None, workspace=None, stream=None):
    """loss[L] for params[L, P] (rows may be padded: params.stride(0) >= P)."""
    import torch
    _dev_f64(params, "params")
    _dev_f64(obs, "obs")
    if params.dim() != 2 or params.stride(1) != 1 or not obs.is_contiguous():
        raise ValueError("params must be [L, P] with unit inner stride; obs contiguous")
    L = params.shape[0]
    if workspace is not None and loss is not None:     # nothing to allocate: launch directly
        _check(_forward(tape.handle, params.data_ptr(), L, _ld(params), obs.data_ptr(), obs.numel(),
                        loss.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                        _stream_ptr(stream)), "ndvm_forward")
        return loss
    need = workspace_bytes(tape, L, False)
    s = _launch_stream(stream, params.device)
    with torch.cuda.stream(s):
        if loss is None:
            loss = torch.empty(L, dtype=torch.float64, device=params.device)
        ws, nbytes = _workspace(need, params.device, workspace)
        _check(_forward(tape.handle, params.data_ptr(), L, _ld(params), obs.data_ptr(), obs.numel(),
                        loss.data_ptr(), ws.data_ptr(), nbytes, s.cuda_stream), "ndvm_forward")
    return loss


def grad(tape: Tape, params, obs, loss=None, grad_out=None, workspace=None, stream=None):
    """(loss[L], grad[L, P]) for params[L, P]."""
    import torch
    _dev_f64(params, "params")
    _dev_f64(obs, "obs")
    if params.dim() != 2 or params.stride(1) != 1 or not obs.is_contiguous():
        raise ValueError("params must be [L, P] with unit inner stride; obs contiguous")
    L, P = params.shape
    if workspace is not None and loss is not None and grad_out is not None:   # launch directly
        _check(_grad(tape.handle, params.data_ptr(), L, _ld(params), obs.data_ptr(), obs.numel(),
                     loss.data_ptr(), grad_out.data_ptr(), _ld(grad_out), workspace.data_ptr(),
                     workspace.numel() * workspace.element_size(), _stream_ptr(stream)), "ndvm_grad")
        return loss, grad_out
    need = workspace_bytes(tape, L, True)
    s = _launch_stream(stream, params.device)
    with torch.cuda.stream(s):
        if loss is None:
            loss = torch.empty(L, dtype=torch.float64, device=params.device)
        if grad_out is None:
            grad_out = torch.empty((L, P), dtype=torch.float64, device=params.device)
        ws, nbytes = _workspace(need, params.device, workspace)
        _check(_grad(tape.handle, params.data_ptr(), L, _ld(params), obs.data_ptr(), obs.numel(),
                     loss.data_ptr(), grad_out.data_ptr(), _ld(grad_out), ws.data_ptr(), nbytes,
                     s.cuda_stream), "ndvm_grad")
    return loss, grad_out


def grad_noalloc(tape: Tape, params, obs, loss, grad_out, stream=None):
    """ndvm_grad_noalloc: (loss[L], grad[L, P]) into the caller's buffers with
    no workspace (the library's static scratch array serves).  The lane count
    must have been prepared with workspace_bytes(tape, L, True)."""
    for name, x in (("params", params), ("obs", obs), ("loss", loss), ("grad", grad_out)):
        _dev_f64(x, name)
    if params.dim() != 2 or params.stride(1) != 1 or not obs.is_contiguous() or grad_out.stride(1) != 1:
        raise ValueError("params and grad must be [L, P] with unit inner stride; obs contiguous")
    L = params.shape[0]
    if loss.numel() < L or grad_out.shape[0] < L:
        raise ValueError("loss and grad must hold L rows")
    _check(_grad_noalloc(tape.handle, params.data_ptr(), L, _ld(params), obs.data_ptr(), obs.numel(),
                         loss.data_ptr(), grad_out.data_ptr(), _ld(grad_out), _stream_ptr(stream)),
           "ndvm_grad_noalloc")
    return loss, grad_out


def workspace_bytes_points(tape: Tape, L: int, n_points: int) -> int:
    n = _sz()
    _check(_ws_bytes_points(tape.handle, L, n_points, ctypes.byref(n)), "ndvm_workspace_bytes_points")
    return n.value


def grad_points(tape: Tape, params, points, scale: float, loss=None, grad_out=None, workspace=None, stream=None):
    """Flattened data axis (ndvm_grad_points): `tape` is the per-point term
    program; points[N, D] holds each data point's observation row; returns
    (loss[L], grad[L, P]) of scale * sum over points of the term."""
    import torch
    _dev_f64(params, "params")
    _dev_f64(points, "points")
    if params.dim() != 2 or params.stride(1) != 1 or points.dim() != 2 or points.stride(1) != 1:
        raise ValueError("params [L, P] and points [N, D] need unit inner stride")
    L, P = params.shape
    N = points.shape[0]
    if workspace is not None and loss is not None and grad_out is not None:   # launch directly
        _check(_grad_points(tape.handle, params.data_ptr(), L, _ld(params), points.data_ptr(), N, _ld(points),
                            float(scale), loss.data_ptr(), grad_out.data_ptr(), _ld(grad_out), workspace.data_ptr(),
                            workspace.numel() * workspace.element_size(), _stream_ptr(stream)), "ndvm_grad_points")
        return loss, grad_out
    need = workspace_bytes_points(tape, L, N)
    s = _launch_stream(stream, params.device)
    with torch.cuda.stream(s):
        if loss is None:
            loss = torch.empty(L, dtype=torch.float64, device=params.device)
        if grad_out is None:
            grad_out = torch.empty((L, P), dtype=torch.float64, device=params.device)
        ws, nbytes = _workspace(need, params.device, workspace)
        _check(_grad_points(tape.handle, params.data_ptr(), L, _ld(params), points.data_ptr(), N,
                            _ld(points), float(scale), loss.data_ptr(), grad_out.data_ptr(), _ld(grad_out),
                            ws.data_ptr(), nbytes, s.cuda_stream), "ndvm_grad_points")
    return loss, grad_out


def grad_many(tapes: Sequence[Tape], params, obs, loss=None, grad_out=None, workspace=None, stream=None):
    """Many programs in one launch: params[n_prog, L, Pmax] -> loss[n_prog, L],
    grad[n_prog, L, Pmax] (entries beyond a program's own P are left as is)."""
    import torch
    _dev_f64(params, "params")
    _dev_f64(obs, "obs")
    if params.dim() != 3 or params.stride(2) != 1 or not obs.is_contiguous():
        raise ValueError("params must be [n_prog, L, Pmax] with unit inner stride")
    n_prog, L, P = params.shape
    if n_prog != len(tapes):
        raise ValueError("one tape per program row")
    need = workspace_bytes_many(tapes, L)
    s = _launch_stream(stream, params.device)
    with torch.cuda.stream(s):
        if loss is None:
            loss = torch.empty((n_prog, L), dtype=torch.float64, device=params.device)
        if grad_out is None:
            grad_out = torch.zeros((n_prog, L, P), dtype=torch.float64, device=params.device)
        ws, nbytes = _workspace(need, params.device, workspace)
        arr = (_vp * n_prog)(*[t.handle for t in tapes])
        ldp, ldg = _ld(params, 1), _ld(grad_out, 1)
        sp = params.stride(0) if n_prog > 1 else L * ldp
        sg = grad_out.stride(0) if n_prog > 1 else L * ldg
        _check(_grad_many(arr, n_prog, params.data_ptr(), L, ldp, sp, obs.data_ptr(),
                          obs.numel(), loss.data_ptr(), grad_out.data_ptr(), ldg,
                          sg, ws.data_ptr(), nbytes, s.cuda_stream), "ndvm_grad_many")
    return loss, grad_out


class WalkSet:
    """Owner of a program set prepared for the device walker."""

    def __init__(self, handle: int, n_prog: int):
        self.handle = handle
        self.n_prog = n_prog

    def __del__(self, _free_fn=_walk_free, _finalizing=sys.is_finalizing):
        h, self.handle = getattr(self, "handle", None), None
        if h and not _finalizing():
            _free_fn(h)


def walk_prepare(bytecodes: Sequence[bytes], stream=None) -> WalkSet:
    """Validate stack-bytecode programs and copy them to the GPU for the
    device walker (ndvm_walk_prepare): no tape, no scheduling."""
    n = len(bytecodes)
    arr = (ctypes.c_char_p * n)(*bytecodes)
    lens = (_sz * n)(*[len(b) for b in bytecodes])
    h = _vp()
    _check(_walk_prepare(arr, lens, n, _stream_ptr(stream), ctypes.byref(h)), "ndvm_walk_prepare")
    return WalkSet(h.value, n)


def walk_measure(bytecode: bytes) -> dict:
    """Host-only validation and structural measurement of one program for the
    device walker (ndvm_walk_measure)."""
    info = _WalkInfo()
    _check(_walk_measure(bytecode, len(bytecode), ctypes.byref(info)), "ndvm_walk_measure")
    return {k: getattr(info, k) for k, _ in _WalkInfo._fields_}


def walk_workspace_bytes(ws: WalkSet, L: int) -> int:
    n = _sz()
    _check(_walk_ws_bytes(ws.handle, int(L), ctypes.byref(n)), "ndvm_walk_workspace_bytes")
    return n.value


def walk_grad(ws: WalkSet, params, obs, loss=None, grad_out=None, workspace=None, stream=None):
    """The device walk of every program of the set: params[n_prog, L, Pmax]
    (or [L, P] for one program) -> loss, grad of the same leading shape
    (entries beyond a program's own P are left as is)."""
    import torch
    _dev_f64(params, "params")
    _dev_f64(obs, "obs")
    single = params.dim() == 2
    p3 = params.unsqueeze(0) if single else params
    if p3.dim() != 3 or p3.stride(2) != 1 or not obs.is_contiguous():
        raise ValueError("params must be [n_prog, L, Pmax] (or [L, P]) with unit inner stride")
    n_prog, L, P = p3.shape
    if n_prog != ws.n_prog:
        raise ValueError("one parameter block per program of the set")
    need = walk_workspace_bytes(ws, L)
    s = _launch_stream(stream, params.device)
    with torch.cuda.stream(s):
        if loss is None:
            loss = torch.empty((n_prog, L) if not single else (L,), dtype=torch.float64, device=params.device)
        if grad_out is None:
            grad_out = torch.zeros(tuple(params.shape), dtype=torch.float64, device=params.device)
        g3 = grad_out.unsqueeze(0) if single else grad_out
        work, nbytes = _workspace(need, params.device, workspace)
        ldp, ldg = _ld(p3, 1), _ld(g3, 1)
        sp = p3.stride(0) if n_prog > 1 else L * ldp
        sg = g3.stride(0) if n_prog > 1 else L * ldg
        _check(_walk_grad(ws.handle, p3.data_ptr(), L, ldp, sp, obs.data_ptr(), obs.numel(), loss.data_ptr(),
                          g3.data_ptr(), ldg, sg, work.data_ptr(), nbytes, s.cuda_stream), "ndvm_walk_grad")
    return loss, grad_out


def walk_status(workspace, stream=None):
    """Synchronise `stream` and raise if a walk that used `workspace` met a
    bound its validation should have excluded (ndvm_walk_status)."""
    _check(_walk_status(workspace.data_ptr(), _stream_ptr(stream)), "ndvm_walk_status")


def adam_step(params, grad_in, m, v, t: int, lr: float, beta1: float = 0.9, beta2: float = 0.999,
              eps: float = 1e-8, stream=None):
    """One Adam step for params[L, P] in place (ndvm_adam_step); m and v are
    [L, P] contiguous moment buffers, zero before step t = 1."""
    for name, x in (("params", params), ("grad", grad_in), ("m", m), ("v", v)):
        _dev_f64(x, name)
    if params.dim() != 2 or params.stride(1) != 1 or grad_in.stride(1) != 1:
        raise ValueError("params and grad must be [L, P] with unit inner stride")
    L, P = params.shape
    if tuple(grad_in.shape) != (L, P) or tuple(m.shape) != (L, P) or tuple(v.shape) != (L, P) \
            or not m.is_contiguous() or not v.is_contiguous():
        raise ValueError("grad, m and v must match params [L, P]; m and v contiguous")
    _check(_adam(params.data_ptr(), grad_in.data_ptr(), m.data_ptr(), v.data_ptr(), L, P, _ld(params),
                 _ld(grad_in), int(t), float(lr), float(beta1), float(beta2), float(eps),
                 _stream_ptr(stream)), "ndvm_adam_step")
    return params


# ---------------------------------------------------------------- encoder operators
# These are called for single tokens too, whose kernels take a few microseconds:
# the checks below are written to cost little when they pass.  Their results carry no
# gradient, whatever the arguments require: torch_api has the differentiable forms.
class _Torch:
    """torch, the type codes, and the look-ups of the current device and a device's current stream, found once."""

    def __init__(self):
        import torch
        self.torch = torch
        self.codes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
        self.f32, self.u8, self.i64, self.e4m3 = torch.float32, torch.uint8, torch.int64, torch.float8_e4m3fn
        self.Tensor, self.empty_like = torch.Tensor, torch.empty_like
        self.grad_enabled, self.increment_version = torch.is_grad_enabled, torch.autograd.graph.increment_version
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.raw_stream = raw or (lambda index: torch.cuda.current_stream(index).cuda_stream)
        self.current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


_torch_once = None


def _t():
    global _torch_once
    if _torch_once is None:
        _torch_once = _Torch()
    return _torch_once


def _op_type(t, x, name):
    """The dtype code of x, a tensor of a supported type on the GPU."""
    if isinstance(x, t.Tensor) and x.is_cuda:
        code = t.codes.get(x.dtype)
        if code is not None:
            return code
    raise TypeError(f"{name} must be a float32, bfloat16 or float16 CUDA/ROCm tensor")


def _alike(x, *others):
    """Raises unless the (name, tensor) pairs have the type and device of x."""
    for name, o in others:
        if getattr(o, "dtype", None) is not x.dtype or o.device != x.device:
            raise TypeError(f"{name} must be a tensor of the type and device of the first")


def _of(x, name, dtype, shape, device):
    """Address of a contiguous tensor of that type and shape, or None."""
    if x is None:
        return None
    if getattr(x, "dtype", None) is not dtype or x.device != device:
        raise TypeError(f"{name} must be a {dtype} tensor on {device}")
    if x.shape != shape or not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous, of shape {tuple(shape)}")
    return x.data_ptr()


def _to_write(t, x, name):
    """Before a call that writes x through its address: autograd has to see the write, so that a backward pass
    that saved x refuses to run on the new values, and a graph that x is part of may not lose it."""
    if x.requires_grad and t.grad_enabled():
        raise ValueError(f"{name} is written in place, which has no gradient: detach it")
    t.increment_version(x)


def _apart(out, *inputs):
    """Raises where `out` plainly lies over one of the (name, tensor) pairs, which the call reads after it has written there."""
    at = out.data_ptr()
    for name, x in inputs:
        p = x.data_ptr()
        if p == at or (out.is_contiguous() and x.is_contiguous() and p < at + out.numel() * out.element_size()
                       and at < p + x.numel() * x.element_size()):
            if out.numel() and x.numel():
                raise ValueError(f"out shares memory with {name}")


def _row_stride(x, name):
    """Stride of the rows (last axis) of a tensor whose other axes flatten into one."""
    shape = x.shape
    if not shape:
        raise ValueError(f"{name} must have rows")
    n = shape[-1]
    if x.is_contiguous():
        return n if n > 1 else 1
    strides = x.stride()
    if n > 1 and strides[-1] != 1:
        raise ValueError(f"{name} must have unit inner stride")
    step, ld = None, max(n, 1)
    for size, stride in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if size == 1:
            continue
        if step is None:
            ld = stride
        elif stride != step:
            raise ValueError(f"{name}: leading axes must flatten into rows of one stride")
        step = stride * size
    return ld


def _like(t, x):
    """A contiguous tensor of x's shape (empty_like takes half a microsecond less than new_empty)."""
    return t.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


class _On:
    """Where a call launches and allocates: the current stream of the tensors'
    device, or the given one (see _launch_stream).  A launch goes to the current
    device (a default stream's handle, 0, names none), so another one is made current
    meanwhile; where the tensors' is, there is nothing to switch."""
    __slots__ = ("ctx", "ptr")

    def __init__(self, t, stream, device):
        if stream is None:
            self.ctx = None if device.index == t.current_device() else t.torch.cuda.device(device)
            self.ptr = t.raw_stream(device.index)
        else:
            s = _launch_stream(stream, device)
            if s.device != device:
                raise ValueError(f"stream must be on {device}, where the tensors are, not on {s.device}")
            self.ctx, self.ptr = t.torch.cuda.stream(s), s.cuda_stream

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        return self.ptr

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out=None, stream=None):
    """(y, mean, rstd) of the rows (last axis) of x (ndvm_layer_norm); mean and
    rstd are float32 of x's leading shape, what layer_norm_grad takes.  (With
    autograd: torch_api.layer_norm.)"""
    t = _t()
    dt, dtype, dev, shape = _op_type(t, x, "x"), x.dtype, x.device, x.shape
    ld = _row_stride(x, "x")
    n, lead = shape[-1], shape[:-1]
    rows = x.numel() // n if n else 0
    w, b = _of(weight, "weight", dtype, (n,), dev), _of(bias, "bias", dtype, (n,), dev)
    with _On(t, stream, dev) as s:
        if out is None:
            out, ld_out = _like(t, x), n
        else:
            _alike(x, ("out", out))
            if out.shape != shape:
                raise ValueError("out must have the shape of x")
            ld_out = _row_stride(out, "out")
            _to_write(t, out, "out")
        mean = x.new_empty(lead, dtype=t.f32)
        rstd = t.empty_like(mean)
        st = _norm(dt, x.data_ptr(), rows, n, ld, w, b, eps, out.data_ptr(), ld_out, mean.data_ptr(), rstd.data_ptr(), s)
        if st:
            _check(st, "ndvm_layer_norm")
    return out, mean, rstd


def layer_norm_grad(dy, x, weight, mean, rstd, need_input: bool = True, need_weight: bool = True, stream=None):
    """(dx, dweight, dbias) of layer_norm (ndvm_layer_norm_grad); what is not
    needed is None.  weight may be None (no dweight's factor; its gradient is
    still that of a weight of ones)."""
    t = _t()
    dt, dtype, dev, shape = _op_type(t, x, "x"), x.dtype, x.device, x.shape
    _alike(x, ("dy", dy))
    if dy.shape != shape:
        raise ValueError("dy must have the shape of x")
    ld_x, ld_dy = _row_stride(x, "x"), _row_stride(dy, "dy")
    n, lead = shape[-1], shape[:-1]
    rows = x.numel() // n if n else 0
    w = _of(weight, "weight", dtype, (n,), dev)
    m, r = _of(mean, "mean", t.f32, lead, dev), _of(rstd, "rstd", t.f32, lead, dev)
    with _On(t, stream, dev) as s:
        dx = _like(t, x) if need_input else None
        dw = db = ws = None
        need = _sz()
        if need_weight:
            dw = x.new_empty(n)
            db = t.empty_like(dw)
            _check(_norm_ws(rows, n, ctypes.byref(need)), "ndvm_layer_norm_workspace_bytes")
            ws = x.new_empty(need.value, dtype=t.u8)
        _check(_norm_grad(dt, dy.data_ptr(), ld_dy, x.data_ptr(), ld_x, rows, n, w, m, r,
                          dx.data_ptr() if need_input else None, n, dw.data_ptr() if need_weight else None,
                          db.data_ptr() if need_weight else None, ws.data_ptr() if need_weight else None, need.value, s),
               "ndvm_layer_norm_grad")
    return dx, dw, db


def _rms_args(t, x, weight, residual):
    """Checks of the norm's inputs: type, rows, their width, strides of x and of the residual, and addresses."""
    dt, dtype, dev, shape = _op_type(t, x, "x"), x.dtype, x.device, x.shape
    ld = _row_stride(x, "x")
    n = shape[-1]
    w, r, ld_r = _of(weight, "weight", dtype, (n,), dev), None, 0
    if residual is not None:
        _alike(x, ("residual", residual))
        if residual.shape != shape:
            raise ValueError("residual must have the shape of x")
        r, ld_r = residual.data_ptr(), _row_stride(residual, "residual")
    return dt, x.numel() // n if n else 0, n, ld, w, r, ld_r


def rms_norm(x, weight=None, residual=None, eps: float = 1e-5, out=None, stream=None):
    """(y, h, rstd) of the rows (last axis) of x (ndvm_rms_norm): h = x + residual
    (x itself without one, which `out` may then not lie over), y its norm; rstd, float32
    of x's leading shape, is what rms_norm_grad takes.  (With autograd: torch_api.rms_norm.)"""
    t = _t()
    dt, rows, n, ld, w, r, ld_r = _rms_args(t, x, weight, residual)
    with _On(t, stream, x.device) as s:
        if out is None:
            out, ld_out = _like(t, x), n
        else:
            _alike(x, ("out", out))
            if out.shape != x.shape:
                raise ValueError("out must have the shape of x")
            if r is None:
                _apart(out, ("x", x))
            ld_out = _row_stride(out, "out")
            _to_write(t, out, "out")
        h = x if r is None else _like(t, x)
        rstd = x.new_empty(x.shape[:-1], dtype=t.f32)
        st = _rms(dt, x.data_ptr(), rows, n, ld, r, ld_r, w, eps, out.data_ptr(), ld_out, h.data_ptr(), n, rstd.data_ptr(), s)
        if st:
            _check(st, "ndvm_rms_norm")
    return out, h, rstd


def rms_norm_grad(dy, h, weight, rstd, dh=None, need_input: bool = True, need_weight: bool = True, stream=None):
    """(dx, dweight) of rms_norm (ndvm_rms_norm_grad), dx with dh, what arrives at h
    from elsewhere, added: it is the residual's gradient too.  What is not needed is
    None; weight may be None (its gradient is still that of a weight of ones)."""
    t = _t()
    dt, dtype, dev, shape = _op_type(t, h, "h"), h.dtype, h.device, h.shape
    _alike(h, ("dy", dy))
    if dy.shape != shape:
        raise ValueError("dy must have the shape of h")
    ld_h, ld_dy = _row_stride(h, "h"), _row_stride(dy, "dy")
    n, lead = shape[-1], shape[:-1]
    rows = h.numel() // n if n else 0
    w, r = _of(weight, "weight", dtype, (n,), dev), _of(rstd, "rstd", t.f32, lead, dev)
    more, ld_more = None, 0
    if dh is not None:
        _alike(h, ("dh", dh))
        if dh.shape != shape:
            raise ValueError("dh must have the shape of h")
        more, ld_more = dh.data_ptr(), _row_stride(dh, "dh")
    with _On(t, stream, dev) as s:
        dx = _like(t, h) if need_input else None
        dw = ws = None
        need = _sz()
        if need_weight:
            dw = h.new_empty(n)
            _check(_rms_ws(rows, n, ctypes.byref(need)), "ndvm_rms_norm_workspace_bytes")
            ws = h.new_empty(need.value, dtype=t.u8)
        _check(_rms_grad(dt, dy.data_ptr(), ld_dy, h.data_ptr(), ld_h, rows, n, w, r, more, ld_more,
                         dx.data_ptr() if need_input else None, n, dw.data_ptr() if need_weight else None,
                         ws.data_ptr() if need_weight else None, need.value, s), "ndvm_rms_norm_grad")
    return dx, dw


def rms_norm_8bit(x, weight=None, residual=None, eps: float = 1e-5, stream=None):
    """(y, scale, h) (ndvm_rms_norm_8bit): rms_norm's y rounded once to float8_e4m3fn, whose
    values stand for themselves times their row's scale (float32 of x's leading shape).
    There is no gradient through it."""
    t = _t()
    dt, rows, n, ld, w, r, ld_r = _rms_args(t, x, weight, residual)
    with _On(t, stream, x.device) as s:
        y = x.new_empty(x.shape, dtype=t.e4m3)
        h = x if r is None else _like(t, x)
        scale = x.new_empty(x.shape[:-1], dtype=t.f32)
        _check(_rms_8bit(dt, x.data_ptr(), rows, n, ld, r, ld_r, w, eps, y.data_ptr(), n, scale.data_ptr(), h.data_ptr(), n, s),
               "ndvm_rms_norm_8bit")
    return y, scale, h


def quantize_rows(x, stream=None):
    """(y, scale) (ndvm_quantize_rows): the rows of x in float8_e4m3fn and their scales, as
    rms_norm_8bit returns them; for the weights of linear_8bit."""
    t = _t()
    dt, rows, n, ld, _, _, _ = _rms_args(t, x, None, None)
    with _On(t, stream, x.device) as s:
        y, scale = x.new_empty(x.shape, dtype=t.e4m3), x.new_empty(x.shape[:-1], dtype=t.f32)
        _check(_quantize(dt, x.data_ptr(), rows, n, ld, y.data_ptr(), n, scale.data_ptr(), s), "ndvm_quantize_rows")
    return y, scale


def _heads(x, name, lead, heads, width):
    """An ndvm_heads of x [seqs, tokens, heads, width] (lead of two) or [tokens, heads, width]."""
    if x.shape != (*lead, heads, width):
        raise ValueError(f"{name} must have shape {(*lead, heads, width)}, not {tuple(x.shape)}")
    strides = x.stride()
    if width > 1 and strides[-1] != 1:
        raise ValueError(f"{name} must have unit inner stride")
    if len(lead) == 2:
        return _Heads(x.data_ptr(), strides[0], strides[1], strides[2])
    return _Heads(x.data_ptr(), 0, strides[0], strides[1])


def _attention(t, q, k, v, log_decay, offsets, scale):
    """Checks of the arguments that the attention calls share: shape struct, q, k, v, decay and offset pointers."""
    dt = _op_type(t, q, "q")
    _alike(q, ("k", k), ("v", v))
    packed = offsets is not None
    if packed:
        off = _of(offsets, "offsets", t.i64, (offsets.numel(),), q.device)
        if offsets.numel() < 1:
            raise ValueError("offsets must hold one more than there are sequences")
    if q.dim() != (3 if packed else 4) or k.dim() != q.dim() or v.dim() != q.dim():
        raise ValueError("q, k and v must be [sequences, tokens, heads, d], or [tokens, heads, d] with offsets")
    *lead, H, dk = q.shape
    lead = tuple(lead)
    Hk, dv = v.shape[-2:]
    decay = _of(log_decay, "log_decay", t.f32, (H,), q.device)
    if packed:
        n_seq, n = offsets.numel() - 1, lead[0]
    else:
        off, n_seq, n = None, lead[0], lead[0] * lead[1]
    shape = _AttentionShape(dt, n_seq, n, H, Hk, dk, dv, dk ** -0.5 if scale is None else scale)
    return (shape, lead, off, decay, _heads(q, "q", lead, H, dk), _heads(k, "k", lead, Hk, dk),
            _heads(v, "v", lead, Hk, dv))


def _attention_workspace(t, x, shape, packed, grad):
    need = _sz()
    _check(_attn_ws(shape, packed, grad, ctypes.byref(need)), "ndvm_linear_attention_workspace_bytes")
    ws = x.new_empty(need.value, dtype=t.u8) if need.value else None
    return ws, ws.data_ptr() if ws is not None else None, need.value


def linear_attention(q, k, v, log_decay, offsets=None, scale=None, initial_state=None, out=None,
                     final_state: bool = False, stream=None):
    """Linear attention with a decay for each head (ndvm_linear_attention):
    (o, final state or None) for q [sequences, tokens, heads, dk], k and v
    [.., kv_heads, dk or dv]; with `offsets` (int64 [sequences + 1], on the
    device, from 0 to the number of tokens) the sequences lie one after the other in
    [tokens, heads, d]; tokens outside them get no output.
    log_decay: float32 [heads]; scale: dk**-0.5 unless given; states are
    float32 [sequences, heads, dk, dv].  (With autograd: torch_api.linear_attention.)"""
    t = _t()
    shape, lead, off, decay, hq, hk, hv = _attention(t, q, k, v, log_decay, offsets, scale)
    dims, dev = (shape.n_seq, shape.heads, shape.dk, shape.dv), q.device
    s0 = _of(initial_state, "initial_state", t.f32, dims, dev)
    with _On(t, stream, dev) as s:
        if out is None:
            out = q.new_empty((*lead, shape.heads, shape.dv))
        else:
            _alike(q, ("out", out))
            _to_write(t, out, "out")
        last = q.new_empty(dims, dtype=t.f32) if final_state else None
        ws, ws_ptr, need = _attention_workspace(t, q, shape, off is not None, 0)
        _check(_attn(shape, hq, hk, hv, decay, off, s0, _heads(out, "out", lead, shape.heads, shape.dv),
                     last.data_ptr() if final_state else None, ws_ptr, need, s), "ndvm_linear_attention")
    return out, last


def linear_attention_grad(do, q, k, v, log_decay, offsets=None, scale=None, initial_state=None,
                          grad_final_state=None, need=(True, True, True), stream=None):
    """(dq, dk, dv, d initial_state) of linear_attention (ndvm_linear_attention_grad);
    what is not needed, or has no initial state, is None."""
    t = _t()
    shape, lead, off, decay, hq, hk, hv = _attention(t, q, k, v, log_decay, offsets, scale)
    _alike(q, ("do", do))
    H, Hk, dk, dv, dev = shape.heads, shape.kv_heads, shape.dk, shape.dv, q.device
    dims = (shape.n_seq, H, dk, dv)
    s0 = _of(initial_state, "initial_state", t.f32, dims, dev)
    ds = _of(grad_final_state, "grad_final_state", t.f32, dims, dev)
    hdo = _heads(do, "do", lead, H, dv)
    with _On(t, stream, dev) as s:
        def empty(wanted, heads, width):
            if not wanted:
                return None, _Heads(None, 0, 0, 0)
            x = q.new_empty((*lead, heads, width))
            return x, _heads(x, "", lead, heads, width)

        gq, hgq = empty(need[0], H, dk)
        gk, hgk = empty(need[1], Hk, dk)
        gv, hgv = empty(need[2], Hk, dv)
        d0 = q.new_empty(dims, dtype=t.f32) if s0 is not None and need[2] else None
        ws, ws_ptr, n = _attention_workspace(t, q, shape, off is not None, 1)
        _check(_attn_grad(shape, hq, hk, hv, decay, off, s0, hdo, ds, hgq, hgk, hgv,
                          d0.data_ptr() if d0 is not None else None, ws_ptr, n, s), "ndvm_linear_attention_grad")
    return gq, gk, gv, d0


def linear_attention_step(q, k, v, log_decay, state, slots=None, scale=None, out=None, stream=None):
    """One new token of every stream (ndvm_linear_attention_step): q [streams,
    heads, dk], k and v [streams, kv_heads, d]; stream i's state is
    state[slots[i]] (float32 [slots, heads, dk, dv], updated in place; slot i
    without `slots`), or none, with output 0, where slots[i] is out of range.
    Returns o [streams, heads, dv].  There is no gradient through a step."""
    t = _t()
    dt = _op_type(t, q, "q")
    _alike(q, ("k", k), ("v", v))
    if q.dim() != 3 or v.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k and v must be [streams, heads, d]")
    n, H, dk = q.shape
    Hk, dv = v.shape[1:]
    dev = q.device
    if state.dim() != 4:
        raise ValueError("state must be [slots, heads, dk, dv]")
    st = _of(state, "state", t.f32, (state.shape[0], H, dk, dv), dev)
    sl = _of(slots, "slots", t.i64, (n,), dev)
    decay = _of(log_decay, "log_decay", t.f32, (H,), dev)

    def one(x, name, heads, width):
        strides = x.stride()
        if x.shape != (n, heads, width) or (width > 1 and strides[2] != 1):
            raise ValueError(f"{name} must have shape {(n, heads, width)} and unit inner stride")
        return _Heads(x.data_ptr(), strides[0], 0, strides[1])

    hq, hk, hv = one(q, "q", H, dk), one(k, "k", Hk, dk), one(v, "v", Hk, dv)
    shape = _AttentionShape(dt, n, 0, H, Hk, dk, dv, dk ** -0.5 if scale is None else scale)
    with _On(t, stream, dev) as s:
        if out is None:
            out = q.new_empty((n, H, dv))
        else:
            _alike(q, ("out", out))
            _to_write(t, out, "out")
        _to_write(t, state, "state")
        _check(_attn_step(shape, hq, hk, hv, decay, st, state.shape[0], sl, one(out, "out", H, dv), s),
               "ndvm_linear_attention_step")
    return out


def _gates(x, name, lead, heads):
    """An ndvm_heads of x [seqs, tokens, heads] (lead of two) or [tokens, heads]."""
    if x.shape != (*lead, heads):
        raise ValueError(f"{name} must have shape {(*lead, heads)}, not {tuple(x.shape)}")
    strides = x.stride()
    if len(lead) == 2:
        return _Heads(x.data_ptr(), strides[0], strides[1], strides[2])
    return _Heads(x.data_ptr(), 0, strides[0], strides[1])


def _delta_args(t, q, k, v, g, beta, offsets, scale):
    """Checks of the arguments that the delta rule's calls share: shape struct, leading sizes, offset pointer, and q, k, v,
    g and beta."""
    dt = _op_type(t, q, "q")
    _alike(q, ("k", k), ("v", v), ("g", g), ("beta", beta))
    packed = offsets is not None
    if packed:
        off = _of(offsets, "offsets", t.i64, (offsets.numel(),), q.device)
        if offsets.numel() < 1:
            raise ValueError("offsets must hold one more than there are sequences")
    if q.dim() != (3 if packed else 4) or k.dim() != q.dim() or v.dim() != q.dim():
        raise ValueError("q, k and v must be [sequences, tokens, heads, d], or [tokens, heads, d] with offsets")
    *lead, Hk, dk = q.shape
    lead = tuple(lead)
    H, dv = v.shape[-2:]
    if packed:
        n_seq, n = offsets.numel() - 1, lead[0]
    else:
        off, n_seq, n = None, lead[0], lead[0] * lead[1]
    shape = _DeltaShape(dt, n_seq, n, H, Hk, dk, dv, dk ** -0.5 if scale is None else scale)
    return (shape, lead, off, _heads(q, "q", lead, Hk, dk), _heads(k, "k", lead, Hk, dk), _heads(v, "v", lead, H, dv),
            _gates(g, "g", lead, H), _gates(beta, "beta", lead, H))


def _delta_workspace(t, x, shape, packed, grad):
    need = _sz()
    _check(_delta_ws(shape, packed, grad, ctypes.byref(need)), "ndvm_delta_attention_workspace_bytes")
    ws = x.new_empty(need.value, dtype=t.u8)
    return ws, ws.data_ptr(), need.value


def delta_attention(q, k, v, g, beta, offsets=None, scale=None, initial_state=None, out=None, final_state: bool = False,
                    stream=None):
    """Attention by the gated delta rule (ndvm_delta_attention): (o, final state or None)
    for q and k [sequences, tokens, qk_heads, dk], v [.., heads, dv], and g (log decays) and
    beta [.., heads]; with `offsets` (int64 [sequences + 1], on the device, from 0 to the
    number of tokens) the sequences lie one after the other in [tokens, heads, ..]; tokens
    outside them get no output.  heads: a multiple of qk_heads; scale: dk**-0.5 unless
    given; states are float32 [sequences, heads, dk, dv]; `out` may not lie over an input.
    (With autograd: torch_api.delta_attention.)"""
    t = _t()
    shape, lead, off, *heads = _delta_args(t, q, k, v, g, beta, offsets, scale)
    dims, dev = (shape.n_seq, shape.heads, shape.dk, shape.dv), q.device
    s0 = _of(initial_state, "initial_state", t.f32, dims, dev)
    with _On(t, stream, dev) as s:
        if out is None:
            out = q.new_empty((*lead, shape.heads, shape.dv))
        else:
            _alike(q, ("out", out))
            _apart(out, ("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta))
            _to_write(t, out, "out")
        last = q.new_empty(dims, dtype=t.f32) if final_state else None
        ws, ws_ptr, need = _delta_workspace(t, q, shape, off is not None, 0)
        _check(_delta(shape, *heads, off, s0, _heads(out, "out", lead, shape.heads, shape.dv),
                      last.data_ptr() if final_state else None, ws_ptr, need, s), "ndvm_delta_attention")
    return out, last


def delta_attention_grad(do, q, k, v, g, beta, offsets=None, scale=None, initial_state=None, grad_final_state=None,
                         need=(True, True, True, True, True), stream=None):
    """(dq, dk, dv, dg, dbeta, d initial_state) of delta_attention
    (ndvm_delta_attention_grad); what is not needed, or has no initial state, is None;
    tokens outside the sequences of `offsets` have gradient 0."""
    t = _t()
    shape, lead, off, *heads = _delta_args(t, q, k, v, g, beta, offsets, scale)
    _alike(q, ("do", do))
    H, Hk, dk, dv, dev = shape.heads, shape.qk_heads, shape.dk, shape.dv, q.device
    dims = (shape.n_seq, H, dk, dv)
    s0 = _of(initial_state, "initial_state", t.f32, dims, dev)
    ds = _of(grad_final_state, "grad_final_state", t.f32, dims, dev)
    hdo = _heads(do, "do", lead, H, dv)
    with _On(t, stream, dev) as s:
        def made(wanted, *size):
            if not wanted:
                return None, _Heads(None, 0, 0, 0)
            x = (q.new_empty if off is None else q.new_zeros)((*lead, *size))
            return x, _heads(x, "", lead, *size) if len(size) == 2 else _gates(x, "", lead, *size)

        grads, to = zip(*(made(*w) for w in ((need[0], Hk, dk), (need[1], Hk, dk), (need[2], H, dv), (need[3], H), (need[4], H))))
        d0 = q.new_empty(dims, dtype=t.f32) if s0 is not None else None
        ws, ws_ptr, n = _delta_workspace(t, q, shape, off is not None, 1)
        _check(_delta_grad(shape, *heads, off, s0, hdo, ds, *to, d0.data_ptr() if d0 is not None else None, ws_ptr, n, s),
               "ndvm_delta_attention_grad")
    return (*grads, d0)


def delta_attention_step(q, k, v, g, beta, state, slots=None, scale=None, out=None, stream=None):
    """One new token of every stream (ndvm_delta_attention_step): q and k [streams,
    qk_heads, dk], v [streams, heads, dv], g and beta [streams, heads]; stream i's state is
    state[slots[i]] (float32 [slots, heads, dk, dv], updated in place; slot i without
    `slots`), or none, with output 0, where slots[i] is out of range.  Returns o [streams,
    heads, dv].  There is no gradient through a step."""
    t = _t()
    dt = _op_type(t, q, "q")
    _alike(q, ("k", k), ("v", v), ("g", g), ("beta", beta))
    if q.dim() != 3 or v.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k and v must be [streams, heads, d]")
    n, Hk, dk = q.shape
    H, dv = v.shape[1:]
    dev = q.device
    if state.dim() != 4:
        raise ValueError("state must be [slots, heads, dk, dv]")
    st = _of(state, "state", t.f32, (state.shape[0], H, dk, dv), dev)
    sl = _of(slots, "slots", t.i64, (n,), dev)

    def one(x, name, *shape):
        strides = x.stride()
        if x.shape != (n, *shape) or (len(shape) == 2 and shape[1] > 1 and strides[2] != 1):
            raise ValueError(f"{name} must have shape {(n, *shape)} and unit inner stride")
        return _Heads(x.data_ptr(), strides[0], 0, strides[1])

    heads = (one(q, "q", Hk, dk), one(k, "k", Hk, dk), one(v, "v", H, dv), one(g, "g", H), one(beta, "beta", H))
    shape = _DeltaShape(dt, n, 0, H, Hk, dk, dv, dk ** -0.5 if scale is None else scale)
    with _On(t, stream, dev) as s:
        if out is None:
            out = q.new_empty((n, H, dv))
        else:
            _alike(q, ("out", out))
            _apart(out, ("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta))
            _to_write(t, out, "out")
        _to_write(t, state, "state")
        _check(_delta_step(shape, *heads, st, state.shape[0], sl, one(out, "out", H, dv), s), "ndvm_delta_attention_step")
    return out


def _ffn_args(t, x, w_gate, w_up, activation):
    dt = _op_type(t, x, "x")
    _alike(x, ("w_gate", w_gate), ("w_up", w_up))
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
    if w_gate.dim() != 2 or w_gate.shape != w_up.shape or x.dim() < 1 or x.shape[-1] != w_gate.shape[1]:
        raise ValueError("w_gate and w_up must be [n_out, n_in], x [.., n_in]")
    n_out, n_in = w_gate.shape
    return dt, act, x.numel() // n_in if n_in else 0, n_in, n_out


def _ffn_workspace(t, x, dt, rows, n_in, n_out, grad):
    need = _sz()
    _check(_ffn_ws(dt, rows, n_in, n_out, grad, ctypes.byref(need)), "ndvm_gated_ffn_workspace_bytes")
    ws = x.new_empty(need.value, dtype=t.u8) if need.value else None
    return ws, ws.data_ptr() if ws is not None else None, need.value


def gated_ffn(x, w_gate, w_up, activation: str = "silu", out=None, stream=None):
    """act(x w_gate^T) * (x w_up^T) (ndvm_gated_ffn) for x [.., n_in] and weights [n_out, n_in].
    (With autograd: torch_api.gated_ffn.)"""
    t = _t()
    dt, act, rows, n_in, n_out = _ffn_args(t, x, w_gate, w_up, activation)
    ld_x, ld_g, ld_u = _row_stride(x, "x"), _row_stride(w_gate, "w_gate"), _row_stride(w_up, "w_up")
    with _On(t, stream, x.device) as s:
        if out is None:
            out, ld_out = x.new_empty((*x.shape[:-1], n_out)), n_out
        else:
            _alike(x, ("out", out))
            if out.shape != (*x.shape[:-1], n_out):
                raise ValueError("out must be [.., n_out]")
            ld_out = _row_stride(out, "out")
            _to_write(t, out, "out")
        ws, ws_ptr, need = _ffn_workspace(t, x, dt, rows, n_in, n_out, 0)
        _check(_ffn(dt, act, x.data_ptr(), rows, n_in, ld_x, w_gate.data_ptr(), ld_g, w_up.data_ptr(), ld_u, n_out,
                    out.data_ptr(), ld_out, ws_ptr, need, s), "ndvm_gated_ffn")
    return out


def gated_ffn_grad(dh, x, w_gate, w_up, activation: str = "silu", need_input: bool = True, need_weight: bool = True,
                   stream=None):
    """(dx, dw_gate, dw_up) of gated_ffn (ndvm_gated_ffn_grad); what is not needed is None."""
    t = _t()
    dt, act, rows, n_in, n_out = _ffn_args(t, x, w_gate, w_up, activation)
    _alike(x, ("dh", dh))
    if dh.shape != (*x.shape[:-1], n_out):
        raise ValueError("dh must be [.., n_out]")
    with _On(t, stream, x.device) as s:
        dx = _like(t, x) if need_input else None
        dg = du = None
        if need_weight:
            dg, du = _like(t, w_gate), _like(t, w_up)
        ws, ws_ptr, need = _ffn_workspace(t, x, dt, rows, n_in, n_out, 1)
        _check(_ffn_grad(dt, act, dh.data_ptr(), _row_stride(dh, "dh"), x.data_ptr(), rows, n_in, _row_stride(x, "x"),
                         w_gate.data_ptr(), _row_stride(w_gate, "w_gate"), w_up.data_ptr(), _row_stride(w_up, "w_up"),
                         n_out, dx.data_ptr() if need_input else None, n_in, dg.data_ptr() if need_weight else None,
                         n_in, du.data_ptr() if need_weight else None, n_in, ws_ptr, need, s),
               "ndvm_gated_ffn_grad")
    return dx, dg, du


def _linear_sizes(x, weight, activation):
    """Checks of a projection's activation and sizes: (its code, rows, n_in, n_out)."""
    act = ACT_NONE if activation is None else ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be None or one of {sorted(ACTIVATIONS)}")
    if weight.dim() != 2 or x.dim() < 1 or x.shape[-1] != weight.shape[1]:
        raise ValueError("weight must be [n_out, n_in], x [.., n_in]")
    n_out, n_in = weight.shape
    return act, x.numel() // n_in if n_in else 0, n_in, n_out


def _linear_out(t, x, weight, dtype, n_out, residual, out):
    """Output of a projection, and the residual's address and stride; under the call's stream."""
    shape = (*x.shape[:-1], n_out)
    r, ld_r = None, 0
    if residual is not None:
        if getattr(residual, "dtype", None) is not dtype or residual.device != x.device:
            raise TypeError("residual must be a tensor of the output's type and device")
        if residual.shape != shape:
            raise ValueError("residual must be [.., n_out]")
        r, ld_r = residual.data_ptr(), _row_stride(residual, "residual")
    if out is None:
        return x.new_empty(shape, dtype=dtype), n_out, r, ld_r
    if getattr(out, "dtype", None) is not dtype or out.device != x.device:
        raise TypeError("out must be a tensor of the output's type and device")
    if out.shape != shape:
        raise ValueError("out must be [.., n_out]")
    _apart(out, ("x", x), ("weight", weight))
    ld = _row_stride(out, "out")
    _to_write(t, out, "out")
    return out, ld, r, ld_r


def linear(x, weight, bias=None, activation: Optional[str] = None, residual=None, out=None, stream=None):
    """act(x weight^T + bias) + residual (ndvm_linear) for x [.., n_in], weight [n_out, n_in],
    bias [n_out] and residual [.., n_out]; activation: None, silu, gelu, sigmoid or relu.
    `out` may be the residual, not lie over x or weight.  (With autograd: torch_api.linear.)"""
    t = _t()
    dt = _op_type(t, x, "x")
    _alike(x, ("weight", weight))
    act, rows, n_in, n_out = _linear_sizes(x, weight, activation)
    ld_x, ld_w = _row_stride(x, "x"), _row_stride(weight, "weight")
    b = _of(bias, "bias", x.dtype, (n_out,), x.device)
    with _On(t, stream, x.device) as s:
        out, ld_out, r, ld_r = _linear_out(t, x, weight, x.dtype, n_out, residual, out)
        need = _sz()
        _check(_linear_ws(dt, act, rows, n_in, n_out, 0, ctypes.byref(need)), "ndvm_linear_workspace_bytes")
        ws = x.new_empty(need.value, dtype=t.u8) if need.value else None
        _check(_linear(dt, act, x.data_ptr(), rows, n_in, ld_x, weight.data_ptr(), ld_w, n_out, b, r, ld_r, out.data_ptr(), ld_out,
                       ws.data_ptr() if ws is not None else None, need.value, s), "ndvm_linear")
    return out


def linear_grad(dy, x, weight, bias=None, activation: Optional[str] = None, need_input: bool = True, need_weight: bool = True,
                need_bias: bool = True, stream=None):
    """(dx, dweight, dbias) of linear (ndvm_linear_grad); what is not needed is None, as is
    dbias without a bias.  (The residual's gradient is dy.)"""
    t = _t()
    dt = _op_type(t, x, "x")
    _alike(x, ("weight", weight), ("dy", dy))
    act, rows, n_in, n_out = _linear_sizes(x, weight, activation)
    if dy.shape != (*x.shape[:-1], n_out):
        raise ValueError("dy must be [.., n_out]")
    b = _of(bias, "bias", x.dtype, (n_out,), x.device)
    ld_dy, ld_x, ld_w = _row_stride(dy, "dy"), _row_stride(x, "x"), _row_stride(weight, "weight")
    with _On(t, stream, x.device) as s:
        dx = _like(t, x) if need_input else None
        dw = _like(t, weight) if need_weight else None
        db = x.new_empty(n_out) if need_bias and b is not None else None
        need = _sz()
        _check(_linear_ws(dt, act, rows, n_in, n_out, 1, ctypes.byref(need)), "ndvm_linear_workspace_bytes")
        ws = x.new_empty(need.value, dtype=t.u8)
        _check(_linear_grad(dt, act, dy.data_ptr(), ld_dy, x.data_ptr(), rows, n_in, ld_x, weight.data_ptr(), ld_w, n_out, b,
                            dx.data_ptr() if dx is not None else None, n_in, dw.data_ptr() if dw is not None else None, n_in,
                            db.data_ptr() if db is not None else None, ws.data_ptr(), need.value, s), "ndvm_linear_grad")
    return dx, dw, db


def linear_8bit(x, x_scale, weight, weight_scale, bias=None, activation: Optional[str] = None, residual=None, dtype=None,
                out=None, stream=None):
    """linear of 8-bit rows (ndvm_linear_8bit): x [.., n_in] and weight [n_out, n_in] in
    float8_e4m3fn with a float32 scale for each row (rms_norm_8bit, quantize_rows); the
    result, bias and residual have the type `dtype` (bfloat16, unless it is float16).  There is
    no gradient through it."""
    t = _t()
    dtype = t.torch.bfloat16 if dtype is None else dtype
    dt = t.codes.get(dtype)
    if dt is None or dtype is t.f32:
        raise TypeError("dtype must be bfloat16 or float16")
    if not isinstance(x, t.Tensor) or not x.is_cuda or x.dtype is not t.e4m3:
        raise TypeError("x must be a float8_e4m3fn CUDA/ROCm tensor")
    _alike(x, ("weight", weight))
    act, rows, n_in, n_out = _linear_sizes(x, weight, activation)
    ld_x, ld_w = _row_stride(x, "x"), _row_stride(weight, "weight")
    xs, ws_ = _of(x_scale, "x_scale", t.f32, x.shape[:-1], x.device), _of(weight_scale, "weight_scale", t.f32, (n_out,), x.device)
    b = _of(bias, "bias", dtype, (n_out,), x.device)
    with _On(t, stream, x.device) as s:
        out, ld_out, r, ld_r = _linear_out(t, x, weight, dtype, n_out, residual, out)
        need = _sz()
        _check(_linear8_ws(rows, n_in, n_out, ctypes.byref(need)), "ndvm_linear_8bit_workspace_bytes")
        ws = x.new_empty(need.value, dtype=t.u8) if need.value else None
        _check(_linear8(dt, act, x.data_ptr(), xs, rows, n_in, ld_x, weight.data_ptr(), ws_, ld_w, n_out, b, r, ld_r, out.data_ptr(),
                        ld_out, ws.data_ptr() if ws is not None else None, need.value, s), "ndvm_linear_8bit")
    return out
