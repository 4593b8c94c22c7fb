"""Binding of a worker's layers (include/gar_linear.h): argument marshalling only, as in worker.py.

Every function has the name of its C entry point.  Matrices are 2-D CUDA tensors with unit column
stride and any row stride that keeps the rows apart; outputs and workspaces are allocated, unless given, on the stream
the call runs on.  The products are those of bfloat16 or float16 tensors.  There is no autograd: the gradient of a call is the call
that computes it.  Tensors that a call writes count as modified in place.  With stream= the inputs have to
stay alive until that stream has read them.  Nothing is computed here and there is no fallback.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Union

import torch

from . import worker
from .binding import GRAD_DTYPES, _check
from .worker import ACTIVATIONS, Activation, Checkpoint, GarCheckpoint, TokenLogprobs, _handle


class GarLinearLogprobsParams(C.Structure):
    """Mirror of gar_linear_logprobs_params_t."""
    _fields_ = [("dtype", C.c_int32), ("rows", C.c_int64), ("hidden", C.c_int64), ("vocab", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("weight", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p), ("targets", C.c_void_p), ("logprobs", C.c_void_p),
                ("lse", C.c_void_p), ("lse_lo", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class GarLinearLogprobsGradParams(C.Structure):
    """Mirror of gar_linear_logprobs_grad_params_t."""
    _fields_ = [("dtype", C.c_int32), ("grads_dtype", C.c_int32), ("workers", C.c_int32), ("tokens", C.c_int64), ("hidden", C.c_int64),
                ("vocab", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64), ("weight", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p),
                ("targets", C.c_void_p), ("lse", C.c_void_p), ("lse_lo", C.c_void_p), ("grad_logprobs", C.c_void_p), ("dx", C.c_void_p),
                ("lddx", C.c_int64), ("weight_grads", C.c_void_p), ("bias_grads", C.c_void_p), ("ld_grads", C.c_int64), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class GarGatedLinearParams(C.Structure):
    """Mirror of gar_gated_linear_params_t."""
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("group", C.c_int32), ("rows", C.c_int64), ("hidden", C.c_int64), ("inner", C.c_int64),
                ("x", C.c_void_p), ("ldx", C.c_int64), ("w_gate", C.c_void_p), ("ld_gate", C.c_int64), ("w_up", C.c_void_p), ("ld_up", C.c_int64),
                ("b_gate", C.c_void_p), ("b_up", C.c_void_p), ("y", C.c_void_p), ("ldy", C.c_int64), ("gate_saved", GarCheckpoint),
                ("up_saved", GarCheckpoint), ("y_saved", GarCheckpoint), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
                ("stream", C.c_void_p)]


class GarGatedLinearGradParams(C.Structure):
    """Mirror of gar_gated_linear_grad_params_t."""
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("group", C.c_int32), ("rows", C.c_int64), ("hidden", C.c_int64), ("inner", C.c_int64),
                ("dy", C.c_void_p), ("lddy", C.c_int64), ("gate_saved", GarCheckpoint), ("up_saved", GarCheckpoint), ("w_gate", C.c_void_p),
                ("ld_gate", C.c_int64), ("w_up", C.c_void_p), ("ld_up", C.c_int64), ("dgate", C.c_void_p), ("ld_dgate", C.c_int64),
                ("dup", C.c_void_p), ("ld_dup", C.c_int64), ("dx", C.c_void_p), ("lddx", C.c_int64), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class GarDropoutParams(C.Structure):
    """Mirror of gar_dropout_params_t."""
    _fields_ = [("dtype", C.c_int32), ("p", C.c_float), ("rows", C.c_int64), ("cols", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("residual", C.c_void_p), ("ld_residual", C.c_int64), ("y", C.c_void_p), ("ldy", C.c_int64), ("seed", C.c_uint64),
                ("offset", C.c_uint64), ("counter", C.c_void_p), ("stream", C.c_void_p)]


_typed = False


def lib():
    """libgar.so with the entry points of the layers typed."""
    global _typed
    L = worker.lib()
    if not _typed:
        for name, params in (("gar_linear_logprobs", GarLinearLogprobsParams), ("gar_linear_logprobs_backward", GarLinearLogprobsGradParams),
                             ("gar_gated_linear_forward", GarGatedLinearParams), ("gar_gated_linear_backward", GarGatedLinearGradParams),
                             ("gar_dropout", GarDropoutParams)):
            getattr(L, name).argtypes = [C.POINTER(params)]
        for name, params in (("gar_linear_logprobs_workspace_bytes", GarLinearLogprobsParams),
                             ("gar_linear_logprobs_backward_workspace_bytes", GarLinearLogprobsGradParams),
                             ("gar_gated_linear_workspace_bytes", GarGatedLinearParams),
                             ("gar_gated_linear_backward_workspace_bytes", GarGatedLinearGradParams)):
            getattr(L, name).argtypes = [C.POINTER(params)]
            getattr(L, name).restype = C.c_size_t
        _typed = True
    return L


def _native():
    return worker._native or worker._load()


class LinearLogprobs(NamedTuple):
    """What gar_linear_logprobs returns; also what its backward pass needs."""
    logprobs: Optional[torch.Tensor]        # float32 [rows]; None without targets
    lse: torch.Tensor                       # float32 [rows]
    lse_lo: Optional[torch.Tensor] = None   # float32 [rows]: what rounding lse to float32 left out


class GatedLinearGrad(NamedTuple):
    """What gar_gated_linear_backward returns.  Unless given, dgate and dup are made with rows that start on 32 bytes
    (a row stride of a multiple of 16), as the products read them fastest."""
    dx: Optional[torch.Tensor]
    dgate: torch.Tensor
    dup: torch.Tensor


def _place(t: torch.Tensor):
    """Address, rows, columns and row stride of a matrix, as the sizes calls look at them."""
    return t.data_ptr() or 16, t.shape[0], t.shape[1], t.stride(0) if t.shape[0] > 1 else t.shape[1]


def gar_linear_logprobs_workspace_bytes(x: torch.Tensor, weight: torch.Tensor) -> int:
    """Bytes of the workspace gar_linear_logprobs takes for these operands."""
    p = GarLinearLogprobsParams(dtype=GRAD_DTYPES[x.dtype])
    p.x, p.rows, p.hidden, p.ldx = _place(x)
    p.weight, p.vocab, _, p.ldw = _place(weight)
    return int(lib().gar_linear_logprobs_workspace_bytes(C.byref(p)))


def gar_linear_logprobs_backward_workspace_bytes(x: torch.Tensor, weight: torch.Tensor, grads: Optional[torch.Tensor] = None, bias: bool = False,
                                                 dx: bool = True) -> int:
    """Bytes of the workspace gar_linear_logprobs_backward takes for these operands; bias: whether bias gradients are asked for."""
    p = GarLinearLogprobsGradParams(dtype=GRAD_DTYPES[x.dtype], workers=1, dx=16 if dx else None)
    p.x, p.tokens, p.hidden, p.ldx = _place(x)
    p.weight, p.vocab, _, p.ldw = _place(weight)
    if grads is not None:
        p.workers, p.tokens, p.grads_dtype, p.weight_grads = grads.shape[0], x.shape[0] // grads.shape[0], GRAD_DTYPES[grads.dtype], 16
        p.bias_grads = 16 if bias else None
    return int(lib().gar_linear_logprobs_backward_workspace_bytes(C.byref(p)))


def gar_gated_linear_workspace_bytes(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor) -> int:
    """Bytes of the workspace gar_gated_linear_forward takes for these operands (0: none)."""
    p = GarGatedLinearParams(dtype=GRAD_DTYPES[x.dtype], group=128, y=16)
    p.x, p.rows, p.hidden, p.ldx = _place(x)
    p.w_gate, p.inner, _, p.ld_gate = _place(w_gate)
    p.w_up, _, _, p.ld_up = _place(w_up)
    return int(lib().gar_gated_linear_workspace_bytes(C.byref(p)))


def gar_gated_linear_backward_workspace_bytes(w_gate: torch.Tensor, w_up: torch.Tensor, dgate: torch.Tensor, dup: torch.Tensor) -> int:
    """Bytes of the workspace gar_gated_linear_backward takes for these operands (0: none)."""
    p = GarGatedLinearGradParams(dtype=GRAD_DTYPES[dgate.dtype], group=128, dy=16, dx=16)
    p.w_gate, p.inner, p.hidden, p.ld_gate = _place(w_gate)
    p.w_up, _, _, p.ld_up = _place(w_up)
    p.dgate, p.rows, _, p.ld_dgate = _place(dgate)
    p.dup, _, _, p.ld_dup = _place(dup)
    return int(lib().gar_gated_linear_backward_workspace_bytes(C.byref(p)))


def gar_linear_logprobs(x: torch.Tensor, weight: torch.Tensor, targets: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None) -> LinearLogprobs:
    """gar_linear_logprobs: x [rows, hidden], weight [vocab, hidden], bias [vocab], targets int64 [rows] (negative: none).
    The softmax cross entropy of a token is minus its log probability."""
    r = _native().linear_logprobs(x, weight, targets, bias, workspace, _handle(stream))
    if type(r) is int:
        _check(r, "gar_linear_logprobs")
    return LinearLogprobs(*r)


def gar_linear_logprobs_backward(x: torch.Tensor, weight: torch.Tensor, saved: Union[LinearLogprobs, TokenLogprobs], targets: torch.Tensor,
                                 grad_logprobs: torch.Tensor, bias: Optional[torch.Tensor] = None, grads: Optional[torch.Tensor] = None,
                                 weight_offset: int = 0, bias_offset: Optional[int] = None, dx: Union[bool, torch.Tensor] = True,
                                 workspace: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """gar_linear_logprobs_backward: returns the gradient at x (dx: True, or a tensor it goes into; False: not computed).
    grads: the gradient block [workers, d], row w of which gets the weight gradient (vocab x hidden, row-major) of the
    w-th of `workers` equal runs of x's rows from column weight_offset on and, with bias_offset, the bias gradient from there on."""
    if bias_offset is not None and bias_offset < 0:
        raise ValueError("bias_offset must not be negative")
    if grads is None and (weight_offset != 0 or bias_offset is not None):
        raise ValueError("offsets need `grads`")
    if not isinstance(dx, torch.Tensor):
        dx = bool(dx)
    r = _native().linear_logprobs_backward(x, weight, saved.lse, saved.lse_lo, targets, grad_logprobs, bias, grads, weight_offset,
                                           -1 if bias_offset is None else bias_offset, dx, workspace, _handle(stream))
    if type(r) is int:
        _check(r, "gar_linear_logprobs_backward")
    return r[0]


def gar_gated_linear_forward(act: str, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, b_gate: Optional[torch.Tensor] = None,
                             b_up: Optional[torch.Tensor] = None, group: int = 128, save_input: bool = True, save_output: bool = False,
                             y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> Activation:
    """gar_gated_linear_forward: y = act(x w_gate^T + b_gate) * (x w_up^T + b_up), with the checkpoints of the activation's two inputs
    (.x the gate's, .up) and / or of the output (.out), as gar_activation_forward returns them."""
    r = _native().gated_linear_forward(ACTIVATIONS[act], x, w_gate, w_up, b_gate, b_up, group, save_input, save_output, y, workspace, _handle(stream))
    if type(r) is int:
        _check(r, "gar_gated_linear_forward")
    inner, dtype = w_gate.shape[0], x.dtype
    y, gq, gs, uq, us, oq, os_ = r
    return Activation(y, None if gq is None else Checkpoint(gq, gs, inner, group, dtype), None if uq is None else Checkpoint(uq, us, inner, group, dtype),
                      None if oq is None else Checkpoint(oq, os_, inner, group, dtype))


def gar_gated_linear_backward(act: str, dy: torch.Tensor, gate: Checkpoint, up: Checkpoint, w_gate: torch.Tensor, w_up: torch.Tensor,
                              dx: Union[bool, torch.Tensor] = True, dgate: Optional[torch.Tensor] = None, dup: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, stream=None) -> GatedLinearGrad:
    """gar_gated_linear_backward: the gradients at x (dx: True, or a tensor it goes into; False: not computed) and at both projections
    (dgate may be dy: in place), from which gar_linear_weight_grad makes the workers' weight gradients."""
    if dy.dtype != gate.dtype:
        raise TypeError("dy must be of the checkpoints' type")
    if up.group != gate.group or up.dtype != gate.dtype or up.cols != gate.cols:
        raise ValueError("both checkpoints must have the same shape, group and type")
    if not isinstance(dx, torch.Tensor):
        dx = bool(dx)
    r = _native().gated_linear_backward(ACTIVATIONS[act], dy, gate.q, gate.scales, up.q, up.scales, gate.cols, gate.group, w_gate, w_up, dx, dgate, dup,
                                        workspace, _handle(stream))
    if type(r) is int:
        _check(r, "gar_gated_linear_backward")
    return GatedLinearGrad(*r)


def gar_dropout(x: torch.Tensor, p: float, seed: int, offset: int = 0, residual: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                counter: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """gar_dropout: y = [residual +] keep * x / (1 - p) for x [rows, cols], the mask a function of (seed, offset [+ counter], row, column):
    the same call on the gradient is the backward pass (without the residual).  seed and offset: 0 .. 2^64 - 1.  y may be x or the residual:
    in place.  counter: int64 CUDA tensor of one element, read when the call runs; a captured graph that is replayed takes its
    next mask by advancing it."""
    r = _native().dropout(x, p, seed, offset, residual, y, counter, _handle(stream))
    if type(r) is int:
        _check(r, "gar_dropout")
    return r
