"""Binding of the worker-side operators (include/gar_worker.h): argument marshalling only.

Every function has the name of its C entry point.  Matrices are 2-D CUDA tensors with unit column
stride and any row stride that keeps the rows apart (an expanded tensor, whose rows share memory, is
refused: make it contiguous); outputs are allocated, unless given, on the stream the call runs on.
There is no autograd: results carry no gradient function whatever the inputs require, and the gradient of
a call is the call that computes it.  Tensors that a call writes (y=, dx=, dup=, dlogits=, out=, grads)
count as modified in place, so autograd refuses a backward pass that saved one of them.  With stream= the
inputs have to stay alive until that stream has read them.  The marshalling
itself is compiled (csrc/worker_binding.cpp); the ctypes mirrors of the parameter blocks are for
callers of the C ABI.  Nothing is computed here and there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple, Optional

import torch

from .binding import GRAD_DTYPES, _check, lib as _base_lib

GAR_MAX_TOP = 32
ACTIVATIONS = {"identity": 0, "relu": 1, "silu": 2, "gelu": 3}


class GarCheckpoint(C.Structure):
    """Mirror of gar_checkpoint_t."""
    _fields_ = [("q", C.c_void_p), ("scales", C.c_void_p), ("ldq", C.c_int64)]


class GarLogprobsParams(C.Structure):
    """Mirror of gar_logprobs_params_t."""
    _fields_ = [("dtype", C.c_int32), ("top", C.c_int32), ("rows", C.c_int64), ("vocab", C.c_int64), ("ld", C.c_int64),
                ("logits", C.c_void_p), ("targets", C.c_void_p), ("logprobs", C.c_void_p), ("entropy", C.c_void_p),
                ("lse", C.c_void_p), ("lse_lo", C.c_void_p), ("top_logprobs", C.c_void_p), ("top_index", C.c_void_p), ("stream", C.c_void_p)]


class GarLogprobsGradParams(C.Structure):
    """Mirror of gar_logprobs_grad_params_t."""
    _fields_ = [("dtype", C.c_int32), ("top", C.c_int32), ("rows", C.c_int64), ("vocab", C.c_int64), ("ld", C.c_int64),
                ("logits", C.c_void_p), ("targets", C.c_void_p), ("lse", C.c_void_p), ("lse_lo", C.c_void_p), ("entropy", C.c_void_p),
                ("top_index", C.c_void_p), ("grad_logprobs", C.c_void_p), ("grad_entropy", C.c_void_p),
                ("grad_top", C.c_void_p), ("dlogits", C.c_void_p), ("ld_dlogits", C.c_int64), ("stream", C.c_void_p)]


class GarActivationParams(C.Structure):
    """Mirror of gar_activation_params_t."""
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("group", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int64),
                ("x", C.c_void_p), ("ldx", C.c_int64), ("up", C.c_void_p), ("ldup", C.c_int64), ("y", C.c_void_p),
                ("ldy", C.c_int64), ("x_saved", GarCheckpoint), ("up_saved", GarCheckpoint), ("y_saved", GarCheckpoint),
                ("stream", C.c_void_p)]


class GarActivationGradParams(C.Structure):
    """Mirror of gar_activation_grad_params_t."""
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("group", C.c_int32), ("rows", C.c_int64), ("cols", C.c_int64),
                ("dy", C.c_void_p), ("lddy", C.c_int64), ("x_saved", GarCheckpoint), ("up_saved", GarCheckpoint),
                ("dx", C.c_void_p), ("lddx", C.c_int64), ("dup", C.c_void_p), ("lddup", C.c_int64), ("stream", C.c_void_p)]


class GarWeightGradParams(C.Structure):
    """Mirror of gar_weight_grad_params_t."""
    _fields_ = [("dtype", C.c_int32), ("grads_dtype", C.c_int32), ("group", C.c_int32), ("workers", C.c_int32),
                ("tokens", C.c_int64), ("out_features", C.c_int64), ("in_features", C.c_int64), ("dy", C.c_void_p),
                ("ld_dy", C.c_int64), ("x_saved", GarCheckpoint), ("lengths", C.c_void_p), ("weight_grads", C.c_void_p),
                ("bias_grads", C.c_void_p), ("ld_grads", C.c_int64), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


_typed = False
_native = None
_NATIVE_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_gar_worker.so")


def lib():
    """libgar.so with the worker-side entry points typed."""
    global _typed
    L = _base_lib()
    if not _typed:
        L.gar_token_logprobs.argtypes = [C.POINTER(GarLogprobsParams)]
        L.gar_token_logprobs_backward.argtypes = [C.POINTER(GarLogprobsGradParams)]
        L.gar_activation_forward.argtypes = [C.POINTER(GarActivationParams)]
        L.gar_activation_backward.argtypes = [C.POINTER(GarActivationGradParams)]
        L.gar_checkpoint_pack.argtypes = [C.c_int, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int,
                                          C.POINTER(GarCheckpoint), C.c_void_p]
        L.gar_checkpoint_unpack.argtypes = [C.c_int, C.POINTER(GarCheckpoint), C.c_int64, C.c_int64, C.c_int, C.c_void_p,
                                            C.c_int64, C.c_void_p]
        L.gar_linear_weight_grad.argtypes = [C.POINTER(GarWeightGradParams)]
        L.gar_weight_grad_workspace_bytes.argtypes = [C.POINTER(GarWeightGradParams)]
        L.gar_weight_grad_workspace_bytes.restype = C.c_size_t
        L.gar_weight_grad_wants_workspace.argtypes = [C.POINTER(GarWeightGradParams)]
        _typed = True
    return L


def _load():
    """The compiled marshalling module.  Raises if it has not been built."""
    global _native
    if not os.path.exists(_NATIVE_PATH):
        raise RuntimeError(f"{_NATIVE_PATH} is missing: build it with "
                           "`python -m paper_1905_04374_b200.build`; there is no fallback")
    _base_lib()
    from . import _gar_worker
    _native = _gar_worker
    return _native


def _handle(stream):
    """A stream argument as the number of its CUDA handle; None: the current stream."""
    return None if stream is None else stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


class TokenLogprobs(NamedTuple):
    """What gar_token_logprobs returns; also what its backward pass needs."""
    logprobs: Optional[torch.Tensor]        # float32 [rows]; None without targets
    entropy: torch.Tensor                   # float32 [rows]
    lse: torch.Tensor                       # float32 [rows]
    top_logprobs: Optional[torch.Tensor]    # float32 [rows, top]; None for top = 0
    top_index: Optional[torch.Tensor]       # int64 [rows, top]
    lse_lo: Optional[torch.Tensor] = None   # float32 [rows]: what rounding lse to float32 left out


class Checkpoint(NamedTuple):
    """An activation [rows, cols] in 8 bits: codes and one scale per `group` columns of a row."""
    q: torch.Tensor                         # int8 [rows, cols rounded up to 16]
    scales: torch.Tensor                    # float32 [rows, ceil(cols / group)]
    cols: int
    group: int
    dtype: torch.dtype                      # what it is restored to


class Activation(NamedTuple):
    """What gar_activation_forward returns: the output and the checkpoints that were asked for."""
    y: torch.Tensor
    x: Optional[Checkpoint]
    up: Optional[Checkpoint]
    out: Optional[Checkpoint]


class ActivationGrad(NamedTuple):
    dx: torch.Tensor
    dup: Optional[torch.Tensor]


def gar_token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 0, stream=None) -> TokenLogprobs:
    """gar_token_logprobs: logits [rows, vocab], targets int64 [rows] (negative: none)."""
    r = (_native or _load()).token_logprobs(logits, targets, top, _handle(stream))
    if type(r) is int:
        _check(r, "gar_token_logprobs")
    return TokenLogprobs(*r)


def gar_token_logprobs_backward(logits: torch.Tensor, saved: TokenLogprobs, targets: Optional[torch.Tensor] = None,
                                grad_logprobs: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None,
                                grad_top: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                                stream=None) -> torch.Tensor:
    """gar_token_logprobs_backward: the gradient at the logits (dlogits may be logits: in place)."""
    r = (_native or _load()).token_logprobs_backward(logits, saved.lse, saved.lse_lo, saved.entropy, saved.top_index, targets,
                                                     grad_logprobs, grad_entropy, grad_top, dlogits, _handle(stream))
    if type(r) is int:
        _check(r, "gar_token_logprobs_backward")
    return r


def gar_checkpoint_pack(x: torch.Tensor, group: int = 128, stream=None) -> Checkpoint:
    """gar_checkpoint_pack: x [rows, cols] in 8 bits."""
    r = (_native or _load()).checkpoint_pack(x, group, _handle(stream))
    if type(r) is int:
        _check(r, "gar_checkpoint_pack")
    return Checkpoint(*r, x.shape[1], group, x.dtype)


def gar_checkpoint_unpack(saved: Checkpoint, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """gar_checkpoint_unpack: the restored activation [rows, cols]."""
    r = (_native or _load()).checkpoint_unpack(saved.q, saved.scales, saved.cols, saved.group, GRAD_DTYPES[saved.dtype], out,
                                               _handle(stream))
    if type(r) is int:
        _check(r, "gar_checkpoint_unpack")
    return r


def gar_activation_forward(act: str, x: torch.Tensor, up: Optional[torch.Tensor] = None, group: int = 128,
                           save_input: bool = True, save_output: bool = False, y: Optional[torch.Tensor] = None,
                           stream=None) -> Activation:
    """gar_activation_forward: y = act(x) (* up), with the checkpoints of the inputs and / or the output."""
    r = (_native or _load()).activation_forward(ACTIVATIONS[act], x, up, group, save_input, save_output, y, _handle(stream))
    if type(r) is int:
        _check(r, "gar_activation_forward")
    cols, dtype = x.shape[1], x.dtype
    y, xq, xs, uq, us, oq, os_ = r
    return Activation(y, None if xq is None else Checkpoint(xq, xs, cols, group, dtype),
                      None if uq is None else Checkpoint(uq, us, cols, group, dtype),
                      None if oq is None else Checkpoint(oq, os_, cols, group, dtype))


def gar_activation_backward(act: str, dy: torch.Tensor, x: Checkpoint, up: Optional[Checkpoint] = None,
                            dx: Optional[torch.Tensor] = None, dup: Optional[torch.Tensor] = None,
                            stream=None) -> ActivationGrad:
    """gar_activation_backward: gradients at x (and up) from the checkpoints (dx may be dy: in place)."""
    if dy.dtype != x.dtype:
        raise TypeError("dy must be of the checkpoint's type")
    if up is not None and (up.group != x.group or up.dtype != x.dtype or up.cols != x.cols):
        raise ValueError("both checkpoints must have the same shape, group and type")
    r = (_native or _load()).activation_backward(ACTIVATIONS[act], dy, x.q, x.scales, None if up is None else up.q,
                                                 None if up is None else up.scales, x.cols, x.group, dx, dup, _handle(stream))
    if type(r) is int:
        _check(r, "gar_activation_backward")
    return ActivationGrad(*r)


def gar_weight_grad_workspace_bytes(dy: torch.Tensor, x: Checkpoint, lengths: Optional[torch.Tensor] = None, bias: bool = False) -> int:
    """Bytes of the workspace gar_linear_weight_grad takes for these operands (0: it uses none)."""
    return (_native or _load()).weight_grad_workspace_bytes(dy, x.cols, x.group, lengths is not None, bias)


def gar_linear_weight_grad(dy: torch.Tensor, x: Checkpoint, grads: Optional[torch.Tensor] = None, weight_offset: int = 0,
                           bias_offset: Optional[int] = None, lengths: Optional[torch.Tensor] = None,
                           grads_dtype: torch.dtype = torch.float32, workspace=None, stream=None) -> torch.Tensor:
    """gar_linear_weight_grad: dy [workers, tokens, out] and the checkpoint of x [workers * tokens, in]
    into the gradient block `grads` [workers, d]: row w gets dW_w (out x in, row-major) from column
    weight_offset on and, with bias_offset, db_w from there on.  lengths int32 [workers]: tokens that
    count.  Without `grads` a block [workers, out * in] of grads_dtype is made.  workspace: None lets the
    call allocate one for layers where it is faster, False never (the codes are then restored tile by
    tile), or a uint8 CUDA tensor of gar_weight_grad_workspace_bytes.  That is room for the activation restored
    to 16 bits, twice the checkpoint (and for a copy of dy if its rows do not start on 16 bytes), or for the parts
    of a sum of many tokens: False where memory is shorter than time."""
    if dy.dtype != x.dtype:
        raise TypeError("dy and the checkpoint must be of one type")
    if dy.dim() != 3:
        raise ValueError("dy must be [workers, tokens, out]")
    out = dy.shape[2]
    if grads is None:
        if weight_offset != 0 or bias_offset is not None:
            raise ValueError("offsets need `grads`")
        grads = torch.empty(dy.shape[0], out * x.cols, dtype=grads_dtype, device=dy.device)
    if bias_offset is not None and bias_offset < 0:
        raise ValueError("bias_offset must not be negative")
    r = (_native or _load()).linear_weight_grad(dy, x.q, x.scales, x.cols, x.group, grads, weight_offset,
                                                -1 if bias_offset is None else bias_offset, lengths, workspace, _handle(stream))
    if r:
        _check(r, "gar_linear_weight_grad")
    return grads
