"""ctypes binding of the worker-side operators (include/gar_worker.h): argument marshalling only.

Every function has the name of its C entry point.  Matrices are 2-D CUDA tensors with unit column
stride (any row stride); outputs are allocated on the current stream unless given.  Nothing is
computed here and there is no fallback.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch

from .binding import GRAD_DTYPES, _check, _stream, lib as _base_lib

GAR_MAX_TOP = 32
# Outputs from which gar_linear_weight_grad takes a workspace by itself: every 256 outputs restore the
# activation once more.
WORKSPACE_OUT = 1024
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
        _typed = True
    return L


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


def _matrix(t: torch.Tensor, name: str, dtype=None, shape=None):
    """(pointer, rows, cols, row stride) of a 2-D CUDA tensor with unit column stride."""
    if not t.is_cuda or t.dtype not in GRAD_DTYPES or (dtype is not None and t.dtype != dtype):
        raise TypeError(f"{name} must be a CUDA {dtype or 'float32, bfloat16 or float16'} tensor")
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be 2-D with unit column stride")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}")
    rows, cols = t.shape
    return t.data_ptr() or 16, rows, cols, t.stride(0) if rows > 1 else cols


def _vector(t: Optional[torch.Tensor], name: str, dtype, numel: int, device):
    """Pointer of a contiguous CUDA tensor of `numel` elements (None stays None)."""
    if t is None:
        return None
    if not (t.is_cuda and t.device == device and t.dtype == dtype and t.is_contiguous() and t.numel() == numel):
        raise TypeError(f"{name} must be a contiguous {dtype} tensor of {numel} elements on {device}")
    return t.data_ptr()


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} must sit on {device}")


def _new_checkpoint(rows: int, cols: int, group: int, like: torch.Tensor) -> Checkpoint:
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    q = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device=like.device)
    return Checkpoint(q, torch.empty(rows, -(-cols // group), dtype=torch.float32, device=like.device), cols, group, like.dtype)


def _saved(ck: Optional[Checkpoint], name: str, device, rows: int, cols: int) -> GarCheckpoint:
    s = GarCheckpoint()
    if ck is None:
        return s
    if ck.cols != cols or ck.q.dim() != 2 or ck.q.shape[0] != rows or ck.q.shape[1] < cols:
        raise ValueError(f"{name} does not hold [{rows}, {cols}]")
    if not (ck.q.device == device and ck.q.dtype == torch.int8 and ck.q.stride(1) == 1):
        raise TypeError(f"{name}.q must be an int8 tensor with unit column stride on {device}")
    s.scales = _vector(ck.scales, f"{name}.scales", torch.float32, rows * -(-cols // ck.group), device)
    s.q, s.ldq = ck.q.data_ptr(), ck.q.stride(0) if rows > 1 else ck.q.shape[1]
    if rows == 0:
        s.q = s.scales = 16
    return s


def gar_token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 0, stream=None) -> TokenLogprobs:
    """gar_token_logprobs: logits [rows, vocab], targets int64 [rows] (negative: none)."""
    ptr, rows, vocab, ld = _matrix(logits, "logits")
    dev = logits.device
    f32 = dict(dtype=torch.float32, device=dev)
    r = TokenLogprobs(torch.empty(rows, **f32) if targets is not None else None, torch.empty(rows, **f32),
                      torch.empty(rows, **f32), torch.empty(rows, top, **f32) if top > 0 else None,
                      torch.empty(rows, top, dtype=torch.int64, device=dev) if top > 0 else None, torch.empty(rows, **f32))
    p = GarLogprobsParams()
    p.dtype, p.top, p.rows, p.vocab, p.ld, p.logits = GRAD_DTYPES[logits.dtype], top, rows, vocab, ld, ptr
    p.targets = _vector(targets, "targets", torch.int64, rows, dev)
    p.entropy, p.lse = r.entropy.data_ptr() or 16, r.lse.data_ptr() or 16
    p.lse_lo = r.lse_lo.data_ptr()
    p.logprobs = r.logprobs.data_ptr() if targets is not None else None
    if top > 0:
        p.top_logprobs, p.top_index = r.top_logprobs.data_ptr() or 16, r.top_index.data_ptr() or 16
    with torch.cuda.device(dev):
        p.stream = _stream(stream)
        st = lib().gar_token_logprobs(C.byref(p))
    _check(st, "gar_token_logprobs")
    return r


def gar_token_logprobs_backward(logits: torch.Tensor, saved: TokenLogprobs, targets: Optional[torch.Tensor] = None,
                                grad_logprobs: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None,
                                grad_top: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                                stream=None) -> torch.Tensor:
    """gar_token_logprobs_backward: the gradient at the logits (dlogits may be logits: in place)."""
    ptr, rows, vocab, ld = _matrix(logits, "logits")
    dev = logits.device
    if dlogits is None:
        dlogits = torch.empty(rows, vocab, dtype=logits.dtype, device=dev)
    p = GarLogprobsGradParams()
    p.dtype, p.rows, p.vocab, p.ld, p.logits = GRAD_DTYPES[logits.dtype], rows, vocab, ld, ptr
    p.dlogits, _, _, p.ld_dlogits = _matrix(dlogits, "dlogits", logits.dtype, (rows, vocab))
    _same_device(dev, dlogits=dlogits)
    p.lse = _vector(saved.lse, "saved.lse", torch.float32, rows, dev) or 16
    p.lse_lo = _vector(saved.lse_lo, "saved.lse_lo", torch.float32, rows, dev)
    p.targets = _vector(targets, "targets", torch.int64, rows, dev)
    p.grad_logprobs = _vector(grad_logprobs, "grad_logprobs", torch.float32, rows, dev)
    p.grad_entropy = _vector(grad_entropy, "grad_entropy", torch.float32, rows, dev)
    if grad_entropy is not None:
        p.entropy = _vector(saved.entropy, "saved.entropy", torch.float32, rows, dev)
    if grad_top is not None:
        if saved.top_index is None:
            raise ValueError("grad_top needs the saved top_index")
        p.top = saved.top_index.shape[1]
        p.top_index = _vector(saved.top_index, "saved.top_index", torch.int64, rows * p.top, dev) or 16
        p.grad_top = _vector(grad_top, "grad_top", torch.float32, rows * p.top, dev) or 16
    with torch.cuda.device(dev):
        p.stream = _stream(stream)
        st = lib().gar_token_logprobs_backward(C.byref(p))
    _check(st, "gar_token_logprobs_backward")
    return dlogits


def gar_checkpoint_pack(x: torch.Tensor, group: int = 128, stream=None) -> Checkpoint:
    """gar_checkpoint_pack: x [rows, cols] in 8 bits."""
    ptr, rows, cols, ld = _matrix(x, "x")
    ck = _new_checkpoint(rows, cols, group, x)
    s = _saved(ck, "checkpoint", x.device, rows, cols)
    with torch.cuda.device(x.device):
        st = lib().gar_checkpoint_pack(GRAD_DTYPES[x.dtype], ptr, rows, cols, ld, group, C.byref(s), _stream(stream))
    _check(st, "gar_checkpoint_pack")
    return ck


def gar_checkpoint_unpack(saved: Checkpoint, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """gar_checkpoint_unpack: the restored activation [rows, cols]."""
    rows, dev = saved.q.shape[0], saved.q.device
    if out is None:
        out = torch.empty(rows, saved.cols, dtype=saved.dtype, device=dev)
    ptr, _, _, ld = _matrix(out, "out", saved.dtype, (rows, saved.cols))
    _same_device(dev, out=out)
    s = _saved(saved, "saved", dev, rows, saved.cols)
    with torch.cuda.device(dev):
        st = lib().gar_checkpoint_unpack(GRAD_DTYPES[saved.dtype], C.byref(s), rows, saved.cols, saved.group, ptr, ld,
                                         _stream(stream))
    _check(st, "gar_checkpoint_unpack")
    return out


def gar_activation_forward(act: str, x: torch.Tensor, up: Optional[torch.Tensor] = None, group: int = 128,
                           save_input: bool = True, save_output: bool = False, y: Optional[torch.Tensor] = None,
                           stream=None) -> Activation:
    """gar_activation_forward: y = act(x) (* up), with the checkpoints of the inputs and / or the output."""
    ptr, rows, cols, ld = _matrix(x, "x")
    dev = x.device
    p = GarActivationParams()
    p.dtype, p.act, p.group, p.rows, p.cols = GRAD_DTYPES[x.dtype], ACTIVATIONS[act], group, rows, cols
    p.x, p.ldx = ptr, ld
    if up is not None:
        p.up, _, _, p.ldup = _matrix(up, "up", x.dtype, (rows, cols))
    if y is None:
        y = torch.empty(rows, cols, dtype=x.dtype, device=dev)
    p.y, _, _, p.ldy = _matrix(y, "y", x.dtype, (rows, cols))
    _same_device(dev, up=up, y=y)
    r = Activation(y, _new_checkpoint(rows, cols, group, x) if save_input else None,
                   _new_checkpoint(rows, cols, group, x) if save_input and up is not None else None,
                   _new_checkpoint(rows, cols, group, x) if save_output else None)
    p.x_saved = _saved(r.x, "x", dev, rows, cols)
    p.up_saved = _saved(r.up, "up", dev, rows, cols)
    p.y_saved = _saved(r.out, "out", dev, rows, cols)
    with torch.cuda.device(dev):
        p.stream = _stream(stream)
        st = lib().gar_activation_forward(C.byref(p))
    _check(st, "gar_activation_forward")
    return r


def gar_activation_backward(act: str, dy: torch.Tensor, x: Checkpoint, up: Optional[Checkpoint] = None,
                            dx: Optional[torch.Tensor] = None, dup: Optional[torch.Tensor] = None,
                            stream=None) -> ActivationGrad:
    """gar_activation_backward: gradients at x (and up) from the checkpoints (dx may be dy: in place)."""
    ptr, rows, cols, ld = _matrix(dy, "dy", x.dtype)
    dev = dy.device
    if up is not None and (up.group != x.group or up.dtype != x.dtype):
        raise ValueError("both checkpoints must have the same group and type")
    p = GarActivationGradParams()
    p.dtype, p.act, p.group, p.rows, p.cols = GRAD_DTYPES[dy.dtype], ACTIVATIONS[act], x.group, rows, cols
    p.dy, p.lddy = ptr, ld
    p.x_saved, p.up_saved = _saved(x, "x", dev, rows, cols), _saved(up, "up", dev, rows, cols)
    if dx is None:
        dx = torch.empty(rows, cols, dtype=dy.dtype, device=dev)
    p.dx, _, _, p.lddx = _matrix(dx, "dx", dy.dtype, (rows, cols))
    if up is not None:
        if dup is None:
            dup = torch.empty(rows, cols, dtype=dy.dtype, device=dev)
        p.dup, _, _, p.lddup = _matrix(dup, "dup", dy.dtype, (rows, cols))
    elif dup is not None:
        raise ValueError("dup needs up")
    _same_device(dev, dx=dx, dup=dup)
    with torch.cuda.device(dev):
        p.stream = _stream(stream)
        st = lib().gar_activation_backward(C.byref(p))
    _check(st, "gar_activation_backward")
    return ActivationGrad(dx, dup)


def _weight_grad_params(dy: torch.Tensor, x: Checkpoint) -> GarWeightGradParams:
    if dy.dim() != 3 or not dy.is_cuda or dy.dtype not in GRAD_DTYPES or (dy.shape[2] > 1 and dy.stride(2) != 1):
        raise ValueError("dy must be a CUDA tensor [workers, tokens, out] with unit column stride")
    workers, tokens, out = dy.shape
    ld_dy = dy.stride(1) if tokens > 1 else dy.stride(0) if workers > 1 else out
    if workers > 1 and tokens > 1 and dy.stride(0) != tokens * ld_dy:
        raise ValueError("dy: the workers' tokens must be evenly spaced rows")
    if dy.dtype != x.dtype:
        raise TypeError("dy and the checkpoint must be of one type")
    p = GarWeightGradParams()
    p.dtype, p.group, p.workers = GRAD_DTYPES[dy.dtype], x.group, workers
    p.tokens, p.out_features, p.in_features = tokens, out, x.cols
    p.dy, p.ld_dy = dy.data_ptr() or 16, ld_dy
    return p


def gar_weight_grad_workspace_bytes(dy: torch.Tensor, x: Checkpoint) -> int:
    """Bytes of the workspace gar_linear_weight_grad takes for these operands."""
    return lib().gar_weight_grad_workspace_bytes(C.byref(_weight_grad_params(dy, x)))


def gar_linear_weight_grad(dy: torch.Tensor, x: Checkpoint, grads: Optional[torch.Tensor] = None, weight_offset: int = 0,
                           bias_offset: Optional[int] = None, lengths: Optional[torch.Tensor] = None,
                           grads_dtype: torch.dtype = torch.float32, workspace=None, stream=None) -> torch.Tensor:
    """gar_linear_weight_grad: dy [workers, tokens, out] and the checkpoint of x [workers * tokens, in]
    into the gradient block `grads` [workers, d]: row w gets dW_w (out x in, row-major) from column
    weight_offset on and, with bias_offset, db_w from there on.  lengths int32 [workers]: tokens that
    count.  Without `grads` a block [workers, out * in] of grads_dtype is made.  workspace: None lets the
    call allocate one for layers where it is faster, False never (the codes are then restored tile by
    tile), or a uint8 CUDA tensor of gar_weight_grad_workspace_bytes."""
    p = _weight_grad_params(dy, x)
    workers, tokens, out = dy.shape
    dev = dy.device
    if grads is None:
        if weight_offset != 0 or bias_offset is not None:
            raise ValueError("offsets need `grads`")
        grads = torch.empty(workers, out * x.cols, dtype=grads_dtype, device=dev)
    ptr, n, d, ld = _matrix(grads, "grads")
    _same_device(dev, grads=grads)
    if n != workers or weight_offset < 0 or weight_offset + out * x.cols > d:
        raise ValueError("grads must have a row per worker and room for the weights at weight_offset")
    if bias_offset is not None and (bias_offset < 0 or bias_offset + out > d):
        raise ValueError("grads has no room for the bias at bias_offset")
    p.grads_dtype = GRAD_DTYPES[grads.dtype]
    p.x_saved = _saved(x, "x", dev, workers * tokens, x.cols)
    p.lengths = _vector(lengths, "lengths", torch.int32, workers, dev)
    p.weight_grads, p.ld_grads = ptr + weight_offset * grads.element_size(), ld
    p.bias_grads = ptr + bias_offset * grads.element_size() if bias_offset is not None else None
    if workspace is None and out > WORKSPACE_OUT:
        workspace = torch.empty(lib().gar_weight_grad_workspace_bytes(C.byref(p)), dtype=torch.uint8, device=dev)
    if workspace is not None and workspace is not False:
        p.workspace, p.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    with torch.cuda.device(dev):
        p.stream = _stream(stream)
        st = lib().gar_linear_weight_grad(C.byref(p))
    _check(st, "gar_linear_weight_grad")
    return grads
