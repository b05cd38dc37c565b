"""ctypes binding of the vocabulary head's entry points (include/sip_head.h), with torch tensors standing in for device
pointers.  Argument marshalling only; there is no fallback.

A call runs on ``stream`` (default: torch's current stream).  The outputs and the scratch memory that it allocates because they
were not supplied belong to that stream, as under ``torch.cuda.stream(stream)``.  The calls are no operations of torch's: a tensor that
requires a gradient is read like any other, and nothing is recorded; gradients are what sip_xent_backward returns."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple

import torch

from . import binding
from .binding import SIP_BF16, SIP_F32, SIP_OK, SipError, _empty, _nbytes, _on, _ptr, _stream_handle

SIP_MAX_D = 16384
SIP_MAX_TOKENS = 65536
SIP_MAX_TENSORS = 65536

_DTYPES = {torch.float32: SIP_F32, torch.bfloat16: SIP_BF16}
_p, _i, _l, _f, _z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


class SipGrad(ctypes.Structure):
    """sip_grad of include/sip_head.h, field for field."""
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64), ("dtype", ctypes.c_int)]


_SIGNATURES = {
    "sip_xent_workspace_bytes": (_z, [_i, _i, _i, _i]),
    "sip_xent_forward": (ctypes.c_int, [_p, _i, _i, _l, _p, _i, _l, _p, _f, _p, _p, _p, _z, _p]),
    "sip_xent_backward": (ctypes.c_int, [_p, _i, _i, _l, _p, _i, _l, _p, _f, _p, _p, _p, _f, _p, _l, _p, _l, _p, _z, _p]),
    "sip_grad_clip_workspace_bytes": (_z, [_i]),
    "sip_grad_clip": (ctypes.c_int, [ctypes.POINTER(SipGrad), _i, _f, _f, _p, _p, _z, _p]),
    "sip_head_quantize": (ctypes.c_int, [_p, _i, _i, _l, _i, _p, _l, _p, ctypes.c_int, _p, _p]),
    "sip_head_workspace_bytes": (_z, [_i, _i, _i, _i]),
    "sip_head_logits": (ctypes.c_int, [_p, _i, _i, _l, ctypes.c_int, _p, _l, _p, ctypes.c_int, _p, _i, _i, _p, _l,
                                       ctypes.c_int, _p, _z, _p]),
}
_ready = None


def _load() -> ctypes.CDLL:
    global _ready
    lib = binding.load()
    if _ready is not lib:
        for name, (restype, argtypes) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = restype, argtypes
        _ready = lib
    return lib


def _call(name: str, dev: torch.device, stream: Optional[torch.cuda.Stream], *args) -> None:
    """The library's ``name`` on ``stream`` (its last argument), with the tensors' device as the current one: a device's default
    stream is that of whichever is current."""
    fn = getattr(_load(), name)
    if dev.index == torch.cuda.current_device():
        status = fn(*args, _stream_handle(dev, stream))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _stream_handle(dev, stream))
    if status != SIP_OK:
        raise SipError(status, name)


def _matrix(t: torch.Tensor, name: str, dtypes, shape=None) -> torch.Tensor:
    if not t.is_cuda or t.dim() != 2 or t.stride(1) != 1 or t.dtype not in dtypes:
        raise TypeError(f"{name} must be a 2-D device tensor with contiguous rows of {' or '.join(map(str, dtypes))}")
    if shape is not None and tuple(t.shape) != shape:
        raise TypeError(f"{name} must be {shape}, got {tuple(t.shape)}")
    return t


def _vector(t: torch.Tensor, name: str, dtype, n: int) -> torch.Tensor:
    if not t.is_cuda or t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous device tensor of {n} x {dtype}")
    return t


def _same_device(device: torch.device, *tensors: Optional[torch.Tensor]) -> None:
    for t in tensors:
        if t is not None and t.device != device:
            raise TypeError(f"tensors of one call must be on one device: {device} and {t.device}")


def _stride(t: torch.Tensor) -> int:
    """Row stride; that of a single row says nothing, and its width serves."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _scratch(workspace: Optional[torch.Tensor], need: int, dev, stream) -> torch.Tensor:
    if workspace is None:
        return _empty(stream, max(need, 256), dtype=torch.uint8, device=dev)
    _same_device(dev, workspace)
    if not workspace.is_contiguous():
        raise TypeError("a workspace must be contiguous")
    return workspace


# ---- cross entropy

def sip_xent_workspace_bytes(N: int, V: int, D: int, backward: bool) -> int:
    return int(_load().sip_xent_workspace_bytes(N, V, D, int(backward)))


def _xent_operands(hidden, weight, targets):
    _matrix(hidden, "hidden", (torch.bfloat16,))
    _matrix(weight, "weight", (torch.bfloat16,))
    if hidden.shape[1] != weight.shape[1]:
        raise TypeError(f"hidden [N, D] and weight [V, D] differ in D: {hidden.shape[1]} and {weight.shape[1]}")
    _vector(targets, "targets", torch.int32, hidden.shape[0])
    _same_device(hidden.device, weight, targets)
    return hidden.shape[0], weight.shape[0], hidden.shape[1]


def sip_xent_forward(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, logit_scale: float = 1.0, *,
                     loss: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                     ) -> Tuple[torch.Tensor, torch.Tensor]:
    """(loss [N], lse [N]): the negative log-probability of each target under the head and the log-sum-exp of its
    logits.  ``hidden`` [N, D] and ``weight`` [V, D] are bf16, ``targets`` int32; a target outside [0, V) masks its row."""
    lib = _load()
    N, V, D = _xent_operands(hidden, weight, targets)
    dev = hidden.device
    loss = _empty(stream, N, dtype=torch.float32, device=dev) if loss is None else _vector(loss, "loss", torch.float32, N)
    lse = _empty(stream, N, dtype=torch.float32, device=dev) if lse is None else _vector(lse, "lse", torch.float32, N)
    _same_device(dev, loss, lse)
    if N == 0:
        return loss, lse
    ws = _scratch(workspace, 0 if workspace is not None else lib.sip_xent_workspace_bytes(N, V, D, 0), dev, stream)
    _call("sip_xent_forward", dev, stream, _ptr(hidden), N, D, _stride(hidden), _ptr(weight), V, _stride(weight),
          _ptr(targets), logit_scale, _ptr(loss), _ptr(lse), _ptr(ws), _nbytes(ws))
    return loss, lse


def sip_xent_backward(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, loss: torch.Tensor,
                      lse: torch.Tensor, grad_loss: Optional[torch.Tensor] = None, scale: float = 1.0,
                      logit_scale: float = 1.0, *, grad_hidden: Optional[torch.Tensor] = None,
                      grad_weight: Optional[torch.Tensor] = None, want_hidden: bool = True, want_weight: bool = True,
                      workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                      ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(grad_hidden [N, D], grad_weight [V, D]), bf16, of ``scale * sum(grad_loss * loss)`` with ``loss`` and ``lse``
    from sip_xent_forward.  ``want_hidden`` / ``want_weight``: False leaves that one out (None is returned)."""
    lib = _load()
    N, V, D = _xent_operands(hidden, weight, targets)
    dev = hidden.device
    _vector(loss, "loss", torch.float32, N)
    _vector(lse, "lse", torch.float32, N)
    if grad_loss is not None:
        _vector(grad_loss, "grad_loss", torch.float32, N)
    gh = gw = None
    if want_hidden:
        gh = (_empty(stream, N, D, dtype=torch.bfloat16, device=dev) if grad_hidden is None
              else _matrix(grad_hidden, "grad_hidden", (torch.bfloat16,), (N, D)))
    if want_weight:
        gw = (_empty(stream, V, D, dtype=torch.bfloat16, device=dev) if grad_weight is None
              else _matrix(grad_weight, "grad_weight", (torch.bfloat16,), (V, D)))
    _same_device(dev, loss, lse, grad_loss, gh, gw)
    if N == 0:
        if gw is not None:
            with _on(stream):
                gw.zero_()
        return gh, gw
    ws = _scratch(workspace, 0 if workspace is not None else lib.sip_xent_workspace_bytes(N, V, D, 1), dev, stream)
    _call("sip_xent_backward", dev, stream, _ptr(hidden), N, D, _stride(hidden), _ptr(weight), V, _stride(weight),
          _ptr(targets), logit_scale, _ptr(loss), _ptr(lse), _ptr(grad_loss), scale, _ptr(gh),
          0 if gh is None else _stride(gh), _ptr(gw), 0 if gw is None else _stride(gw), _ptr(ws), _nbytes(ws))
    return gh, gw


# ---- gradient norm and clipping

class GradTable:
    """The gradients of a model, and where their clipped values go (``outs``: None = in place): what sip_grad_clip
    reads.  Made once and kept as long as the tensors' memory stays where it is."""

    def __init__(self, grads: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None):
        grads = list(grads)
        outs = grads if outs is None else list(outs)
        if len(outs) != len(grads):
            raise TypeError("as many outputs as gradients are needed")
        self.table = (SipGrad * max(1, len(grads)))()
        self.n, self.device = len(grads), grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
        self.keep = (grads, outs)
        for e, g, o in zip(self.table, grads, outs):
            if g.dtype not in _DTYPES or not g.is_cuda or not g.is_contiguous() or g.device != self.device:
                raise TypeError("gradients must be contiguous float32 or bfloat16 tensors of one device")
            if o.dtype != g.dtype or o.device != g.device or not o.is_contiguous() or o.numel() != g.numel():
                raise TypeError("an output must be contiguous, and of its gradient's type, size and device")
            e.grad, e.out, e.count, e.dtype = g.data_ptr(), o.data_ptr(), g.numel(), _DTYPES[g.dtype]


def sip_grad_clip_workspace_bytes(n_tensors: int) -> int:
    return int(_load().sip_grad_clip_workspace_bytes(n_tensors))


def sip_grad_clip(grads, max_norm: float, *, eps: float = 1e-6, norm: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Scale ``grads`` (a GradTable, or a sequence of tensors: in place) by min(1, max_norm / (norm + eps)); returns
    their 2-norm before that, one float32 on the device."""
    lib = _load()
    t = grads if isinstance(grads, GradTable) else GradTable(grads)
    norm = _empty(stream, (), dtype=torch.float32, device=t.device) if norm is None else _vector(norm, "norm", torch.float32, 1)
    _same_device(t.device, norm)
    ws = _scratch(workspace, 0 if workspace is not None else lib.sip_grad_clip_workspace_bytes(t.n), t.device, stream)
    _call("sip_grad_clip", t.device, stream, t.table, t.n, max_norm, eps, _ptr(norm), _ptr(ws), _nbytes(ws))
    return norm


# ---- 4-bit head

def _codes_operands(codes, scales, zeros):
    _matrix(codes, "codes", (torch.uint8,))
    V, D = codes.shape[0], codes.shape[1] * 2
    if not scales.is_cuda or scales.dim() != 2 or not scales.is_contiguous() or scales.dtype not in _DTYPES or \
            scales.shape[0] != V or scales.shape[1] == 0 or D % scales.shape[1] != 0:
        raise TypeError("scales must be a contiguous device tensor [V, D / group] of float32 or bfloat16")
    if zeros is not None:
        _vector(zeros, "zeros", torch.uint8, scales.numel())
    return V, D, D // scales.shape[1]


def sip_head_quantize(weight: torch.Tensor, group: int = 128, *, use_zeros: bool = True,
                      scales_dtype: torch.dtype = torch.bfloat16, codes: Optional[torch.Tensor] = None,
                      scales: Optional[torch.Tensor] = None, zeros: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None
                      ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """(codes [V, D / 2], scales [V, D / group], zeros or None) of bf16 ``weight`` [V, D].  Outputs are allocated when
    not supplied, ``zeros`` if ``use_zeros``; where both ``codes`` and ``scales`` are, ``zeros`` alone says whether the groups
    have zero points."""
    _matrix(weight, "weight", (torch.bfloat16,))
    V, D = weight.shape
    if group <= 0 or D % group != 0:
        raise TypeError(f"the width {D} is no multiple of the group {group}")
    dev = weight.device
    if zeros is None and use_zeros and (codes is None or scales is None):
        zeros = _empty(stream, V, D // group, dtype=torch.uint8, device=dev)
    if codes is None:
        codes = _empty(stream, V, D // 2, dtype=torch.uint8, device=dev)
    if scales is None:
        scales = _empty(stream, V, D // group, dtype=scales_dtype, device=dev)
    if _codes_operands(codes, scales, zeros) != (V, D, group):
        raise TypeError("codes and scales do not fit the weight and the group")
    _same_device(dev, codes, scales, zeros)
    _call("sip_head_quantize", dev, stream, _ptr(weight), V, D, _stride(weight), group, _ptr(codes), _stride(codes),
          _ptr(scales), _DTYPES[scales.dtype], _ptr(zeros))
    return codes, scales, zeros


def sip_head_workspace_bytes(B: int, V: int, D: int, group: int) -> int:
    return int(_load().sip_head_workspace_bytes(B, V, D, group))


def sip_head_logits(hidden: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                    zeros: Optional[torch.Tensor] = None, *, out: Optional[torch.Tensor] = None,
                    dtype: torch.dtype = torch.float32, workspace: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Logits [B, V] of ``hidden`` [B, D] (bf16 or fp32) under a head of 4-bit codes.  Without ``out`` the rows are laid
    out as sip_sample takes them (their stride whole 16-byte groups), in ``dtype``."""
    lib = _load()
    _matrix(hidden, "hidden", (torch.bfloat16, torch.float32))
    V, D, group = _codes_operands(codes, scales, zeros)
    B, dev = hidden.shape[0], hidden.device
    if hidden.shape[1] != D:
        raise TypeError(f"hidden [B, D] and codes [V, D / 2] differ in D: {hidden.shape[1]} and {D}")
    if out is None:
        out = _empty(stream, B, (V + 7) // 8 * 8, dtype=dtype, device=dev)[:, :V]
    _matrix(out, "out", (torch.bfloat16, torch.float32), (B, V))
    _same_device(dev, codes, scales, zeros, out)
    if B == 0:
        return out
    ws = _scratch(workspace, 0 if workspace is not None else lib.sip_head_workspace_bytes(B, V, D, group), dev, stream)
    _call("sip_head_logits", dev, stream, _ptr(hidden), B, D, _stride(hidden), _DTYPES[hidden.dtype], _ptr(codes),
          _stride(codes), _ptr(scales), _DTYPES[scales.dtype], _ptr(zeros), group, V, _ptr(out), _stride(out),
          _DTYPES[out.dtype], _ptr(ws), _nbytes(ws))
    return out
