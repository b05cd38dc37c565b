"""ctypes binding of the beam search's entry points (include/sip_beam.h), with torch tensors standing in for device pointers.
Argument marshalling only; there is no fallback.  ``stream`` as in head.py."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import binding
from .binding import _empty, _nbytes, _ptr
from .head import _DTYPES, _call, _matrix, _same_device, _scratch, _vector

SIP_MAX_BEAMS = 64
SIP_MAX_CONTINUATIONS = 128

_p, _i, _l, _f, _z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t

_SIGNATURES = {
    "sip_beam_workspace_bytes": (_z, [_i, _i, _i, _i]),
    "sip_beam_select": (ctypes.c_int, [_p, _i, _i, _i, _l, ctypes.c_int, _f, _p, _p, _i, _p, _i, _p, _p, _p, _p, _z, _p]),
    "sip_state_reorder": (ctypes.c_int, [_p, _z, _i, _i, _i, _i, _p, _p, _p, _p]),
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


def sip_beam_workspace_bytes(groups: int, width: int, V: int, n: int) -> int:
    return int(_load().sip_beam_workspace_bytes(groups, width, V, n))


def sip_beam_select(logits: torch.Tensor, scores: torch.Tensor, width: int, n: Optional[int] = None, *,
                    finished: Optional[torch.Tensor] = None, rank_scale: Optional[torch.Tensor] = None,
                    end_token: Optional[int] = None, logit_scale: float = 1.0, tokens: Optional[torch.Tensor] = None,
                    parents: Optional[torch.Tensor] = None, out_scores: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                    ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(tokens, parents, scores), each [groups, n] in descending order: the ``n`` (default: ``width``) best continuations of every
    group of ``width`` beams, from ``logits`` [groups * width, V] (float32 or bfloat16) and the beams' ``scores`` so far (float32,
    -inf = no such beam).  ``finished`` (uint8 or bool): those beams go on at no cost with ``end_token`` alone, which has to be given
    then.  ``rank_scale`` (float32, > 0): what totals are multiplied with for comparison.  Missing continuations are token -1, parent -1,
    score -inf."""
    lib = _load()
    _matrix(logits, "logits", (torch.bfloat16, torch.float32))
    (R, V), dev = logits.shape, logits.device
    if width <= 0 or R % width != 0:
        raise TypeError(f"{R} rows of logits are no whole number of groups of {width} beams")
    groups, n = R // width, width if n is None else n
    _vector(scores, "scores", torch.float32, R)
    if finished is not None:
        if end_token is None:
            raise TypeError("finished beams go on with end_token: it has to be given")
        _vector(finished, "finished", torch.bool if finished.dtype == torch.bool else torch.uint8, R)
    if rank_scale is not None:
        _vector(rank_scale, "rank_scale", torch.float32, R)

    def out(t, name, dtype):
        if t is None:
            return _empty(stream, groups, n, dtype=dtype, device=dev)
        return _vector(t, name, dtype, groups * n)

    tokens, parents = out(tokens, "tokens", torch.int32), out(parents, "parents", torch.int32)
    out_scores = out(out_scores, "out_scores", torch.float32)
    _same_device(dev, scores, finished, rank_scale, tokens, parents, out_scores)
    if R == 0:
        return tokens, parents, out_scores
    ws = _scratch(workspace, 0 if workspace is not None else lib.sip_beam_workspace_bytes(groups, width, V, n), dev, stream)
    stride = logits.stride(0) if R > 1 else (V + 7) // 8 * 8                 # (that of a single row says nothing)
    _call("sip_beam_select", dev, stream, _ptr(logits), groups, width, V, stride, _DTYPES[logits.dtype], logit_scale,
          _ptr(scores), _ptr(finished), 0 if end_token is None else end_token, _ptr(rank_scale), n, _ptr(tokens), _ptr(parents),
          _ptr(out_scores), _ptr(ws), _nbytes(ws))
    return tokens, parents, out_scores


def sip_state_reorder(state: torch.Tensor, slots: int, L_max: int, slot_of_row: torch.Tensor, parents: torch.Tensor, width: int,
                      tokens: Optional[torch.Tensor] = None, *, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Row r's slot takes the history of its parent, beam ``parents[r]`` of the row's group of ``width``, and ``tokens[r]`` behind
    it: what sip_beam_select() of ``width`` continuations returned goes in as it is.  In place, all rows at once."""
    if not state.is_cuda or state.dtype != torch.uint8 or not state.is_contiguous():
        raise TypeError("state must be a contiguous device tensor of bytes")
    R = slot_of_row.numel()
    if width <= 0 or R % width != 0:
        raise TypeError(f"{R} rows are no whole number of groups of {width} beams")
    _vector(slot_of_row, "slot_of_row", torch.int32, R)
    _vector(parents, "parents", torch.int32, R)
    if tokens is not None:
        _vector(tokens, "tokens", torch.int32, R)
    _same_device(state.device, slot_of_row, parents, tokens)
    _load()
    _call("sip_state_reorder", state.device, stream, _ptr(state), _nbytes(state), slots, L_max, R // width, width,
          _ptr(slot_of_row), _ptr(parents), _ptr(tokens))
