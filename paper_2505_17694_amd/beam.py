"""Beam search around a decode step: choosing continuations, moving the beams' states (marshalling only)."""
from __future__ import annotations

import torch

from . import binding as B
from .cache import _enter, _on

_CODE = {torch.float16: B.CODEC_DTYPE_FP16, torch.bfloat16: B.CODEC_DTYPE_BF16, torch.float32: B.CODEC_DTYPE_FP32}


def _reach(t: torch.Tensor) -> int:
    """Elements from the first of a tensor to behind its last."""
    return 1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())) if t.numel() else 0


def _check_storage(t: torch.Tensor, what: str) -> None:
    """A tensor keeps its shape when its storage is given back: the memory behind it is what counts."""
    if t.untyped_storage().nbytes() // t.element_size() - t.storage_offset() < _reach(t):
        raise ValueError(f"{what}: the tensor's storage ends before its last element")


def _dense(t: torch.Tensor, what: str, shape, dtypes, device: torch.device) -> int:
    if t.shape != shape or t.dtype not in dtypes or t.device != device or not t.is_contiguous():
        raise ValueError(f"{what}: need a contiguous tensor of shape {tuple(shape)}, one of {dtypes}, on {device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    _check_storage(t, what)
    return t.data_ptr()


def beam_select(logits: torch.Tensor, scores: torch.Tensor, k: int, finished: torch.Tensor = None, eos: int = 0, stream=None):
    """The k best continuations of every search: logits [batch, beams, vocab] (16 or 32 bits), scores [batch, beams] (32 bits),
    ``finished`` [batch, beams] (truth values) beams go on with ``eos`` alone.  Returns (scores, beams, tokens), each
    [batch, k], best first; ties go to the lowest beam, then the lowest token (see codec_beam_select)."""
    if logits.dim() != 3 or logits.dtype not in _CODE or logits.device.type != "cuda":
        raise ValueError(f"logits: need [batch, beams, vocab] of 16 or 32 bits on a GPU, got {logits.dtype} {tuple(logits.shape)} on {logits.device}")
    s = _enter(logits.device, stream)
    if s is None:
        with _on(logits.device, stream) as s:
            return _select(logits, scores, k, finished, eos, s)
    return _select(logits, scores, k, finished, eos, s)


def _select(logits, scores, k, finished, eos, s):
    device, (batch, beams, vocab) = logits.device, logits.shape
    if vocab > 1 and logits.stride(2) != 1:
        raise ValueError(f"logits: the tokens of a beam must be contiguous, strides are {logits.stride()}")
    _check_storage(logits, "logits")
    config = B.codec_beam_config(batch, beams, vocab, k, _CODE[logits.dtype], eos)
    scores_at = _dense(scores, "scores", (batch, beams), (torch.float32,), device)
    finished_at = None if finished is None else _dense(finished, "finished", (batch, beams), (torch.bool, torch.uint8), device)
    need = B.codec_beam_workspace_bytes(config)
    rows = max(0, k)
    out_scores = torch.empty((batch, rows), dtype=torch.float32, device=device)
    picked = torch.empty((2, batch, rows), dtype=torch.int32, device=device)
    workspace = torch.empty(need, dtype=torch.uint8, device=device)
    at = picked.data_ptr()
    st = B.codec_beam_select(config, logits.data_ptr(), logits.stride(0) if batch > 1 else 0, logits.stride(1) if beams > 1 else 0,
                             scores_at, finished_at, out_scores.data_ptr(), at, at + 4 * batch * rows, workspace.data_ptr(), need, s)
    if st != B.CODEC_OK:
        raise B.CodecError(st, "codec_beam_select")
    return out_scores, picked[0], picked[1]


def beam_reorder(states, beams: torch.Tensor, out=None, stream=None):
    """The states of the beams that go on: of every tensor [batch, beams, ...] in ``states`` the rows ``beams`` [batch, n]
    (int32) names, as new tensors [batch, n, ...] or in those of ``out``.  Rows have to be contiguous.  A row whose entry is no
    beam is left as it was (in a new tensor: undefined)."""
    states = list(states)
    if beams.dim() != 2 or beams.device.type != "cuda":
        raise ValueError(f"beams: need [batch, n] on a GPU, got {tuple(beams.shape)} on {beams.device}")
    s = _enter(beams.device, stream)
    if s is None:
        with _on(beams.device, stream) as s:
            return _reorder(states, beams, out, s)
    return _reorder(states, beams, out, s)


def _state_row(t: torch.Tensor, what: str) -> None:
    n = 1
    for size, stride in zip(reversed(t.shape[2:]), reversed(t.stride()[2:])):
        if size != 1 and stride != n:
            raise ValueError(f"{what}: the row of a beam must be contiguous, strides are {t.stride()}")
        n *= size
    _check_storage(t, what)


def _reorder(states, beams, out, s):
    batch, n = beams.shape
    device = beams.device
    beams_at = _dense(beams, "beams", (batch, n), (torch.int32,), device)
    if out is None:
        out = [torch.empty((batch, n, *x.shape[2:]), dtype=x.dtype, device=device) for x in states]
    if len(out) != len(states):
        raise ValueError(f"out: {len(out)} tensors for {len(states)} states")
    wide = states[0].shape[1] if states and states[0].dim() >= 2 else 1
    items = []
    for i, (x, y) in enumerate(zip(states, out)):
        if x.dim() < 2 or x.shape[:2] != (batch, wide) or x.device != device:
            raise ValueError(f"states[{i}]: need [{batch}, {wide}, ...] on {device}, got {tuple(x.shape)} on {x.device}")
        if y.shape != (batch, n, *x.shape[2:]) or y.dtype != x.dtype or y.device != device:
            raise ValueError(f"out[{i}]: need {x.dtype} [{batch}, {n}, ...] like states[{i}] on {device}, got {y.dtype} {tuple(y.shape)} on {y.device}")
        if not x.is_contiguous():
            _state_row(x, f"states[{i}]")
        else:
            _check_storage(x, f"states[{i}]")
        if not y.is_contiguous():
            _state_row(y, f"out[{i}]")
        else:
            _check_storage(y, f"out[{i}]")
        size = x.element_size()
        row = size * (x.numel() // (batch * wide)) if batch * wide else 0
        items.append(B.codec_state(x.data_ptr(), y.data_ptr(), row, size * x.stride(0), size * x.stride(1), size * y.stride(0),
                                   size * y.stride(1)))
    if n and wide:
        st = B.codec_beam_reorder(items, beams_at, batch, wide, n, s)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_beam_reorder")
    return out
