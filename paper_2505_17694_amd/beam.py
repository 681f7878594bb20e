"""Beam search around a decode step: choosing continuations, moving the beams' states (marshalling only)."""
from __future__ import annotations

import torch

from . import binding as B
from .cache import _check_reach, _enter, _on

_is_conj, _is_neg = torch.Tensor.is_conj, torch.Tensor.is_neg
_CODE = {torch.float16: B.CODEC_DTYPE_FP16, torch.bfloat16: B.CODEC_DTYPE_BF16, torch.float32: B.CODEC_DTYPE_FP32}


def _dense(t: torch.Tensor, what: str, rows: int, columns: int, dtypes, index: int) -> int:
    shape = t.shape
    if len(shape) != 2 or shape[0] != rows or shape[1] != columns or t.dtype not in dtypes or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{what}: need a contiguous tensor of shape {(rows, columns)}, one of {dtypes}, on cuda:{index}, "
                         f"got {t.dtype} {tuple(shape)} on {t.device}")
    _check_reach(t, what, rows * columns, t.element_size())
    return t.data_ptr()


_SCORES, _FLAGS, _BEAMS = (torch.float32,), (torch.bool, torch.uint8), (torch.int32,)


def beam_select(logits: torch.Tensor, scores: torch.Tensor, k: int, finished: torch.Tensor = None, eos: int = 0, stream=None):
    """The k best continuations of every search: logits [batch, beams, vocab] (16 or 32 bits), scores [batch, beams] (32 bits),
    ``finished`` [batch, beams] (truth values) beams go on with ``eos`` alone.  Returns (scores, beams, tokens), each
    [batch, k], best first; ties go to the lowest beam, then the lowest token (see codec_beam_select).  The three share one
    allocation (to keep one of them for long, clone it) and have no gradient."""
    if logits.dim() != 3 or logits.dtype not in _CODE or not logits.is_cuda:
        raise ValueError(f"logits: need [batch, beams, vocab] of 16 or 32 bits on a GPU, got {logits.dtype} {tuple(logits.shape)} on {logits.device}")
    s = _enter(logits.get_device(), stream)
    if s is None:
        with _on(logits.device, stream) as s:
            return _select(logits, scores, k, finished, eos, s)
    return _select(logits, scores, k, finished, eos, s)


def _select(logits, scores, k, finished, eos, s):
    batch, beams, vocab = logits.shape
    strides, index = logits.stride(), logits.get_device()
    if logits.is_neg() or scores.is_neg():
        raise ValueError("logits or scores: a view that is negated when it is read (see torch.Tensor.resolve_neg)")
    if vocab > 1 and strides[2] != 1:
        raise ValueError(f"logits: the tokens of a beam must be contiguous, strides are {strides}")
    if batch and beams and vocab:
        _check_reach(logits, "logits", (batch - 1) * strides[0] + (beams - 1) * strides[1] + vocab, logits.element_size())
    if (batch | beams | vocab | abs(k) | abs(eos)) >> 31:
        raise ValueError(f"batch {batch}, beams {beams}, vocab {vocab}, k {k}, eos {eos}: one of them is out of range")
    config = B.codec_beam_config(batch, beams, vocab, k, _CODE[logits.dtype], eos)
    scores_at = _dense(scores, "scores", batch, beams, _SCORES, index)
    finished_at = None if finished is None else _dense(finished, "finished", batch, beams, _FLAGS, index)
    need = B.codec_beam_workspace_bytes(config)
    rows = k if need else 0                 # 0: a configuration that the call refuses
    out = logits.new_empty((3, batch, rows), dtype=torch.int32)
    workspace = logits.new_empty((need,), dtype=torch.uint8)
    at, size = out.data_ptr(), 4 * batch * rows
    st = B.codec_beam_select(config, logits.data_ptr(), strides[0] if batch > 1 else 0, strides[1] if beams > 1 else 0, scores_at,
                             finished_at, at, at + size, at + 2 * size, workspace.data_ptr(), need, s)
    if st != B.CODEC_OK:
        raise B.CodecError(st, "codec_beam_select")
    out_scores, out_beams, out_tokens = out.unbind(0)
    return out_scores.view(torch.float32), out_beams, out_tokens


def beam_reorder(states, beams: torch.Tensor, out=None, stream=None):
    """The states of the beams that go on: of every tensor [batch, beams, ...] in ``states`` the rows ``beams`` [batch, n]
    (int32) names, as new tensors [batch, n, ...] or in those of ``out`` (memory apart from the states, from ``beams`` and from
    one another).  Rows have to be contiguous.  A row whose entry is no
    beam is left as it was (in a new tensor: undefined).  New tensors of neighbouring states of one shape and type share an
    allocation, which lives as long as one of them: to keep one for long, or to save it alone, clone it.  Bytes are moved: the new
    tensors have no gradient."""
    states = list(states)
    if beams.dim() != 2 or not beams.is_cuda:
        raise ValueError(f"beams: need [batch, n] on a GPU, got {tuple(beams.shape)} on {beams.device}")
    s = _enter(beams.get_device(), stream)
    if s is None:
        with _on(beams.device, stream) as s:
            return _reorder(states, beams, out, s)
    return _reorder(states, beams, out, s)


def _state(t: torch.Tensor, what: str, i: int, batch: int, beams: int, index: int):
    """Checks [batch, beams, ...] with contiguous rows in storage that is there; (bytes of a row, strides in bytes)."""
    shape, size = t.shape, t.element_size()
    if len(shape) < 2 or shape[0] != batch or shape[1] != beams or t.get_device() != index:
        raise ValueError(f"{what}[{i}]: need [{batch}, {beams}, ...] on cuda:{index}, got {tuple(shape)} on {t.device}")
    if t.is_contiguous():
        count = t.numel()
        if count == 0:
            return 0, 0, 0
        _check_reach(t, what, count, size)
        row = count * size // (batch * beams)
        return row, beams * row, row
    row, strides = 1, t.stride()
    for n, stride in zip(shape[:1:-1], strides[:1:-1]):
        if n != 1 and stride != row:
            raise ValueError(f"{what}[{i}]: the row of a beam must be contiguous, strides are {strides}")
        row *= n
    if row:
        _check_reach(t, what, (batch - 1) * strides[0] + (beams - 1) * strides[1] + row, size)
    return row * size, strides[0] * size, strides[1] * size


def _states(tensors, what: str, batch: int, beams: int, index: int):
    """_state of each; a dense tensor like the one before it is only looked at for what may differ."""
    if any(map(_is_conj, tensors)) or any(map(_is_neg, tensors)):
        raise ValueError(f"{what}: a view that is conjugated or negated when it is read (bytes are moved as they are; see torch.Tensor.resolve_conj)")
    out, shape, dtype, dense, fields = [], None, None, False, None
    for i, t in enumerate(tensors):
        if dense and t.shape == shape and t.dtype is dtype and t.is_contiguous() and t.get_device() == index:
            if fields[0]:
                if not count:
                    count, size = t.numel(), t.element_size()
                _check_reach(t, what, count, size)
        else:
            fields = _state(t, what, i, batch, beams, index)
            shape, dtype, dense, count = t.shape, t.dtype, t.is_contiguous(), 0
        out.append(fields)
    return out


def _like(states, shapes, n: int, wide: int):
    """New dense tensors for the states' rows.  Neighbours of one shape and type share an allocation, where each begins at a
    multiple of 16 bytes."""
    out, i = [], 0
    while i < len(states):
        x, j = states[i], i + 1
        while j < len(states) and states[j].shape == x.shape and states[j].dtype is x.dtype:
            j += 1
        batch, row = x.shape[0], shapes[i][0]
        if j - i > 1 and batch * n * row % 16 == 0:
            out += x.new_empty((j - i, batch, n, *x.shape[2:])).unbind(0)
        elif n == wide and x.is_contiguous():
            out += [torch.empty_like(x) for x in states[i:j]]           # (two thirds of the time of what follows)
        else:
            out += [x.new_empty((batch, n, *x.shape[2:])) for x in states[i:j]]
        i = j
    return out


def _reorder(states, beams, out, s):
    batch, n = beams.shape
    index = beams.get_device()
    beams_at = _dense(beams, "beams", batch, n, _BEAMS, index)
    wide = states[0].shape[1] if states and states[0].dim() >= 2 else 1
    if (batch | wide | n) >> 31:
        raise ValueError(f"batch {batch}, beams {wide}, n {n}: one of them is out of range")
    src = _states(states, "states", batch, wide, index)
    if out is None:
        out = _like(states, src, n, wide)
        dst = [(row, n * row, row) for row, _, _ in src]
    else:
        if len(out) != len(states):
            raise ValueError(f"out: {len(out)} tensors for {len(states)} states")
        for i, (x, y) in enumerate(zip(states, out)):
            if y.dtype != x.dtype or y.shape[2:] != x.shape[2:]:
                raise ValueError(f"out[{i}]: need {x.dtype} [{batch}, {n}, ...] like states[{i}], got {y.dtype} {tuple(y.shape)}")
        dst = _states(out, "out", batch, n, index)
    if batch and n and wide:
        fields = []
        for x, y, (row, x_batch, x_beam), (_, y_batch, y_beam) in zip(states, out, src, dst):
            fields += (x.data_ptr(), y.data_ptr(), row, x_batch, x_beam, y_batch, y_beam)
        st = B.codec_beam_reorder(fields, beams_at, batch, wide, n, s)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_beam_reorder")
    return out
