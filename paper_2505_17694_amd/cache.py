"""Page pools of a K/V cache with what fills them, and rotary positions (marshalling only)."""
from __future__ import annotations

import contextlib
from types import SimpleNamespace

import numpy as np
import torch

from . import binding as B
from .runtime import _current_stream

_TORCH_DTYPE = {B.CODEC_DTYPE_FP16: torch.float16, B.CODEC_DTYPE_BF16: torch.bfloat16}
_CODE = {t: c for c, t in _TORCH_DTYPE.items()}
_SCALINGS = {"linear": B.CODEC_ROTARY_LINEAR, "ntk": B.CODEC_ROTARY_NTK, "wavelength": B.CODEC_ROTARY_WAVELENGTH,
             "yarn": B.CODEC_ROTARY_YARN}


_current_device = getattr(torch._C, "_cuda_getDevice", None)               # absent in a PyTorch without a GPU runtime
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_Rows = B.codec_rows
_data_ptr, _base_ptr, _nbytes = torch.Tensor.data_ptr, torch.UntypedStorage.data_ptr, torch.UntypedStorage.nbytes
_NO_RUNS = np.empty((0, 5), np.int32)


def _device(device) -> torch.device:
    d = torch.device(device)
    if d.type == "cuda" and d.index is None:
        d = torch.device("cuda", torch.cuda.current_device())
    return d


@contextlib.contextmanager
def _on(device: torch.device, stream):
    """Makes `device` and `stream` the current ones; the handle of the stream.  What is allocated meanwhile belongs to the
    stream that uses it."""
    if stream is not None and stream.device != device:
        raise ValueError(f"stream: on {stream.device}, the tensors are on {device}")
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield _current_stream(device)


def _enter(index: int, stream):
    """The stream's handle if a call on device `index` can go ahead as things are, else None: another device or stream has to be
    made current."""
    return _raw_stream(index) if stream is None and _current_device() == index else None


def _check_reach(t: torch.Tensor, what: str, last: int, size: int) -> None:
    """A tensor keeps its shape when its storage is given back: the memory behind it, `last` elements of `size` bytes from its
    first, is what counts."""
    if t.untyped_storage().nbytes() < (t.storage_offset() + last) * size:
        raise ValueError(f"{what}: the tensor's storage ends before its last element")


def _rows(t: torch.Tensor, what: str, shape, dtype: torch.dtype, index: int):
    """`t` as codec_rows: `shape` = (tokens, heads, head_dim) with contiguous channels, in storage that is there."""
    strides = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index or strides[2] != 1:
        raise ValueError(f"{what}: need a {dtype} tensor of shape {tuple(shape)} with contiguous channels on cuda:{index}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}, strides {strides}")
    tokens, heads, head_dim = shape
    if tokens == 0:
        return _Rows(0, 0, 0)
    token_stride, head_stride, _ = strides
    if tokens == 1:                         # the stride of a single token or head says nothing
        token_stride = 0
    if heads == 1:
        head_stride = 0
    if t.untyped_storage().nbytes() < 2 * (t.storage_offset() + (tokens - 1) * token_stride + (heads - 1) * head_stride + head_dim):
        raise ValueError(f"{what}: the tensor's storage ends before its last element")
    return _Rows(t.data_ptr(), token_stride, head_stride)


def _index(t: torch.Tensor, what: str, tokens: int, index: int) -> int:
    if t.shape != (tokens,) or t.dtype is not torch.int64 or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{what}: need a contiguous int64 tensor of shape {(tokens,)} on cuda:{index}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    if t.untyped_storage().nbytes() < 8 * (t.storage_offset() + tokens):
        raise ValueError(f"{what}: the tensor's storage ends before its last element")
    return t.data_ptr()


class Rotary:
    """Rotary positions: which channels turn and how fast (codec_rotary_config), with the device table behind them.

    ``rotary_dim`` channels of a head turn, in pairs (i, i + rotary_dim / 2) or, with ``interleaved``, (2i, 2i + 1).
    ``scaling``: None or a dict with ``kind`` ("linear", "ntk", "wavelength", "yarn"), ``factor`` and, for the last two,
    ``original_length`` and ``low``, ``high`` (wavelength; 1 and 4 unless given) or ``fast``, ``slow`` (yarn; 32 and 1).
    ``magnitude`` overrides the factor on turned channels that belongs to the scaling.
    """

    def __init__(self, rotary_dim, theta=10000.0, interleaved=False, scaling=None, device="cuda:0", magnitude=None):
        s = None
        if scaling is not None:
            known = {"kind", "factor", "original_length", "low", "high", "fast", "slow"}
            if scaling.get("kind") not in _SCALINGS or set(scaling) - known:
                raise ValueError(f"scaling: kind is one of {sorted(_SCALINGS)}, beside {sorted(known - {'kind'})}; got {scaling}")
            if not B._is_int32(scaling.get("original_length", 0)):
                raise B.CodecError(B.CODEC_ERR_INVALID_ARGUMENT, "codec_rotary_turns")
            s = B.codec_rotary_scaling(_SCALINGS[scaling["kind"]], scaling.get("original_length", 0), scaling.get("factor", 0.0),
                                       scaling.get("low", 1.0), scaling.get("high", 4.0), scaling.get("fast", 32.0),
                                       scaling.get("slow", 1.0))
        st, turns, factor = B.codec_rotary_turns(rotary_dim, theta, s)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_rotary_turns")
        self.device = _device(device)
        self.rotary_dim = rotary_dim
        self.magnitude = factor if magnitude is None else magnitude
        self._turns = torch.from_numpy(turns).to(self.device)
        layout = B.CODEC_ROTARY_INTERLEAVED if interleaved else B.CODEC_ROTARY_HALF
        self._config = [B.codec_rotary_config(rotary_dim, layout, inverse, self.magnitude, self._turns.data_ptr())
                        for inverse in (0, 1)]

    @property
    def turns(self) -> torch.Tensor:
        """Turns of a pair from one position to the next, 64 bits (a copy: the table itself is what the calls read)."""
        return self._turns.clone()

    def apply(self, x: torch.Tensor, positions: torch.Tensor, inverse=False, out: torch.Tensor = None, stream=None) -> torch.Tensor:
        """x [tokens, heads, head_dim] turned to its positions, or back (the gradient); ``out`` may be x itself.  Gradients pass
        from the result to x, unless ``out`` is given: then x must not want any."""
        if x.dim() != 3 or x.dtype not in _CODE or self.device.type != "cuda":
            raise ValueError(f"x: need a 16-bit tensor [tokens, heads, head_dim] and a GPU, got {x.dtype} {tuple(x.shape)} on {x.device}")
        s = _enter(self.device.index, stream)
        if s is None:
            with _on(self.device, stream) as s:
                return self._apply(x, positions, inverse, out, s)
        return self._apply(x, positions, inverse, out, s)

    def _apply(self, x, positions, inverse, out, s):
        if x.requires_grad and torch.is_grad_enabled():
            if out is not None:
                raise ValueError("out: x wants a gradient, which does not pass through out")
            return _Turn.apply(x, positions, self, inverse, s)
        return self._turn(x, positions, inverse, out, s)

    def _turn(self, x, positions, inverse, out, s):
        shape, index = x.shape, self.device.index
        if (shape[0] | shape[1] | shape[2]) >> 31:
            raise ValueError(f"x: {tuple(shape)} is too large for a call")
        rows = _rows(x, "x", shape, x.dtype, index)
        at = _index(positions, "positions", shape[0], index)
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
        into = _rows(out, "out", shape, x.dtype, index)
        st = B.codec_rotary(self._config[bool(inverse)], shape[1], shape[2], _CODE[x.dtype], rows, into, at, shape[0], s)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_rotary")
        return out


class _Turn(torch.autograd.Function):
    """The turn is linear in x; its transpose is the turn the other way."""

    @staticmethod
    def forward(ctx, x, positions, rotary, inverse, s):
        ctx.rotary, ctx.inverse = rotary, inverse
        ctx.save_for_backward(positions)
        return rotary._turn(x, positions, inverse, None, s)

    @staticmethod
    def backward(ctx, g):
        positions, = ctx.saved_tensors
        if not g.is_contiguous() or g.data_ptr() % 16:
            g = g.clone(memory_format=torch.contiguous_format)
        return ctx.rotary.apply(g, positions, not ctx.inverse), None, None, None, None


class KVCache:
    """The page pools of a cache, one K and one V pool per layer, with the operations that fill them, and who holds which page.

    ``head`` is the attribute bag a plan is built from (num_q_heads, num_kv_heads, head_dim, dtype, page_size).  ``layout``
    "thd": pools [num_pages, page_size, num_kv_heads, head_dim]; "htd": [num_pages, num_kv_heads, page_size, head_dim].
    ``pools``: the (k, v) tensors of the layers if the program has them already (views with other strides too, the same
    in every layer); otherwise they are allocated.  All pages are free at first: page lists that are in use already
    are made known by ``hold``.  Lists of pages, tokens, sequences and runs are arrays of any integer type; a number beyond
    32 bits is refused, and so is a fraction.
    """

    _pages = None

    def __init__(self, head, num_pages, layers=1, layout="htd", device="cuda:0", pools=None):
        if layout not in ("thd", "htd"):
            raise ValueError(f"layout: thd or htd, got {layout!r}")
        if head.dtype not in _TORCH_DTYPE:
            raise ValueError(f"head.dtype: {head.dtype}")
        self.head, self.layout, self.num_pages, self.device = head, layout, int(num_pages), _device(device)
        self.dtype = _TORCH_DTYPE[head.dtype]
        ps, h, d = head.page_size, head.num_kv_heads, head.head_dim
        shape = (self.num_pages, ps, h, d) if layout == "thd" else (self.num_pages, h, ps, d)
        if pools is None:
            pools = [tuple(torch.empty(shape, dtype=self.dtype, device=self.device) for _ in "kv") for _ in range(layers)]
        self._pools = tuple(tuple(kv) for kv in pools)
        flat = [p for kv in self._pools for p in kv]
        if not flat or any(len(kv) != 2 for kv in self._pools):
            raise ValueError("pools: need a (k, v) pair for every layer")
        strides = flat[0].stride()
        for p in flat:
            if p.shape != shape or p.dtype != self.dtype or p.device != self.device or p.stride() != strides or p.stride(3) != 1:
                raise ValueError(f"pools: need {self.dtype} tensors of shape {shape} on {self.device} with the same strides and "
                                 f"contiguous channels, got {p.dtype} {tuple(p.shape)} on {p.device}, strides {p.stride()}")
        page, token, kv_head = (strides[0], strides[1], strides[2]) if layout == "thd" else (strides[0], strides[2], strides[1])
        self.page_stride, self.token_stride, self.head_stride = page, token, kv_head
        self._layout = B.codec_kv_layout(self.num_pages, page, token, kv_head)
        self._head = B.codec_head_config(head.num_q_heads, h, d, head.dtype, ps, 0.0)
        self._index = self.device.index if self.device.type == "cuda" else None
        self._q_row, self._kv_row = (head.num_q_heads, d), (h, d)
        # what a pool has to be when it is used
        self._flat, self._strides, self._count = tuple(flat), strides, flat[0].numel()
        self._reach = (self.num_pages - 1) * page + (ps - 1) * token + (h - 1) * kv_head + d
        # and where the pools were when they were last looked at: address, storage with its address and bytes
        self._places, self._storages = [p.data_ptr() for p in flat], [p.untyped_storage() for p in flat]
        self._bases, self._sizes = [-1] * len(flat), [-1] * len(flat)
        self._copy_status = None            # whether pages of these pools can be copied, once that was asked
        st, self._pages = B.codec_pages_create(self.num_pages)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_pages_create")

    def __del__(self):
        try:
            B.codec_pages_destroy(self._pages)
        except Exception:
            pass

    @property
    def pools(self):
        """The layers' (k, v) tensors."""
        return self._pools

    def paged(self, node_page_off, page_ids):
        """These pools with a forest's page lists: the ``paged`` of a PlannedAttention."""
        return SimpleNamespace(node_page_off=node_page_off, page_ids=page_ids, num_pages=self.num_pages,
                               page_stride=self.page_stride, token_stride=self.token_stride, head_stride=self.head_stride)

    def _check_pool(self, i: int) -> None:
        """Looks at pool i as it is now, and keeps where it is."""
        p = self._flat[i]
        storage = p.untyped_storage()
        if storage.nbytes() < 2 * (p.storage_offset() + self._reach):
            raise ValueError(f"pools of layer {i // 2}: the storage ends before the last page")
        if p.stride() != self._strides or p.numel() != self._count or p.dtype is not self.dtype or p.device != self.device:
            raise ValueError(f"pools of layer {i // 2}: {self._count} elements of {self.dtype} on {self.device} with strides {self._strides} "
                             f"were handed over, now they are {p.dtype} {tuple(p.shape)} on {p.device} with strides {p.stride()}")
        self._places[i], self._storages[i], self._bases[i], self._sizes[i] = p.data_ptr(), storage, storage.data_ptr(), storage.nbytes()
        self._copy_status = None

    def _check_storage(self, layer: int) -> None:
        """A pool is a tensor that others hold too: it may get other memory (``data``, ``set_``), or its storage may.  What has been
        looked at is not looked at again while the tensor begins where it did and the storage, which is held, is still there."""
        for i in (2 * layer, 2 * layer + 1):
            storage = self._storages[i]
            if self._flat[i].data_ptr() != self._places[i] or storage.data_ptr() != self._bases[i] or storage.nbytes() != self._sizes[i]:
                self._check_pool(i)

    def _check_storages(self) -> None:
        """_check_storage of all layers."""
        if (list(map(_data_ptr, self._flat)) != self._places or list(map(_base_ptr, self._storages)) != self._bases
                or list(map(_nbytes, self._storages)) != self._sizes):
            for i in range(len(self._flat)):
                self._check_pool(i)

    def append(self, layer, q, k, v, positions, slots, rotary: Rotary = None, q_out: torch.Tensor = None, stream=None):
        """The step's tokens into ``layer``: queries and keys turned to ``positions``, keys and values stored at ``slots``
        (page * page_size + token; negative: not stored).  Returns the turned queries (``q_out``, which may be q itself);
        q None: keys and values only.  Without ``rotary`` rows pass as they are and ``positions`` may be None.  A cache takes part
        in no gradient: the queries come back without one (Rotary.apply passes it)."""
        if self._index is None:
            raise ValueError(f"append needs pools on a GPU, these are on {self.device}")
        s = _enter(self._index, stream)
        if s is None:
            with _on(self.device, stream) as s:
                return self._append(layer, q, k, v, positions, slots, rotary, q_out, s)
        return self._append(layer, q, k, v, positions, slots, rotary, q_out, s)

    def _append(self, layer, q, k, v, positions, slots, rotary, q_out, s):
        index, dtype, tokens = self._index, self.dtype, k.shape[0]
        if tokens >> 31:
            raise ValueError(f"k: {tokens} tokens, at most 2^31 - 1 go into a call")
        self._check_storage(layer)
        kv_shape = (tokens, *self._kv_row)
        k_rows = _rows(k, "k", kv_shape, dtype, index)
        v_rows = _rows(v, "v", kv_shape, dtype, index)
        q_rows = out_rows = config = at = None
        if q is not None:
            q_shape = (tokens, *self._q_row)
            q_rows = _rows(q, "q", q_shape, dtype, index)
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
            out_rows = _rows(q_out, "q_out", q_shape, dtype, index) if q_out is not q else q_rows
        elif q_out is not None:
            raise ValueError("q_out without q")
        if rotary is not None:
            if rotary.device != self.device:
                raise ValueError(f"rotary is on {rotary.device}, the pools are on {self.device}")
            config, at = rotary._config[0], _index(positions, "positions", tokens, index)
        kp, vp = self._places[2 * layer], self._places[2 * layer + 1]
        st = B.codec_append(self._head, config, q_rows, out_rows, k_rows, v_rows, at, _index(slots, "slots", tokens, index),
                            tokens, kp, vp, self._layout, s)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_append")
        return q_out

    @property
    def free_pages(self) -> int:
        return B.codec_pages_free(self._pages)

    def take(self, n: int) -> np.ndarray:
        """The n lowest free pages, now held."""
        st, ids = B.codec_pages_take(self._pages, n)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_pages_take")
        return ids

    def hold(self, page_ids) -> None:
        """One more holder for every page of the list."""
        st = B.codec_pages_hold(self._pages, page_ids)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_pages_hold")

    def release(self, page_ids) -> None:
        """One holder less for every page of the list; those without are free."""
        st = B.codec_pages_release(self._pages, page_ids)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_pages_release")

    def copy(self, runs, stream=None) -> None:
        """Copies runs of tokens, rows (source page, source token, destination page, destination token, tokens), in the
        pools of every layer.  No token may be written twice, or read and written."""
        self._check_pools()
        self._check_call("copy", stream)
        self._copy_on(runs, stream)

    def _check_pools(self) -> None:
        """Whether pages of the pools can be copied."""
        self._check_storages()
        if self._copy_status is None:
            self._copy_status = self._enqueue(_NO_RUNS, 0)
        if self._copy_status != B.CODEC_OK:
            raise B.CodecError(self._copy_status, "codec_cache_copy")

    def _check_call(self, what: str, stream) -> None:
        if self.device.type != "cuda":
            raise ValueError(f"{what} needs pools on a GPU, these are on {self.device}")
        if stream is not None and stream.device != self.device:
            raise ValueError(f"stream: on {stream.device}, the pools are on {self.device}")

    def _copy_on(self, runs, stream):
        s = _enter(self.device.index, stream)
        if s is None:
            with _on(self.device, stream) as s:
                return self._copy(runs, s)
        self._copy(runs, s)

    def _copy(self, runs, s):
        st = self._enqueue(runs, s)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_cache_copy")

    def _enqueue(self, runs, s):
        return B.codec_cache_copy(self._head, self._layout, self._places[0::2], self._places[1::2], runs, s)

    def fork(self, page_off, page_ids, tokens, parents, stream=None):
        """Sequence s holds the pages page_ids[page_off[s]:page_off[s + 1]] with tokens[s] tokens.  In the place of these
        sequences others go on, sequence j from sequence parents[j]: a sequence may go on once, several times or not at
        all.  Returns the page lists (page_off, page_ids) of those that go on.  They share whole pages; what is partly
        filled is copied on `stream` for all but the first (see codec_pages_fork)."""
        if self._copy_status != B.CODEC_OK:             # not looked at yet, or known to be refused
            self._check_pools()
        self._check_call("fork", stream)
        st, off, ids, runs = B.codec_pages_fork(self._pages, self.head.page_size, page_off, page_ids, tokens, parents)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_pages_fork")
        if len(runs):
            try:
                self._check_pools()
                self._copy_on(runs, stream)
            except Exception:                           # the pages are held by the old lists again
                B.codec_pages_hold(self._pages, page_ids)
                B.codec_pages_release(self._pages, ids)
                raise
        return off, ids

    def compact(self, stream=None) -> np.ndarray:
        """Moves the held pages to the lowest ids, copying them on `stream`.  Returns the new id of every page: page
        lists go on as ``moved[page_ids]``."""
        self._check_pools()
        self._check_call("compact", stream)
        st, runs = B.codec_pages_compact(self._pages, self.head.page_size, self.num_pages // 2)
        if st != B.CODEC_OK:
            raise B.CodecError(st, "codec_pages_compact")
        moved = np.arange(self.num_pages, dtype=np.int32)
        moved[runs[:, 0]] = runs[:, 2]
        if len(runs):
            self._copy_on(runs, stream)
        return moved
