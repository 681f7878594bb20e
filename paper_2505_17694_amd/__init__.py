"""Prefix-shared decode attention for MI355X (gfx950): Python face of libcodec.so.

``binding`` mirrors the C ABI of include/codec.h name for name; ``runtime``
adds a thin holder that keeps a plan together with the PyTorch tensors used as
its device memory; ``cache`` holds the page pools the attention reads, and puts
new tokens into them; ``beam`` chooses the tokens and moves the beams'
states.  There is no CPU fallback: without the built library the
import fails.
"""
from .binding import *          # noqa: F401,F403
from .binding import EXPORTED_SYMBOLS, LIB_PATH, CodecError
from .beam import beam_reorder, beam_select
from .cache import KVCache, Rotary, StepTokens
from .runtime import PlannedAttention

__all__ = ["EXPORTED_SYMBOLS", "LIB_PATH", "CodecError", "KVCache", "PlannedAttention", "Rotary", "StepTokens",
           "beam_reorder", "beam_select"]
