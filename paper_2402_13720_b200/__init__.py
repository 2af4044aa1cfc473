"""Ouroboros verification path for one B200: CUDA library (libouro.so) plus a thin ctypes binding."""
from . import synth  # noqa: F401
from .binding import Engine, OuroError, lib  # noqa: F401
from .paged import PagedCache  # noqa: F401
from .rotary import Rotary  # noqa: F401
from .scores import constrain_logits, token_logprobs  # noqa: F401
