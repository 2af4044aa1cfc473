"""Rotary positions of a model: which dims of a head are turned, in which pairs, how fast, and how a context longer than the trained one is met
(ouro_rotary of include/ouro.h).

    rotary = Rotary(head_dim, theta, rotary_dim=64, interleaved=True, scaling="yarn", factor=16.0, original=4096)
    q = cache.append_rotary(layer, q, k, v, slots, positions, rotary)

Pair i of rotary_dim / 2 turns by theta^(-2i / rotary_dim) radians a position.  Scalings of that, by ``factor``:

  none      as trained
  linear    positions are divided by factor
  ntk       theta is multiplied by factor^(rotary_dim / (rotary_dim - 2)): the slowest pair is slowed down by factor, the fastest stays
  yarn      pairs that turn more than ``beta_fast`` times within the ``original`` context stay, those that turn less than ``beta_slow`` times are slowed
            down by factor, those between partly; rotated vectors grow by 1 + ln(factor) / 10 (Peng et al., YaRN, arXiv 2309.00071, section 3)

A context that grows while a text does ("dynamic") is a new ``Rotary`` whenever the factor changes: it is rotary_dim / 2 numbers, not a table of positions.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from .binding import RotaryC

SCALINGS = ("none", "linear", "ntk", "yarn")


def frequencies(rotary_dim: int, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0, original: int = 0, beta_fast: float = 32.0,
                beta_slow: float = 1.0):
    """Radians a position of every pair (f64, on the CPU), and what rotated vectors are multiplied with."""
    if rotary_dim < 4 or rotary_dim % 2:
        raise ValueError(f"rotary_dim {rotary_dim}: an even number from 4 on is needed")
    if scaling not in SCALINGS:
        raise ValueError(f"scaling {scaling!r}: one of {', '.join(SCALINGS)} is needed")
    if not (theta > 1.0 and math.isfinite(theta) and factor >= 1.0 and math.isfinite(factor)):
        raise ValueError("theta above 1 and factor from 1 on are needed")
    if scaling == "none" and factor != 1.0:
        raise ValueError("a factor needs a scaling")
    if scaling == "ntk":
        theta = theta * factor ** (rotary_dim / (rotary_dim - 2))
    pair = torch.arange(rotary_dim // 2, dtype=torch.float64)
    inv = theta ** (-2.0 * pair / rotary_dim)
    if scaling == "linear":
        return inv / factor, 1.0
    if scaling == "yarn":
        if original < 1 or not beta_fast > beta_slow > 0:
            raise ValueError("yarn needs the original context, and beta_fast > beta_slow > 0")

        def pair_of(turns):                                        # the (fractional) pair that makes so many turns within the original context
            return rotary_dim * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(theta))

        low, high = max(math.floor(pair_of(beta_fast)), 0), min(math.ceil(pair_of(beta_slow)), rotary_dim - 1)
        slowed = ((pair - low) / max(high - low, 0.001)).clamp(0, 1)
        return inv / factor * slowed + inv * (1 - slowed), 0.1 * math.log(factor) + 1.0
    return inv, 1.0


class Rotary:
    """``turns`` [rotary_dim / 2] f64 on the device: whole turns a position."""

    def __init__(self, head_dim: int, theta: float = 10000.0, *, rotary_dim: int | None = None, interleaved: bool = False, scaling: str = "none", factor: float = 1.0,
                 original: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda:0"):
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if rotary_dim < 16 or rotary_dim % 16 or rotary_dim > head_dim:
            raise ValueError(f"rotary_dim {rotary_dim}: a multiple of 16 up to head_dim {head_dim} is needed")
        inv, self.magnitude = frequencies(rotary_dim, theta, scaling, factor, original, beta_fast, beta_slow)
        self.head_dim, self.rotary_dim, self.interleaved = head_dim, rotary_dim, bool(interleaved)
        self.turns = (inv / (2 * math.pi)).to(device)
        self._c = RotaryC(self.turns.data_ptr(), rotary_dim, int(self.interleaved), self.magnitude)
        self._p = C.byref(self._c)
