"""Rotary positions: which columns of a row of Q or K turn with its position, and how fast.

Pair i of the first r columns, columns (2 i, 2 i + 1) or (i, i + r / 2), at position p turns by p * frequencies[i] and is multiplied by
`magnitude`; columns behind r stay as they are.  A product of a turned query and a turned key then depends on the difference of their positions.
`Rotary` is what `autograd.rotary_embedding`, `autograd.flash_attention`, `binding.attn_rotary` and `binding.attn_paged_append` take.
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, *, scaling: Optional[str] = None, factor: float = 1.0,
                       original_length: int = 4096, slow_turns: float = 1.0, fast_turns: float = 32.0) -> Tuple[torch.Tensor, float]:
    """(frequencies, magnitude): float64 [rotary_dim / 2] on the CPU, radians a position.

    Pair i turns by base^(-2 i / rotary_dim).  For contexts `factor` times as long as those that a model was trained on (`original_length` tokens),
    scaling is one of
      "linear"  every frequency divided by the factor: positions are squeezed into the trained range
      "base"    a larger base, base * factor^(r / (r - 2)): the slowest pair is slowed by the factor, the fastest stays
      "parts"   pairs that turn `fast_turns` times or more within the trained length stay, those that turn `slow_turns` times or less are divided by the
                factor, and between them the share that is divided falls evenly with the number of turns; magnitude 0.1 ln(factor) + 1
    """
    if rotary_dim < 2 or rotary_dim % 2 != 0:
        raise ValueError("rotary_dim must be even and at least 2")
    if not (math.isfinite(base) and base > 1.0):
        raise ValueError("base must be finite and greater than 1")
    if not (math.isfinite(factor) and factor >= 1.0):
        raise ValueError("factor must be finite and at least 1")
    if scaling not in (None, "linear", "base", "parts"):
        raise ValueError("scaling must be None, 'linear', 'base' or 'parts'")
    if scaling is None and factor != 1.0:
        raise ValueError("a factor needs a scaling")
    if scaling == "base" and rotary_dim > 2:
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    f = base ** (-2.0 * torch.arange(rotary_dim // 2, dtype=torch.float64) / rotary_dim)
    if scaling == "linear":
        f = f / factor
    magnitude = 1.0
    if scaling == "parts":
        if original_length <= 0 or not fast_turns > slow_turns:
            raise ValueError("original_length must be positive, and fast_turns greater than slow_turns")
        keep = ((f * (original_length / (2.0 * math.pi)) - slow_turns) / (fast_turns - slow_turns)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
        magnitude = 0.1 * math.log(factor) + 1.0
    return f, magnitude


class Rotary:
    """Frequencies (float64 [r / 2], on the GPU of the tensors they turn), the way columns pair up, and the factor of the turned columns."""

    __slots__ = ("frequencies", "interleaved", "magnitude")

    def __init__(self, frequencies: torch.Tensor, *, interleaved: bool = False, magnitude: float = 1.0):
        if frequencies.dtype != torch.float64 or frequencies.dim() != 1 or not frequencies.is_contiguous() or frequencies.numel() == 0:
            raise TypeError("frequencies must be a contiguous float64 tensor [rotary_dim / 2]")
        if not math.isfinite(magnitude):
            raise ValueError("magnitude must be finite")
        self.frequencies, self.interleaved, self.magnitude = frequencies, bool(interleaved), float(magnitude)

    @classmethod
    def make(cls, rotary_dim: int, base: float = 10000.0, *, interleaved: bool = False, device="cuda", **scaling) -> "Rotary":
        """From `rotary_frequencies` (its `scaling`, `factor`, ...)."""
        frequencies, magnitude = rotary_frequencies(rotary_dim, base, **scaling)
        return cls(frequencies.to(device), interleaved=interleaved, magnitude=magnitude)
