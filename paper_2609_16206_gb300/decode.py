"""One decode step of a served model on this GPU: helpers around the operators of ``include/ctr_decode.h``.

``rope_turns`` makes the frequency words of ``ctr.Rope``.
"""
from __future__ import annotations

import math

import torch


def rope_turns(rot_dim: int, base: float = 10000.0, factor: float = 1.0, trained_len: int = 0, fast: float = 32.0,
               slow: float = 1.0, device="cuda") -> torch.Tensor:
    """The frequency word of every rotated pair: base^(-2i / rot_dim) / 2 pi turns per position, times 2^64.

    ``factor`` > 1 scales the positions for contexts longer than the model was trained on: with ``trained_len`` = 0
    every frequency is divided by it (linear interpolation); otherwise a pair that makes at least ``fast`` turns over
    the trained length keeps its frequency, one that makes at most ``slow`` is divided, and those between are blended
    linearly in their number of turns."""
    if rot_dim % 2 != 0 or rot_dim < 0 or factor < 1.0 or base <= 1.0:
        raise ValueError("rot_dim must be even and not negative, factor at least 1, base above 1")
    words = []
    for i in range(rot_dim // 2):
        f = base ** (-2 * i / rot_dim) / (2 * math.pi)
        keep = 0.0
        if trained_len > 0:
            keep = min(1.0, max(0.0, (f * trained_len - slow) / (fast - slow)))
        w = int(f * (keep + (1 - keep) / factor) * 2.0 ** 64)
        words.append(w - (1 << 64) if w >= 1 << 63 else w)
    return torch.tensor(words, dtype=torch.int64, device=device)
