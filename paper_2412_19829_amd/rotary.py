"""Angles per position for gformer_rotary, also of contexts longer than a model was trained on.  Host arithmetic in 64 bits."""
from __future__ import annotations

import math

import torch


def rotary_frequencies(rot: int, base: float = 10000.0, *, stretch: float = 1.0, trained: int = 0, slow: float = 1.0, fast: float = 32.0,
                       device="cuda"):
    """The angle per position of each pair of a head's first `rot` channels, base^(-2 i / rot), as fp32 [rot / 2].

    A context stretched to `stretch` times the trained length: with trained = 0 every pair is slowed by as much; otherwise
    pairs that turn `fast` times and more within the `trained` positions keep their speed, those that turn at most
    `slow` times are slowed, and the ones between go over from one to the other by their number of turns.  rotary_factor()
    is the factor that goes with it."""
    if rot < 2 or rot % 2:
        raise ValueError("rot must be a positive even number")
    if not (math.isfinite(base) and base > 0) or not (math.isfinite(stretch) and stretch >= 1.0):
        raise ValueError("base must be positive, stretch at least 1")
    if trained < 0 or not 0 < slow < fast:
        raise ValueError("trained must not be negative, slow positive and below fast")
    f = torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    keep = torch.zeros_like(f)
    if trained:
        turns = trained * f / (2.0 * math.pi)
        keep = ((turns - slow) / (fast - slow)).clamp(0.0, 1.0)
    return (f * keep + f / stretch * (1.0 - keep)).to(torch.float32).to(device)


def rotary_factor(stretch: float) -> float:
    """What queries and keys are multiplied by in a stretched context, 0.1 ln(stretch) + 1, which sharpens the softmax as the number of
    keys grows."""
    if not (math.isfinite(stretch) and stretch >= 1.0):
        raise ValueError("stretch must be at least 1")
    return 0.1 * math.log(stretch) + 1.0
