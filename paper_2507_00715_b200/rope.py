"""Frequencies of the rotary positions: radians per position of every pair, in double, and the amplitude that goes with them.

The calls (binding.make_rope) take any frequencies; these are the usual ones.  ``scaling`` stretches the positions a model was
trained on (``original`` of them) by ``factor``:

  None      theta^(-2i / rot_dim)
  "linear"  all frequencies divided by the factor
  "base"    theta times factor^(rot_dim / (rot_dim - 2)): the fastest pair keeps its frequency, the slowest is divided by the factor
  "ramp"    pairs that make more than ``fast`` turns over the original length keep their frequency, those with less than ``slow``
            turns are divided by the factor, between them the weight of the old frequency falls linearly with the pair's number,
            from 1 to 0 between the two pairs that make ``fast`` and ``slow`` turns, as real numbers and rounded outward to whole
            ones (as the models that were trained with such a ramp have it); amplitude 0.1 ln(factor) + 1
  "bands"   the same, but the weight grows linearly with the number of turns, and the amplitude is 1

The amplitude is an argument of its own of make_rope, so any of these goes with any amplitude.
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch


def frequencies(rot_dim: int, theta: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0, original: int = 0,
                slow: float = 1.0, fast: float = 32.0) -> Tuple[torch.Tensor, float]:
    """fp64 [rot_dim / 2] on the host, and the amplitude."""
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError(f"rot_dim: {rot_dim}, expected an even number of at least 2")
    if scaling not in (None, "linear", "base", "ramp", "bands"):
        raise ValueError(f"scaling: {scaling!r}")
    if not 0.0 < theta < math.inf or (scaling == "ramp" and theta <= 1.0):
        raise ValueError(f"theta: {theta}, expected a positive number{' greater than 1' if scaling == 'ramp' else ''}")
    if scaling is not None and not 1.0 <= factor < math.inf:
        raise ValueError(f"factor: {factor}, expected at least 1")
    if scaling in ("ramp", "bands") and (original < 1 or not 0 < slow < fast):
        raise ValueError("original length and 0 < slow < fast are needed")
    if scaling == "base" and rot_dim > 2:
        theta = theta * factor ** (rot_dim / (rot_dim - 2))
    f = theta ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "bands":
        keep = ((original * f / (2.0 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    elif scaling == "ramp":
        # the pairs (as real numbers) that make `fast` and `slow` turns: original * theta^(-2i / rot_dim) = 2 pi turns
        first, last = (rot_dim * math.log(original / (2.0 * math.pi * n)) / (2.0 * math.log(theta)) for n in (fast, slow))
        first, last = math.floor(first), math.ceil(last)
        keep = ((last - torch.arange(rot_dim // 2, dtype=torch.float64)) / (last - first)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    return f, 0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0
