"""Rotary positions: the angles of a model, and rows turned by them (plc_rotate; in the paged cache, PagedKVCache.store_rotated).
"""
from __future__ import annotations

import torch

from . import plc


class Rotary:
    """The rotation of heads of d components by position: of the first r of them (default: all), in halves, pairs (i, i + r/2),
    or interleaved, pairs (2i, 2i + 1).

    The angles are base^(-2i/r) radians a position, stretched for contexts longer than a model was trained on by `scaling`:
    "linear" (divided by `factor`), "stretched" (the base times factor^(r/(r-2))), "parts" (divided where there are `low` turns or fewer within the
    `trained` positions, whole from `high` turns on, in proportion between) or "ramp" (in proportion to i between the pairs of `high` and of
    `low` turns); plc.h has the formulas.  Or they are given: `theta`, r/2 numbers.  Rotated rows are multiplied by `magnitude`."""

    def __init__(self, d, r=None, base=10000.0, interleaved=False, scaling="none", factor=1.0, low=1.0, high=2.0, trained=1,
                 magnitude=1.0, theta=None, device="cuda"):
        if theta is not None:
            theta = [float(t) for t in theta]
            if r is not None and r != 2 * len(theta):
                raise ValueError("theta has a number for each of r / 2 pairs")
        else:
            theta = plc.plc_rotary_frequencies(d if r is None else r, scaling, base, factor, low, high, trained)
        if not theta or 2 * len(theta) > d:
            raise ValueError(f"{2 * len(theta)} of {d} components cannot be rotated")
        self.d, self.theta, self.interleaved, self.magnitude = d, theta, bool(interleaved), float(magnitude)
        signed = [t - (1 << 64) if t >> 63 else t for t in plc.plc_rotary_turns(theta)]
        self.turns = torch.tensor(signed, dtype=torch.int64).to(device)
        self.rotary = plc.make_rotary(self.turns, interleaved, magnitude)

    def rotate(self, x, positions, inverse=False, out=None):
        """Rows x [rows, heads, d] (fp16 or bf16) at positions (int32 [rows]); with `inverse` back again.  Returns out, which
        may be x."""
        if x.dim() != 3 or x.shape[2] != self.d:
            raise ValueError(f"rows are [rows, heads, {self.d}]")
        if x.device != self.turns.device:
            raise ValueError("the rows are on another device than the rotation")
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
        plc.plc_rotate(self.rotary, x, positions, inverse, out)
        return out
