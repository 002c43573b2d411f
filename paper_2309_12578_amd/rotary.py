"""Positions as rotations of queries and keys, with one axis (text), two (images) or more (video).  Argument handling only; the operator is a
kernel of the library (csrc/rotary_kernels.hip), its autograd node native (csrc/host_ext.cpp)."""
from __future__ import annotations

import dataclasses
from fractions import Fraction
from typing import Optional, Sequence

import torch

from . import binding as _b

_PI = Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)


@dataclasses.dataclass(frozen=True)
class RotaryAxes:
    """Which axis turns each pair of a head's elements, and how fast: `turns` int64 [head_dim / 2], the frequency (angle of a step) in turns as an
    integer in 2^-64 modulo 2^64, `axis_of` uint8 [head_dim / 2].  Any such tensors will do; `rotary_axes` makes the usual ones.  A program makes
    it once and keeps it."""
    head_dim: int
    count: int
    turns: torch.Tensor
    axis_of: torch.Tensor
    neighbours: bool = False

    def __post_init__(self):
        if self.head_dim < 16 or self.head_dim > 256 or self.head_dim % 16:
            raise ValueError("the head dimension must be a multiple of 16, at most 256")
        if not 1 <= self.count <= 255:
            raise ValueError("1 to 255 axes")
        pairs = (self.head_dim // 2,)
        if self.turns.dtype != torch.int64 or self.turns.shape != pairs or self.axis_of.dtype != torch.uint8 or self.axis_of.shape != pairs:
            raise ValueError("turns must be int64, axis_of uint8, both [head_dim / 2]")
        object.__setattr__(self, "neighbours", bool(self.neighbours))   # (a NumPy truth value, or a number, too)


def _turns(frequency: float) -> int:
    n = round(Fraction(frequency) * 2 ** 64 / (2 * _PI)) % 2 ** 64
    return n - 2 ** 64 if n >= 2 ** 63 else n


def rotary_axes(head_dim: int, sections: Sequence[int], base: float = 10000.0, ladder: str = "shared", neighbours: bool = False,
                device=None) -> RotaryAxes:
    """The usual axes: the first sections[0] of the head_dim / 2 pairs belong to axis 0, the next sections[1] to axis 1 and so on; pairs beyond them
    stay as they are.  ladder: with "shared", pair i turns by base^(-i / (head_dim / 2)) a step whatever its axis; with "own" each axis has all
    frequencies, its j-th pair of n turns by base^(-j / n).  A pair is elements i and i + head_dim / 2, with `neighbours` 2 i and 2 i + 1."""
    pairs = head_dim // 2
    if ladder not in ("shared", "own"):
        raise ValueError("ladder must be 'shared' or 'own'")
    if not sections or min(sections) < 1 or sum(sections) > pairs:
        raise ValueError("every axis needs a pair, and together they can have head_dim / 2")
    if not 1.0 < base < float("inf"):
        raise ValueError("base must be above 1")
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    place = [j / n for n in sections for j in range(n)] if ladder == "own" else [i / pairs for i in range(len(axis))]
    rest = pairs - len(axis)
    turns = [_turns(base ** -p) for p in place] + [0] * rest
    return RotaryAxes(head_dim, len(sections), torch.tensor(turns, dtype=torch.int64, device=device),
                      torch.tensor(axis + [0] * rest, dtype=torch.uint8, device=device), neighbours)


def rotary(x: torch.Tensor, axes: RotaryAxes, positions: torch.Tensor, heads: Optional[int] = None) -> torch.Tensor:
    """x [B, H, L, head_dim], or [B, L, H * head_dim] with heads beside each other as a projection leaves them (bf16 or fp32; any strides, so that transposed views
    of [B, L, H, head_dim] will do; the result lies as x does, if x has no gaps and heads are dense), with the pairs (a, b) of its first `heads` heads (all of them if not given) turned by
    t = position * frequency: (a cos t - b sin t, b cos t + a sin t); the others are copied, so that queries and keys in a joint projection's output are turned in one call.
    positions: int32 or int64 [axes, L], or [axes, B, L], of any sign; angles are exact to position * 2^-65 turns, then in fp32.  A pair that does not turn stays as it is,
    whatever it holds.  Differentiable with respect to x."""
    return (_b._host or _b._native()).rotary(x, axes.turns, axes.axis_of, positions, axes.count, heads, axes.neighbours)
