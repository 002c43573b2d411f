"""What a Transformer adds to the sparse attention: a learned relative position bias by buckets and dropout whose mask is
never stored.  Argument handling only; the operators are kernels of the library (csrc/attn_extras_kernels.hip,
csrc/dropout_kernels.hip), their autograd nodes native (csrc/host_ext.cpp)."""
from __future__ import annotations

import dataclasses
from typing import List, Optional

import numpy as np
import torch

from . import binding as _b


@dataclasses.dataclass(frozen=True)
class RelativeBuckets:
    """Which bucket of a bias table each distance key - query has: `map[d + length - 1]` for -length < d < length, uint8.  Any map
    will do; `relative_buckets` makes the usual one.  A program makes it once, for its longest sequences, and keeps it."""
    length: int
    count: int
    map: torch.Tensor

    def __post_init__(self):
        if not 1 <= self.count <= 256:
            raise ValueError("1 to 256 buckets")
        if self.map.dtype != torch.uint8 or self.map.shape != (2 * self.length - 1,):
            raise ValueError("the map must be uint8 [2 * length - 1]")


def _bucket_starts(n: int, max_distance: int) -> List[int]:
    """First distance of each of n buckets.  The first n // 2 have one distance each; from `exact` = n // 2 on they grow
    geometrically: bucket exact + j starts at the smallest d with d >= exact (max_distance / exact)^(j / (n - exact)), found
    in integers, so that no rounding decides on a border."""
    exact = n // 2
    wide = n - exact
    starts = list(range(exact))
    for j in range(wide):
        bound = max_distance ** j * exact ** wide
        lo, hi = exact, max_distance
        while lo < hi:
            d = (lo + hi) // 2
            if d ** wide * exact ** j >= bound:
                hi = d
            else:
                lo = d + 1
        starts.append(lo)
    return starts


def relative_buckets(length: int, count: int = 32, max_distance: int = 128, bidirectional: bool = True,
                     device=None) -> RelativeBuckets:
    """The usual buckets: near distances have one each, farther ones share buckets that grow geometrically, everything from
    about `max_distance` on is in the last.  bidirectional: keys behind the query have the first half of the buckets, keys ahead
    of it the second; otherwise all buckets are for keys behind, and keys ahead share bucket 0 with the query's own position."""
    if length < 1:
        raise ValueError("length must be positive")
    if not 1 <= count <= 256 or (bidirectional and count % 2):
        raise ValueError("1 to 256 buckets, an even number of them where both directions have their own")
    n = count // 2 if bidirectional else count
    if n < 2 or max_distance <= n // 2:
        raise ValueError("too few buckets, or max_distance within those of one distance each")
    d = np.arange(-(length - 1), length)
    far = np.abs(d) if bidirectional else np.maximum(-d, 0)
    bucket = np.searchsorted(np.asarray(_bucket_starts(n, max_distance)), far, side="right") - 1
    if bidirectional:
        bucket = bucket + n * (d > 0)
    return RelativeBuckets(length, count, torch.from_numpy(bucket.astype(np.uint8)).to(device))


def _map_for(table: torch.Tensor, buckets: Optional[RelativeBuckets], length: Optional[int] = None) -> torch.Tensor:
    """The buckets of the distances that sequences of `length` tokens have."""
    if not isinstance(buckets, RelativeBuckets):
        raise ValueError("a bias table needs its RelativeBuckets")
    if table.shape[:1] != (buckets.count,):
        raise ValueError("the bias table must have a row for each bucket")
    if length is None or length == buckets.length:
        return buckets.map
    if length > buckets.length:
        raise ValueError("the buckets do not reach over sequences of %d tokens" % length)
    return buckets.map[buckets.length - length:buckets.length + length - 1]


def relative_bias(table: torch.Tensor, buckets: RelativeBuckets, q_len: int, k_len: int, q_start: int = 0) -> torch.Tensor:
    """The bias as a dense tensor [H, q_len, k_len] of the table's dtype (bf16 or fp32), table [buckets, H]: for the dense
    attention before a layer has its pattern, and for single queries (`q_start` is the position of the first one; keys start at
    position 0).  Differentiable with respect to the table; sums in fp32, in a fixed order."""
    return (_b._host or _b._native()).relative_bias(table, _map_for(table, buckets), q_len, k_len, q_start)


def dropout_add(x: torch.Tensor, residual: Optional[torch.Tensor], p: float, rng: torch.Tensor, stream: int = 0) -> torch.Tensor:
    """residual + dropout(x) (residual may be None); bf16 or fp32.  `rng` is an int64 device tensor {seed, offset} that the kernel
    reads when it runs (a captured graph draws anew if the program changes it in between); the backward pass uses the values
    the forward pass had.  The mask is a function of seed, offset (its low 32 bits), `stream` and the element's place, and is
    never stored; p is taken in steps of 2^-16.  Differentiable with respect to x and residual."""
    return (_b._host or _b._native()).dropout_add(x, residual, p, rng, stream)
