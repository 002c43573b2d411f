"""torch.autograd front end of the sparse attention (Section 4.3, "Integration of GPU kernels with
PyTorch": the shared library is loaded once and a custom autograd function calls its forward and
backward entry points).  Glue only: the autograd node is native (csrc/host_ext.cpp), under torch.jit.trace a
Python function that the tracer records, and both directions run in libspion's kernels."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as _b
from .extras import RelativeBuckets, _map_for


class _TracedAttention(torch.autograd.Function):
    """The same calls as the native node, as an operator of a traced graph."""

    @staticmethod
    def forward(ctx, Q, K, V, pattern, scale, flags):
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
        O = torch.empty_like(Q)   # the tracer asks for a tensor that an operator of torch made
        O, LSE = _b.attn_fwd(Q, K, V, pattern, scale=scale, flags=flags, O=O)
        ctx.save_for_backward(Q, K, V, O, LSE)
        ctx.pattern, ctx.scale, ctx.flags = pattern, scale, flags
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, O, LSE = ctx.saved_tensors
        return *_b.attn_bwd(Q, K, V, O, dO.contiguous(), LSE, ctx.pattern, scale=ctx.scale, flags=ctx.flags), None, None, None


def sparse_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, pattern: _b.Pattern,
                     scale: float = 0.0, flags: int = 0, *, bias: Optional[torch.Tensor] = None,
                     buckets: Optional[RelativeBuckets] = None, lengths: Optional[torch.Tensor] = None,
                     dropout: float = 0.0, rng: Optional[torch.Tensor] = None, stream: int = 0) -> torch.Tensor:
    """Eq. 5 on the kept blocks of `pattern` for Q, K, V of shape [B, H, L, 64] (bf16 or fp32);
    differentiable with respect to Q, K and V.

    bias, buckets: a table [buckets, H] (bf16 or fp32) of biases by the distance key - query, added to the scores inside the
    softmax; differentiable as well (one that needs no gradient costs nearly the same).  A bias of -infinity, or down from -1e30, masks.
    lengths: int32 [B], the tokens of each sequence; keys from there on are masked, rows from there on are 0, gradients too.
    dropout, rng, stream: dropout of the probabilities, see `dropout_add`.
    In bf16 the graph keeps a second tensor of O's size, what rounding left of O: the gradients are made from both.
    With any of them flags must be 0, and second derivatives, tracing and transforms are refused."""
    if bias is None and buckets is not None:
        raise ValueError("buckets are those of a bias table, which is missing")
    if bias is None and lengths is None and dropout == 0.0:
        O = (_b._host or _b._native()).sparse_attention(
            Q, K, V, pattern.row_ptr, pattern.col_idx, pattern.col_ptr, pattern.row_idx, pattern.bsr_pos, pattern.nnzb,
            pattern.block, scale, flags)
        return _TracedAttention.apply(Q, K, V, pattern, scale, flags) if O is None else O
    if flags:
        raise ValueError("flags are not supported together with a bias, lengths or dropout")
    return (_b._host or _b._native()).sparse_attention_with(
        Q, K, V, pattern.row_ptr, pattern.col_idx, pattern.col_ptr, pattern.row_idx, pattern.bsr_pos, pattern.nnzb, pattern.block,
        scale, bias, None if bias is None else _map_for(bias, buckets, Q.shape[-2]), lengths, dropout, rng, stream)
