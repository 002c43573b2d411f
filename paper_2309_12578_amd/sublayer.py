"""The sparse multi-head-attention sub-layer of Algorithm 5 as a torch module.

Glue around the library: the four projections (hipBLASLt GEMMs but for the weight gradients) are torch ops, and so are
dropout and the residual unless the caller gives the state to draw from; LayerNorm is the library's, and the head split
and lines 4-7 of Algorithm 5 (SDDMM, sparse softmax, SpMM for every head) are one call into it, forward and backward.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch import nn
from torch.nn.modules import module as _module

from . import binding as _b
from .autograd import sparse_attention
from .extras import RelativeBuckets, _map_for, dropout_add

HEAD_DIM = 64   # the only head dimension the kernels are built for


class _Norm(nn.LayerNorm):
    """nn.LayerNorm by the library's kernels (csrc/norm_kernels.hip) where they take the call."""

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        y = None
        if x.is_cuda and self.weight is not None and self.bias is not None and not torch.compiler.is_compiling():
            y = (_b._host or _b._native()).layer_norm(x, self.weight, self.bias, self.eps)
        return super().forward(x) if y is None else y


class _Projection(nn.Linear):
    """nn.Linear whose bf16 weight gradient, few outputs and a sum over every token, is a kernel of the
    library (csrc/projection_kernels.hip)."""

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        y = None
        if x.is_cuda and not torch.compiler.is_compiling():
            y = (_b._host or _b._native()).projection(x, self.weight, self.bias)
        return super().forward(x) if y is None else y


def _hands_on(projection: nn.Module) -> bool:
    """Whether code other than _Projection's is handed the projection's input or output (a hook, another forward): it may
    change them in place, also where no version counter tells, while the attention beside it has saved them."""
    if getattr(type(projection), "forward", None) is not _Projection.forward:
        return True
    d = projection.__dict__
    return bool(d["_forward_pre_hooks"] or d["_forward_hooks"] or "forward" in d or
                _module._global_forward_pre_hooks or _module._global_forward_hooks)


class SparseMHA(nn.Module):
    """O = dropout(concat_h(sparse_attention(Q_h, K_h, V_h, P)) W^O) + E with
    Q, K, V = LayerNorm(E) W^{Q,K,V} (Algorithm 5).  `embed_dim` must be 64 * heads.

    buckets: adds a learned relative position bias, `bias_table` [buckets.count, heads], to the scores; it starts at 0.
    attn_dropout: dropout of the probabilities while training; it draws from the `rng` of the call."""

    def __init__(self, embed_dim: int, heads: int, dropout: float = 0.0, bias: bool = False,
                 device=None, dtype=None, *, buckets: Optional[RelativeBuckets] = None, attn_dropout: float = 0.0):
        super().__init__()
        if embed_dim != heads * HEAD_DIM:
            raise ValueError("embed_dim must be %d * heads" % HEAD_DIM)
        if not 0.0 <= attn_dropout < 1.0:
            raise ValueError("attn_dropout must be a probability below 1")
        kw = dict(device=device, dtype=dtype)
        self.heads = heads
        self.norm = _Norm(embed_dim, **kw)
        self.w_qkv = _Projection(embed_dim, 3 * embed_dim, bias=bias, **kw)   # W^Q | W^K | W^V
        self.w_o = _Projection(embed_dim, embed_dim, bias=bias, **kw)
        self.drop = nn.Dropout(dropout)
        self.attn_dropout = attn_dropout
        self.bias_table = None if buckets is None else nn.Parameter(torch.zeros(buckets.count, heads, **kw))
        self.register_buffer("bucket_map", None if buckets is None else buckets.map.to(device), persistent=False)

    @property
    def buckets(self) -> Optional[RelativeBuckets]:
        """Of the bias table, on the module's device."""
        if self.bias_table is None:
            return None
        # .data: with a version counter of its own, since DistributedDataParallel writes buffers, with what they hold, at every forward pass
        return RelativeBuckets((self.bucket_map.numel() + 1) // 2, self.bias_table.shape[0], self.bucket_map.data)

    def forward(self, E: torch.Tensor, pattern: _b.Pattern, flags: int = 0, *, lengths: Optional[torch.Tensor] = None,
                rng: Optional[torch.Tensor] = None, stream: int = 0) -> torch.Tensor:
        """E: [B, L, embed_dim] on the GPU (bf16 or fp32); pattern: the layer's sparsity pattern.
        lengths: int32 [B], the tokens of each sequence, see `sparse_attention`; rows from there on leave as they came, but
        for w_o's bias, and have to be finite (the projections' gradients add them up, times 0).
        rng, stream: int64 tensor {seed, offset} and a number of the layer's own, from which both dropouts then draw, see
        `dropout_add`; without it the last one is torch's."""
        B, L, D = E.shape
        w_qkv, w_o = self.w_qkv, self.w_o
        attn_dropout = self.attn_dropout if self.training else 0.0
        plain = self.bias_table is None and lengths is None and attn_dropout == 0.0
        if not plain and flags:
            raise ValueError("flags are not supported together with a bias, lengths or dropout")
        X = self.norm(E)
        qkv = w_qkv(X)
        S, R = None, E
        if qkv.is_cuda and not torch.compiler.is_compiling():
            host = _b._host or _b._native()
            R = host.residual(E, X)   # E, its gradient added up in LayerNorm's pass
            # lines 4-7 for every head, on the heads as they lie in qkv
            index = (qkv, self.heads, pattern.row_ptr, pattern.col_idx, pattern.col_ptr, pattern.row_idx, pattern.bsr_pos,
                     pattern.nnzb, pattern.block)
            apart = _hands_on(w_qkv) or _hands_on(w_o)
            if plain:
                S = host.heads_attention(*index, flags, apart)
            else:
                S = host.heads_attention_with(
                    *index, apart, self.bias_table, None if self.bias_table is None else _map_for(self.bias_table, self.buckets, L),
                    lengths, attn_dropout, rng, stream)
        if S is None:
            qkv = qkv.view(B, L, 3, self.heads, HEAD_DIM)
            # [B, H, L, 64] contiguous per tensor: the layout the kernels take
            Q, K, V = [qkv[:, :, i].transpose(1, 2).contiguous() for i in range(3)]
            S = sparse_attention(Q, K, V, pattern, flags=flags, bias=self.bias_table, buckets=self.buckets, lengths=lengths,
                                 dropout=attn_dropout, rng=rng, stream=stream)   # lines 4-7, all heads at once
            S = S.transpose(1, 2).reshape(B, L, D)                            # concatenate the heads
        if rng is not None and self.training and self.drop.p > 0.0:
            return dropout_add(w_o(S).to(R.dtype), R, self.drop.p, rng, stream)
        return self.drop(w_o(S)) + R
