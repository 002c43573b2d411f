"""The sparse multi-head-attention sub-layer of Algorithm 5 as a torch module.

Glue around the library: the four projections (hipBLASLt GEMMs but for the weight gradients) are torch ops, and so are
dropout and the residual unless the caller gives the state to draw from; LayerNorm is the library's, and the head split
and lines 4-7 of Algorithm 5 (SDDMM, sparse softmax, SpMM for every head) are one call into it, forward and backward.
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import torch
from torch import nn
from torch.nn.modules import module as _module

from . import binding as _b
from .autograd import sparse_attention
from .eight import Packed8, linear8, rms_norm
from .extras import RelativeBuckets, _map_for, dropout_add
from .rotary import RotaryAxes

HEAD_DIM = 64   # the only head dimension the kernels are built for


class _Norm(nn.LayerNorm):
    """nn.LayerNorm by the library's kernels (csrc/norm_kernels.hip) where they take the call."""

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        y = None
        if x.is_cuda and self.weight is not None and self.bias is not None and not torch.compiler.is_compiling():
            y = (_b._host or _b._native()).layer_norm(x, self.weight, self.bias, self.eps)
        return super().forward(x) if y is None else y


class _RmsNorm(nn.Module):
    """rms_norm with its weight."""

    def __init__(self, dim: int, eps: float = 1e-6, device=None, dtype=None):
        super().__init__()
        self.eps = eps
        self.weight = nn.Parameter(torch.ones(dim, device=device, dtype=dtype))

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, checkpoint: bool = False):
        dtype = self.weight.dtype
        if (x.dtype != dtype or residual is not None and residual.dtype != dtype) and torch.is_autocast_enabled():
            # in the weight's type, as LayerNorm under autocast in fp32
            x, residual = x.to(dtype), None if residual is None else residual.to(dtype)
        return rms_norm(x, self.weight, residual, self.eps, checkpoint)


class _Projection(nn.Linear):
    """nn.Linear whose bf16 weight gradient, few outputs and a sum over every token, is a kernel of the
    library (csrc/projection_kernels.hip); with `eight_bit`, linear8."""

    eight_bit = False

    def forward(self, x: torch.Tensor, checkpoint: Optional[Packed8] = None) -> torch.Tensor:
        if self.eight_bit:
            weight, bias = self.weight, self.bias
            if torch.is_autocast_enabled():   # in autocast's type, as nn.Linear; linear8 takes its operands' own
                dtype = torch.get_autocast_dtype("cuda")
                x, weight, bias = x.to(dtype), weight.to(dtype), None if bias is None else bias.to(dtype)
                if checkpoint is not None and checkpoint.weight is not None:   # (a rounding of the codes' factors, 2^-8 of them at most in bf16, beside the codes' own 2^-7)
                    checkpoint = dataclasses.replace(checkpoint, weight=checkpoint.weight.to(dtype))
            return linear8(x, weight, bias, checkpoint)
        y = None
        if x.is_cuda and not torch.compiler.is_compiling():
            y = (_b._host or _b._native()).projection(x, self.weight, self.bias)
        return super().forward(x) if y is None else y


def _runs(module: nn.Module, forward) -> bool:
    """Whether a call of the module runs that forward, neither a subclass's nor one set on the instance."""
    return getattr(type(module), "forward", None) is forward and "forward" not in module.__dict__


def _hands_on(projection: nn.Module) -> bool:
    """Whether code other than _Projection's is handed the projection's input or output (a hook, another forward): it may
    change them in place, also where no version counter tells, while the attention beside it has saved them."""
    if not _runs(projection, _Projection.forward):
        return True
    d = projection.__dict__
    return bool(d["_forward_pre_hooks"] or d["_forward_hooks"] or _module._global_forward_pre_hooks or _module._global_forward_hooks)


class SparseMHA(nn.Module):
    """O = dropout(concat_h(sparse_attention(Q_h, K_h, V_h, P)) W^O) + E with
    Q, K, V = LayerNorm(E) W^{Q,K,V} (Algorithm 5).  `embed_dim` must be 64 * heads.

    buckets: adds a learned relative position bias, `bias_table` [buckets.count, heads], to the scores; it starts at 0.
    attn_dropout: dropout of the probabilities while training; it draws from the `rng` of the call.
    norm: "layer", or "rms" for the root-mean-square norm (`rms_norm`), which also takes the residual of the sub-layer before.
    rotary: turns queries and keys by their positions (`rotary`), heads of 64.
    eight_bit: the graph keeps the input of the joint projection, and with the "rms" norm that of the norm by the same codes, in 8 bits (`linear8`)."""

    def __init__(self, embed_dim: int, heads: int, dropout: float = 0.0, bias: bool = False,
                 device=None, dtype=None, *, buckets: Optional[RelativeBuckets] = None, attn_dropout: float = 0.0, norm: str = "layer",
                 rotary: Optional[RotaryAxes] = None, eight_bit: bool = False):
        super().__init__()
        if norm not in ("layer", "rms"):
            raise ValueError("norm must be 'layer' or 'rms'")
        if rotary is not None and rotary.head_dim != HEAD_DIM:
            raise ValueError("rotary axes must be of heads of %d" % HEAD_DIM)
        if embed_dim != heads * HEAD_DIM:
            raise ValueError("embed_dim must be %d * heads" % HEAD_DIM)
        if not 0.0 <= attn_dropout < 1.0:
            raise ValueError("attn_dropout must be a probability below 1")
        kw = dict(device=device, dtype=dtype)
        self.heads = heads
        self.norm = _Norm(embed_dim, **kw) if norm == "layer" else _RmsNorm(embed_dim, **kw)
        self.w_qkv = _Projection(embed_dim, 3 * embed_dim, bias=bias, **kw)   # W^Q | W^K | W^V
        self.w_qkv.eight_bit = eight_bit
        self.w_o = _Projection(embed_dim, embed_dim, bias=bias, **kw)   # (its input the attention keeps as well)
        self.drop = nn.Dropout(dropout)
        self.attn_dropout = attn_dropout
        self.bias_table = None if buckets is None else nn.Parameter(torch.zeros(buckets.count, heads, **kw))
        self.register_buffer("bucket_map", None if buckets is None else buckets.map.to(device), persistent=False)
        self._axes = (0, False) if rotary is None else (rotary.count, rotary.neighbours)
        self.register_buffer("turns", None if rotary is None else rotary.turns.to(device), persistent=False)
        self.register_buffer("axis_of", None if rotary is None else rotary.axis_of.to(device), persistent=False)

    @property
    def buckets(self) -> Optional[RelativeBuckets]:
        """Of the bias table, on the module's device."""
        if self.bias_table is None:
            return None
        # .data: with a version counter of its own, since DistributedDataParallel writes buffers, with what they hold, at every forward pass
        return RelativeBuckets((self.bucket_map.numel() + 1) // 2, self.bias_table.shape[0], self.bucket_map.data)

    @property
    def rotary(self) -> Optional[RotaryAxes]:
        """On the module's device."""
        if self.turns is None:
            return None
        return RotaryAxes(HEAD_DIM, self._axes[0], self.turns.data, self.axis_of.data, self._axes[1])

    def forward(self, E: torch.Tensor, pattern: _b.Pattern, flags: int = 0, *, lengths: Optional[torch.Tensor] = None,
                rng: Optional[torch.Tensor] = None, stream: int = 0, positions: Optional[torch.Tensor] = None,
                residual: Optional[torch.Tensor] = None):
        """E: [B, L, embed_dim] on the GPU (bf16 or fp32); pattern: the layer's sparsity pattern.
        lengths: int32 [B], the tokens of each sequence, see `sparse_attention`; rows from there on leave as they came, but
        for w_o's bias, and have to be finite (the projections' gradients add them up, times 0).
        rng, stream: int64 tensor {seed, offset} and a number of the layer's own, from which both dropouts then draw, see
        `dropout_add`; without it the last one is torch's.
        positions: int32 or int64 [axes, L] or [axes, B, L], see `rotary`; one axis counts from 0 if they are not given.
        residual: with the "rms" norm, the stream that E, the branch of the sub-layer before, is to be added to.  The result then is (branch,
        stream), not their sum: the next sub-layer's E and residual."""
        B, L, D = E.shape
        w_qkv, w_o, norm, turns = self.w_qkv, self.w_o, self.norm, self.turns
        if positions is not None and turns is None:
            raise ValueError("positions are for a sub-layer with rotary axes")
        attn_dropout = self.attn_dropout if self.training else 0.0
        plain = self.bias_table is None and lengths is None and attn_dropout == 0.0
        if not plain and flags:
            raise ValueError("flags are not supported together with a bias, lengths or dropout")
        S, R, checkpoint = None, E, None
        if isinstance(norm, _RmsNorm):
            # a hook, or another forward, may change what the norm's codes stand for before the projection has it (global hooks: _hands_on)
            shares = (not _hands_on(w_qkv) and w_qkv.eight_bit and torch.is_grad_enabled() and not norm._forward_hooks and
                      _runs(norm, _RmsNorm.forward))   # (_hands_on first: the module in w_qkv's place may be any)
            X, h, checkpoint = norm(E, residual, shares)
            R = E if residual is None else h
        elif residual is not None:
            raise ValueError("a residual goes into the 'rms' norm only")
        else:
            X = norm(E)
        qkv = w_qkv(X) if checkpoint is None else w_qkv(X, checkpoint)
        if qkv.is_cuda and not torch.compiler.is_compiling():
            host = _b._host or _b._native()
            if residual is None:
                R = host.residual(E, X)   # E, its gradient added up in the norm's pass
            if turns is not None:
                qkv = self._turned(qkv, positions)
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
        elif turns is not None:
            qkv = self._turned(qkv, positions)
        if S is None:
            qkv = qkv.view(B, L, 3, self.heads, HEAD_DIM)
            # [B, H, L, 64] contiguous per tensor: the layout the kernels take
            Q, K, V = [qkv[:, :, i].transpose(1, 2).contiguous() for i in range(3)]
            S = sparse_attention(Q, K, V, pattern, flags=flags, bias=self.bias_table, buckets=self.buckets, lengths=lengths,
                                 dropout=attn_dropout, rng=rng, stream=stream)   # lines 4-7, all heads at once
            S = S.transpose(1, 2).reshape(B, L, D)                            # concatenate the heads
        branch = w_o(S)
        draws = rng is not None and self.training and self.drop.p > 0.0
        if residual is not None:
            branch = branch.to(R.dtype)   # (autocast)
            return (dropout_add(branch, None, self.drop.p, rng, stream) if draws else self.drop(branch)), R
        if draws:
            return dropout_add(branch.to(R.dtype), R, self.drop.p, rng, stream)
        return self.drop(branch) + R

    def _turned(self, qkv: torch.Tensor, positions: Optional[torch.Tensor]) -> torch.Tensor:
        """Queries and keys, the first two thirds of the heads beside each other in qkv, turned by their positions."""
        count, neighbours = self._axes
        if positions is None:
            if count != 1:
                raise ValueError("positions of %d axes are missing" % count)
            positions = torch.arange(qkv.shape[1], device=qkv.device)[None]
        # (as `rotary`, without another RotaryAxes a call)
        return (_b._host or _b._native()).rotary(qkv, self.turns.data, self.axis_of.data, positions, count, 2 * self.heads, neighbours)
