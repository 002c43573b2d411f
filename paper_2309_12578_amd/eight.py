"""Root-mean-square norm, and activations kept in 8 bits for the backward pass.  Argument handling only; the operators are kernels of the library
(csrc/rms_norm_kernels.hip, csrc/weight_grad_eight_kernels.hip), their autograd nodes native (csrc/host_ext.cpp)."""
from __future__ import annotations

import dataclasses
from typing import Optional, Tuple

import torch

from . import binding as _b

GROUP = 64   # elements of a row that share a scale


@dataclasses.dataclass(frozen=True)
class Packed8:
    """Rows of `size` elements in 8 bits: codes int8 [..., P] with P the next multiple of 64, exponents uint8 [..., P / 64].  An element is
    code * 2^(exponent - 127) * weight of its column (None: 1); a group of exponent 255 held an infinity or NaN and stands for NaN."""
    codes: torch.Tensor
    exponents: torch.Tensor
    size: int
    weight: Optional[torch.Tensor] = None

    def __post_init__(self):
        pitch = (self.size + GROUP - 1) // GROUP * GROUP
        if self.size < 1 or self.codes.dtype != torch.int8 or self.codes.dim() < 1 or self.codes.shape[-1] != pitch:
            raise ValueError("codes must be int8 [..., P], P the multiple of 64 from size on")
        if self.exponents.dtype != torch.uint8 or self.exponents.shape != (*self.codes.shape[:-1], pitch // GROUP):
            raise ValueError("exponents must be uint8 [..., P / 64]")
        if self.weight is not None and self.weight.shape != (self.size,):
            raise ValueError("weight must be [size]")

    @property
    def shape(self) -> torch.Size:
        return torch.Size((*self.codes.shape[:-1], self.size))


def _packed(codes: torch.Tensor, exponents: torch.Tensor, size: int, weight: Optional[torch.Tensor] = None) -> Packed8:
    """What an operator made, without the checks, which take 4 us, about as long as a call for a token."""
    if torch.compiler.is_compiling():   # torch.compile follows how a dataclass is made, not this
        return Packed8(codes, exponents, size, weight)
    p = object.__new__(Packed8)
    d = p.__dict__
    d["codes"], d["exponents"], d["size"], d["weight"] = codes, exponents, size, weight
    return p


def pack8(x: torch.Tensor) -> Packed8:
    """x [..., D] (bf16 or fp32) in 8 bits.  A row goes in groups of 64; a group's scale is the smallest power of two 2^k with max |x| <= 127 * 2^k, at
    least 2^-126, a code is rint(x / 2^k), ties to even: exact but for that rounding, at most 2^-7 of the group's largest element, and the same on every machine.
    Not differentiable."""
    codes, exponents = (_b._host or _b._native()).pack8(x)
    return _packed(codes, exponents, x.shape[-1])


def unpack8(p: Packed8, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """What p stands for, [..., size] of `dtype` (bf16 or fp32), rounded once; without a weight both hold it exactly.  Not
    differentiable."""
    return (_b._host or _b._native()).unpack8(p.codes, p.exponents, p.weight, p.size, _b._dtype_code(dtype))


def rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6, checkpoint: bool = False
             ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[Packed8]]:
    """(y, h, p) of rows x [..., D], D up to 16384 (bf16 or fp32, weight [D] and residual of the same type): with s = x + residual and
    z = s / sqrt(mean(s^2) + eps), y = z * weight and h = s, the stream that goes on (None without a residual).
    checkpoint: p is z in 8 bits with `weight` as its weight, so that it stands for y; the backward pass then takes z from p's codes and keeps
    neither x nor h, and `linear8` may keep the same codes (else p is None).
    y is a tensor of x's type, and so is its gradient: in bf16 both are rounded on their way between the norm and what takes y.
    Differentiable with respect to x, weight and residual, through y and h."""
    y, h, codes, exponents = (_b._host or _b._native()).rms_norm(x, weight, residual, eps, checkpoint)
    return y, h, None if codes is None else _packed(codes, exponents, x.shape[-1], weight.detach())


def rms_norm8(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6
              ) -> Tuple[Packed8, Optional[torch.Tensor]]:
    """(p, h): as `rms_norm`, with y itself in 8 bits and in no other form.  For inference: not differentiable, inputs that require a gradient are refused
    while gradients are recorded."""
    codes, exponents, h = (_b._host or _b._native()).rms_norm8(x, weight, residual, eps)
    return _packed(codes, exponents, x.shape[-1]), h


def linear8(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, checkpoint: Optional[Packed8] = None) -> torch.Tensor:
    """x weight^T + bias (bf16 or fp32, one type), whose graph keeps x in 8 bits: the weight's gradient is made from the codes, x's and the bias'
    are not touched by it.  checkpoint: codes that stand for x already, such as those of the norm before (the caller's word for it; shapes are
    looked at); without it x is packed, if the weight needs a gradient.  Autocast changes no types here (SparseMHA casts for it)."""
    c = (None, None, None) if checkpoint is None else (checkpoint.codes, checkpoint.exponents, checkpoint.weight)
    if checkpoint is not None and checkpoint.size != (x.shape or (0,))[-1]:   # (the other sizes are the codes')
        raise ValueError("the checkpoint must have x's shape")
    return (_b._host or _b._native()).linear8(x, weight, bias, *c)
