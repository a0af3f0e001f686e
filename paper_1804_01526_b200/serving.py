"""A trained dense layer for serving: its product in 8-bit integers with a scale for each token and channel.

Training keeps the weights in block floating point (``HbfpLinear``); a network that is only run is served with one integer
product per layer (``hbfp_int8_gemm``): the weights are converted once, one FP32 scale per output channel, the activations by
every call, one scale per token. Between such layers attention reads a cache held in 4-bit block floating point
(``binding.kv4_append``, ``binding.kv4_attention``), whose calls take the layers' outputs as they are, slices of a fused projection
among them.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as hb
from .autograd import HbfpLinear


class _Int8LinearFn(torch.autograd.Function):
    """The layer as a Python function, for what has to see one: a trace records it, forward mode and transforms refuse it."""

    @staticmethod
    def forward(ctx, x, layer):
        y = layer._product(x, hb.int8_gemm_recorded)
        ctx.mark_non_differentiable(y)
        return y


class Int8Linear(torch.nn.Module):
    """``y = x W + b`` for inference, W ``[fin][fout]`` held as 8-bit integers; no gradients. It can be traced; the trace calls this
    layer's product, on tokens of any number."""

    def __init__(self, weight: torch.Tensor, bias: Optional[torch.Tensor] = None):
        """``weight`` [fin][fout]: float32, bfloat16 or float16 on the GPU, in any order, converted here; ``bias`` [fout], kept as float32."""
        super().__init__()
        self.fin, self.fout = weight.shape
        rows = hb.int8_quantize(weight.detach().contiguous(), 0)
        self.register_buffer("weight_q", rows.q)
        self.register_buffer("weight_scale", rows.scale)
        self.register_buffer("bias", None if bias is None else bias.detach().float().contiguous())

    def _apply(self, fn, *args, **kwargs):
        """Moves like any module; scales and bias stay float32 where the module is given another type (``module.half()``)."""
        kept = {n: b for n, b in (("weight_scale", self.weight_scale), ("bias", self.bias)) if b is not None}
        super()._apply(fn, *args, **kwargs)
        for n, b in kept.items():
            setattr(self, n, b.to(self.weight_q.device))
        return self

    @classmethod
    def from_hbfp(cls, layer: HbfpLinear) -> "Int8Linear":
        """The layer with the value of a trained ``HbfpLinear``'s weights."""
        return cls(layer.weight, layer.bias)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """x [..][fin] float32, bfloat16 or float16; the result has its type. Leading extents that are one run of rows, each of
        neighbouring values, are taken as they are; other orders (transposed, broadcast) are copied first."""
        return _Int8LinearFn.apply(x, self) if hb.host().recorded(x) else self._product(x, hb.int8_gemm)

    def _product(self, x: torch.Tensor, gemm) -> torch.Tensor:
        if x.dim() == 0 or x.shape[-1] != self.fin:
            raise ValueError(f"x must end in an extent of {self.fin}")
        rows = x.detach().flatten(0, -2) if x.dim() > 1 else x.detach()[None]
        if rows.stride(1) != 1 or rows.stride(0) < self.fin:
            rows = rows.contiguous()
        y = gemm(rows, hb.Int8Rows(self.weight_q, self.weight_scale, self.fin), bias=self.bias)
        return y.view(*x.shape[:-1], self.fout)
