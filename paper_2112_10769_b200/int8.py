"""Answering with a trained model in 8 bits, as modules.

A layer's weight is quantized once, with a scale for each output channel; tokens are quantized on the way into every
product, with a scale each; the products run on the tensor cores' int8 path and leave in the type of the tokens.

    Int8Linear     one weight (from a tensor, ``torch.nn.Linear`` or ``autograd.LuqLinear``), optionally with the
                   layer norm before it in the same call
    Int8Experts    one weight per expert; the rows of an expert follow one another, their numbers stay on the device

These modules compute forward passes only.  Argument handling: every step runs in the library's kernels.
"""
from __future__ import annotations

import torch

from . import autograd


def quantize_weight(w: torch.Tensor):
    """int8 codes and the scale of each output channel of a weight ``[.., N, K]`` (float32 or bfloat16)."""
    lib = autograd.context(w.device)
    if w.dim() == 2:
        return lib.quant_int8_rows(w.detach())
    codes, scale = lib.quant_int8_rows(w.detach().reshape(-1, w.shape[-1]))
    ld = codes.stride(0)
    return codes.as_strided(w.shape, (w.shape[-2] * ld, ld, 1)), scale.view(w.shape[:-1])


def _snapshot(t: torch.Tensor | None):
    """A parameter as it is now, in 32 bits and in memory of its own."""
    return None if t is None else t.detach().to(torch.float32, copy=True).contiguous()


class _Int8Module(autograd.KeepsFloat32):
    """Codes keep rows that start at multiples of 16 bytes: a move or a copy packs them."""

    def _kept(self, t: torch.Tensor) -> torch.Tensor:
        t = super()._kept(t)
        if t.dtype != torch.int8 or (t.stride(-1) == 1 and all(s % 16 == 0 for s in t.stride()[:-1]) and t.data_ptr() % 16 == 0):
            return t
        rows = torch.empty((*t.shape[:-1], -(-t.shape[-1] // 16) * 16), dtype=torch.int8, device=t.device)[..., :t.shape[-1]]
        return rows.copy_(t)


class Int8Linear(_Int8Module):
    """``torch.nn.Linear`` in 8 bits.  ``norm``: a layer norm module (``autograd.LayerNorm`` or
    ``torch.nn.LayerNorm`` over the last dimension) that is applied to the tokens first, in the same call."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None, norm: torch.nn.Module | None = None):
        super().__init__()
        codes, scale = quantize_weight(weight)
        self.register_buffer("codes", codes)
        self.register_buffer("scale", scale)
        self.register_buffer("bias", _snapshot(bias))
        self.eps = None
        if norm is not None:
            if tuple(norm.normalized_shape) != (weight.shape[-1],):
                raise ValueError("the layer norm has to run over the inputs of the layer")
            self.eps = float(norm.eps)
            self.register_buffer("norm_weight", _snapshot(norm.weight))
            self.register_buffer("norm_bias", _snapshot(norm.bias))

    @classmethod
    def of(cls, layer: torch.nn.Module, norm: torch.nn.Module | None = None) -> "Int8Linear":
        """From a module with ``weight`` [N, K] and, maybe, ``bias``."""
        return cls(layer.weight, getattr(layer, "bias", None), norm)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        lib = autograd.context(x.device)
        if self.eps is None:
            z = lib.quant_int8_gemm(x, self.codes, self.scale, self.bias)
        else:
            z = lib.layer_norm_int8_gemm(x, self.norm_weight, self.norm_bias, self.eps, self.codes, self.scale, self.bias)
        return z if x.dim() == 2 else z.reshape(*x.shape[:-1], z.shape[-1])


class Int8Experts(_Int8Module):
    """One weight per expert, ``[E, N, K]``.  ``forward(x, offsets)``: rows ``offsets[e] .. offsets[e + 1] - 1`` of x
    belong to expert e (``offsets``: int32 on the device, E + 1 numbers); rows that belong to none are not written."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None):
        super().__init__()
        codes, scale = quantize_weight(weight)
        self.register_buffer("codes", codes)
        self.register_buffer("scale", scale)
        self.register_buffer("bias", _snapshot(bias))

    def forward(self, x: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
        return autograd.context(x.device).quant_int8_gemm_grouped(x, offsets, self.codes, self.scale, self.bias)

    def route(self, x: torch.Tensor, expert: torch.Tensor) -> torch.Tensor:
        """Rows in any order: ``expert`` [M] names each row's expert; the result comes in the order of x."""
        order = torch.argsort(expert, stable=True)
        counts = torch.bincount(expert, minlength=self.codes.shape[0])
        offsets = torch.zeros(self.codes.shape[0] + 1, dtype=torch.int32, device=x.device)
        offsets[1:] = counts.cumsum(0)
        z = torch.empty(x.shape[0], self.codes.shape[1], dtype=x.dtype, device=x.device)
        z[order] = self.forward(x[order], offsets)
        return z
