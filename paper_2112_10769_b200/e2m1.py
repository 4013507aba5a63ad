"""Answering with a trained model in microscaled 4-bit floating point, as modules.

A layer's weight is quantized once: e2m1 numbers with a scale for each block of 16 (e4m3, and a float32 scale for each
output channel) or of 32 (powers of two).  Tokens are quantized on the way into every product, which the tensor cores
make of the 4-bit numbers and their scales; results leave in the type of the tokens.

    E2m1Linear     one weight (from a tensor, ``torch.nn.Linear`` or ``autograd.LuqLinear``)
    E2m1Experts    one weight per expert, for tokens sorted by expert or for tokens and the positions of their copies

These modules compute forward passes only.  Argument handling: every step runs in the library's kernels.
"""
from __future__ import annotations

import torch

from . import autograd
from .int8 import _snapshot

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _check_block(block: int) -> None:
    if block not in (16, 32):
        raise ValueError("blocks are of 16 or 32 numbers")


def quantize_weight(w: torch.Tensor, block: int = 16):
    """(codes [.., N, ceil(K / 2)], tiles, row scales [.., N] or None) of a weight ``[.., N, K]`` (float32 or bfloat16)."""
    _check_block(block)
    lead = w.shape[:-2]
    planes = lead.numel()
    codes, tiles, scale = autograd.context(w.device).quant_e2m1_rows(w.detach().reshape(-1, w.shape[-1]), block, max(planes, 1))
    ld = codes.stride(0)
    if lead:
        strides, step = [], w.shape[-2] * ld
        for n in reversed(lead):
            strides.insert(0, step)
            step *= n
        codes = codes.as_strided((*lead, w.shape[-2], codes.shape[1]), (*strides, ld, 1))
        scale = None if scale is None else scale.view(w.shape[:-1])
    return codes, tiles, scale


def scale_tiles(scales: torch.Tensor, block: int = 16) -> torch.Tensor:
    """Block scales as bytes ``[.., rows, ceil(K / block)]`` (e4m3 for blocks of 16, power-of-two exponents + 127 for blocks of 32)
    in the tiles of 128 rows x 4 blocks that the products read: ``[rows of tiles, tiles along a row, 512]``."""
    _check_block(block)
    s = scales.view(torch.uint8) if scales.dtype != torch.uint8 else scales
    *lead, rows, blocks = s.shape
    s = torch.nn.functional.pad(s, (0, -blocks % 4, 0, -rows % 128))
    t = s.reshape(-1, s.shape[-2] // 128, 4, 32, s.shape[-1] // 4, 4)        # plane, tile row, 32-row part, row, tile, block
    return t.permute(0, 1, 4, 3, 2, 5).reshape(-1, s.shape[-1] // 4, 512).contiguous()


def scale_rows(tiles: torch.Tensor, rows: int, cols: int, block: int = 16) -> torch.Tensor:
    """The inverse of ``scale_tiles`` for one matrix: bytes ``[rows, ceil(cols / block)]``."""
    _check_block(block)
    t = tiles.view(-1, tiles.shape[1], 32, 4, 4).permute(0, 3, 2, 1, 4)      # tile row, 32-row part, row, tile, block
    return t.reshape(tiles.shape[0] * 128, -1)[:rows, :-(-cols // block)]


def values(codes: torch.Tensor, tiles: torch.Tensor, row_scale: torch.Tensor | None, cols: int, block: int = 16) -> torch.Tensor:
    """What a quantized matrix ``[rows, cols]`` stands for, in 64 bits: for checks and for moving weights elsewhere."""
    _check_block(block)
    rows = codes.shape[0]
    levels = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64, device=codes.device)
    q = levels[torch.stack([codes & 15, codes >> 4], 2).view(rows, -1)[:, :cols].long()]
    s = scale_rows(tiles, rows, cols, block).contiguous()
    if block == 16:
        s = (s & 127).view(torch.float8_e4m3fn).double() * row_scale.double()[:, None]      # (scales have no sign)
    else:
        s = torch.where(s == 255, torch.nan, torch.exp2(s.double() - 127))
    return q * s.repeat_interleave(block, 1)[:, :cols]


class _E2m1Module(autograd.KeepsFloat32):
    """Codes keep rows that start at multiples of 16 bytes: a move or a copy packs them."""

    def _kept(self, t: torch.Tensor) -> torch.Tensor:
        t = super()._kept(t)
        if t.dtype != torch.uint8 or t.dim() < 2 or (t.stride(-1) == 1 and all(s % 16 == 0 for s in t.stride()[:-1]) and t.data_ptr() % 16 == 0):
            return t
        rows = torch.empty((*t.shape[:-1], -(-t.shape[-1] // 16) * 16), dtype=torch.uint8, device=t.device)[..., :t.shape[-1]]
        return rows.copy_(t)

    def _quantize(self, weight: torch.Tensor, bias: torch.Tensor | None, block: int):
        codes, tiles, scale = quantize_weight(weight, block)
        self.block = block
        self.register_buffer("codes", codes)
        self.register_buffer("tiles", tiles)
        self.register_buffer("scale", scale)
        self.register_buffer("bias", _snapshot(bias))


class E2m1Linear(_E2m1Module):
    """``torch.nn.Linear`` in microscaled 4-bit floating point."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None, block: int = 16):
        super().__init__()
        if weight.dim() != 2:
            raise ValueError("a weight [N, K] is expected")
        self._quantize(weight, bias, block)

    @classmethod
    def of(cls, layer: torch.nn.Module, block: int = 16) -> "E2m1Linear":
        """From a module with ``weight`` [N, K] and, maybe, ``bias``."""
        return cls(layer.weight, getattr(layer, "bias", None), block)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        z = autograd.context(x.device).quant_e2m1_gemm(x, self.codes, self.tiles, self.scale, self.bias, self.block)
        return z if x.dim() == 2 else z.reshape(*x.shape[:-1], z.shape[-1])


class E2m1Experts(_E2m1Module):
    """One weight per expert, ``[E, N, K]``.  ``forward(x, offsets)``: rows ``offsets[e] .. offsets[e + 1] - 1`` of x
    belong to expert e.  ``forward(x, offsets, position)``: x holds each token once, its k copies' results are rows
    ``position[t]`` of the result (both from ``experts.order``).  Rows that belong to no expert are not written."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor | None = None, block: int = 16):
        super().__init__()
        if weight.dim() != 3:
            raise ValueError("weights [E, N, K] are expected")
        self._quantize(weight, bias, block)

    def forward(self, x: torch.Tensor, offsets: torch.Tensor, position: torch.Tensor | None = None) -> torch.Tensor:
        return autograd.context(x.device).quant_e2m1_gemm_grouped(x, offsets, self.codes, self.tiles, self.scale, self.bias, self.block,
                                                                  position)
