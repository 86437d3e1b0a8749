"""The 8-bit projections around the attention: PyTorch tensors in, the library's kernels behind them (include/as_fp8.h).

    y8, residual = rms_norm(x, weight, residual=residual, fp8=True)      # norm of x + residual, in 8-bit form
    q = matmul_fp8(y8, wq8, bias=bq, out=q)                              # [B, H, N, d] or [rows, cols], by what `out` is
    w8 = quantize_fp8(weight, block_rows=128)                            # weights, once

A matrix is a tensor [rows, cols], or [B, H, N, d] as the attention has it, which stands for [B * N, H * d].  Any strides are taken
whose innermost one is 1; where those of a call's tensors, and their addresses, are multiples of 16 bytes, rows move faster.

The calls have no gradients: a tensor that requires one is refused unless gradients are off (torch.no_grad()) or it is detached, one with a forward-mode tangent always.  Tensors that are given for outputs count as
modified in place.
"""
from __future__ import annotations

import importlib.machinery
import importlib.util
import os
from typing import NamedTuple

import torch

from . import binding

_F32, _E4M3 = torch.float32, torch.float8_e4m3fn


class BlockFp8(NamedTuple):
    """A matrix in 8-bit form.  Any pair of tensors laid out like this will do in its place.

    data    float8_e4m3fn [rows, cols], rows a multiple of 16 bytes apart
    scales  uint8 [ceil(cols / 512), rows, 4]: the byte of row r and block k = c // 128 is scales[k // 4, r, k % 4], for 2^(byte - 127)
    """
    data: torch.Tensor
    scales: torch.Tensor

    def dequantize(self) -> torch.Tensor:
        """The matrix in fp32 (plain PyTorch; for looking at values)."""
        rows, cols = self.data.shape
        e = self.scales.permute(1, 0, 2).reshape(rows, -1)[:, :(cols + 127) // 128].to(torch.int32)
        factor = torch.where(e == 255, float("nan"), torch.where(e == 0, 2.0 ** -127, (e << 23).view(_F32)))
        return self.data.to(_F32) * factor.repeat_interleave(128, 1)[:, :cols]


def empty_fp8(rows: int, cols: int, device=None) -> BlockFp8:
    """Room for a matrix in 8-bit form."""
    device = device or "cuda"
    return BlockFp8(torch.empty_strided((rows, cols), ((cols + 15) & -16, 1), dtype=_E4M3, device=device),
                    torch.empty_strided(((cols + 511) // 512, rows, 4), (4 * rows, 4, 1), dtype=torch.uint8, device=device))


def _load():
    """The module of these calls (csrc/torch_calls.cpp).  Raises if it has not been built - there is no fallback."""
    path = os.path.join(os.path.dirname(binding.LIB_PATH), "as_torch_calls.so")
    if not os.path.exists(path):
        raise ImportError("as_torch_calls.so is missing at %s; run `python -m paper_2509_24899_b200.build`" % path)
    loader = importlib.machinery.ExtensionFileLoader("as_torch_calls", path)
    module = importlib.util.module_from_spec(importlib.util.spec_from_file_location("as_torch_calls", path, loader=loader))
    loader.exec_module(module)
    module.set_classes(BlockFp8, binding.AsError)
    return module


_calls = _load()


def _on(stream, call, *args):
    """The call on `stream`: it and what it allocates belong there."""
    if stream is None:
        return call(*args)
    with torch.cuda.stream(stream):
        return call(*args)


def rms_norm(x, weight=None, residual=None, eps=1e-6, fp8=False, out=None, residual_out=None, stream=None):
    """y = t * rsqrt(mean(t^2) + eps) * weight over the columns of t = x + residual, in fp32, rounded once.

    x, residual   bf16 or fp32 (residual in fp32 if x is); weight: [cols], bf16 or fp32, or None
    fp8           y in 8-bit form (a BlockFp8, a scale for each row and 128 columns) instead of bf16
    out           where y goes: a tensor [rows, cols] or [B, H, N, d] (its layout need not be x's), with fp8 a BlockFp8
    residual_out  where t goes, in the residual's type; may be `residual` itself

    Returns y, or (y, t) with a residual.  Up to 16384 columns."""
    return _on(stream, _calls.rms_norm, x, weight, residual, eps, fp8, out, residual_out)


def quantize_fp8(x, block_rows=1, out=None, stream=None) -> BlockFp8:
    """x (bf16 or fp32, [rows, cols] or [B, H, N, d]) in 8-bit form; block_rows: rows that share a scale, 1 for activations and
    128 for weights (up to 65535 * 128 rows).  Up to 16384 columns."""
    return _on(stream, _calls.quantize_fp8, x, block_rows, out)


def matmul_fp8(a, w, bias=None, out=None, stream=None):
    """a [M, K] times the transpose of w [N, K], both in 8-bit form, plus bias [N] (bf16): bf16 [M, N], or what `out` is
    ([M, N] with any row stride, [B, H, tokens, d] with B * tokens = M and H * d = N).

    The first call on a device sets the device's context up (it allocates 256 bytes and synchronises): make it outside of a
    stream capture."""
    return _on(stream, _calls.matmul_fp8, a, w, bias, out)


def fp8_last_status(stream=None) -> int:
    """AS_OK, or AS_ERR_DEVICE_TIMEOUT if a wait inside a product on this device ran out since the last call; synchronises."""
    return _on(stream, _calls.last_status)
