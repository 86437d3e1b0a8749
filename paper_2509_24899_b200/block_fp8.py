"""The 8-bit projections around the attention: PyTorch tensors in, the library's kernels behind them (include/as_fp8.h).

    y8, residual = rms_norm(x, weight, residual=residual, fp8=True)      # norm of x + residual, in 8-bit form
    q = matmul_fp8(y8, wq8, bias=bq, out=q)                              # [B, H, N, d] or [rows, cols], by what `out` is
    w8 = quantize_fp8(weight, block_rows=128)                            # weights, once

A matrix is a tensor [rows, cols], or [B, H, N, d] as the attention has it, which stands for [B * N, H * d].  Any strides are taken
whose innermost one is 1; where those of a call's tensors, and their addresses, are multiples of 16 bytes, rows move faster.
"""
from __future__ import annotations

import struct
import threading
from typing import NamedTuple

import torch

from . import binding

_BF16, _F32, _E4M3, _U8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.uint8
_FLOATS, _BF16_ONLY = (_BF16, _F32), (_BF16,)
_current_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
_DTYPES = {_BF16: binding.AS_DTYPE_BF16, _F32: binding.AS_DTYPE_F32}
# as_rows_t: address, dtype, head_dim, tokens, strides of batch, head, token; as_fp8_matrix_t: address, pitch, scales, scale_rows
_ROWS, _MATRIX = "Qiiqqqq", "QqQq"
_NORM = struct.Struct("=Iiq" + 4 * _ROWS + _MATRIX + "Qif")
_QUANT = struct.Struct("=Iiq" + _ROWS + _MATRIX + "ii")
_MATMUL = struct.Struct("=Iiqq" + 2 * _MATRIX + "Q" + _ROWS)
_NONE_ROWS, _NONE_MATRIX = (0,) * 7, (0,) * 4


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


def _refuse(where, what):
    raise ValueError("%s: %s" % (where, what))


def _rows(t, here, where, name):
    """(rows, cols, as_rows_t's fields) of a tensor on device `here`."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None or t.get_device() != here:
        _refuse(where, "%s is a bf16 or fp32 tensor on the current device, cuda:%d, not %s on %s" % (name, here, t.dtype, t.device))
    shape, strides = t.shape, t.stride()
    if len(shape) == 2:
        rows, cols = shape
        if strides[1] != 1 and cols > 1:      # a single row or column leaves its stride open
            _refuse(where, "%s's columns lie next to each other; strides are %s" % (name, strides))
        return rows, cols, (t.data_ptr(), dtype, cols, rows, 0, 0, strides[0] if rows > 1 else 0)
    if len(shape) != 4:
        _refuse(where, "%s is [rows, cols] or [B, H, N, d], not %s" % (name, tuple(shape)))
    (b, h, n, d), (sb, sh, st, one) = shape, strides
    if one != 1 and d > 1:
        _refuse(where, "%s's columns of a head lie next to each other; strides are %s" % (name, strides))
    return b * n, h * d, (t.data_ptr(), dtype, d, n, sb if b > 1 else 0, sh if h > 1 else 0, st if n > 1 else 0)


def _matrix(m, here, where, name):
    """(rows, cols, as_fp8_matrix_t's fields) of a pair on device `here`."""
    data, scales = m
    if data.dtype != _E4M3 or scales.dtype != _U8 or data.get_device() != here or scales.get_device() != here:
        _refuse(where, "%s is a pair of tensors on the current device, cuda:%d: float8_e4m3fn [rows, cols] and uint8 scales" % (name, here))
    shape = data.shape
    if len(shape) != 2:
        _refuse(where, "%s's values are [rows, cols], not %s" % (name, tuple(shape)))
    rows, cols = shape
    groups = (cols + 511) // 512
    if tuple(scales.shape) != (groups, rows, 4):
        _refuse(where, "%s's scales for %s are %s, not %s" % (name, tuple(shape), (groups, rows, 4), tuple(scales.shape)))
    if rows == 0:
        return 0, cols, (16, (cols + 15) & -16, 16, 0)
    (st, one), (sg, sr, s1) = data.stride(), scales.stride()
    if (one != 1 and cols > 1) or s1 != 1 or (sr != 4 and rows > 1) or (groups > 1 and (sg % 4 or sg < 4 * rows)):
        _refuse(where, "%s's strides are %s and %s: values and the four bytes of a row lie next to each other" % (name, data.stride(), scales.stride()))
    return rows, cols, (data.data_ptr(), st if rows > 1 else (cols + 15) & -16, scales.data_ptr(), sg // 4 if groups > 1 else rows)


def _vector(t, n, dtypes, here, where, name):
    """Address of n values next to each other."""
    if t.dtype not in dtypes or t.get_device() != here or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        _refuse(where, "%s is %d values of %s next to each other on cuda:%d" % (name, n, " or ".join(str(d) for d in dtypes), here))
    return t.data_ptr()


def _stream(stream, here):
    return stream.cuda_stream if stream is not None else _raw_stream(here)


def rms_norm(x, weight=None, residual=None, eps=1e-6, fp8=False, out=None, residual_out=None, stream=None):
    """y = t * rsqrt(mean(t^2) + eps) * weight over the columns of t = x + residual, in fp32, rounded once.

    x, residual   bf16 or fp32 (residual in fp32 if x is); weight: [cols], bf16 or fp32, or None
    fp8           y in 8-bit form (a BlockFp8, a scale for each row and 128 columns) instead of bf16
    out           where y goes: a tensor [rows, cols] or [B, H, N, d] (its layout need not be x's), with fp8 a BlockFp8
    residual_out  where t goes, in the residual's type; may be `residual` itself

    Returns y, or (y, t) with a residual.  Up to 16384 columns."""
    here = _current_device()
    rows, cols, xr = _rows(x, here, "rms_norm", "x")
    rr = tr = yr = _NONE_ROWS
    ym = _NONE_MATRIX
    if residual is not None:
        r, c, rr = _rows(residual, here, "rms_norm", "residual")
        if residual_out is None:
            residual_out = torch.empty_like(residual)
        r1, c1, tr = _rows(residual_out, here, "rms_norm", "residual_out")
        if r != rows or c != cols or r1 != rows or c1 != cols or residual_out.dtype != residual.dtype:
            _refuse("rms_norm", "residual and residual_out are %d x %d of one type" % (rows, cols))
    elif residual_out is not None:
        _refuse("rms_norm", "residual_out needs a residual")
    wp = wd = 0
    if weight is not None:
        wp, wd = _vector(weight, cols, _FLOATS, here, "rms_norm", "weight"), _DTYPES[weight.dtype]
    if fp8:
        if out is None:
            out = empty_fp8(rows, cols, x.device)
        r, c, ym = _matrix(out, here, "rms_norm", "out")
    else:
        if out is None:
            out = torch.empty(x.shape, dtype=_BF16, device=x.device)
        r, c, yr = _rows(out, here, "rms_norm", "out")
    if r != rows or c != cols:
        _refuse("rms_norm", "out stands for %d x %d" % (rows, cols))
    if rows and cols:
        binding.as_rms_norm(_NORM.pack(_NORM.size, cols, rows, *xr, *rr, *tr, *yr, *ym, wp, wd, eps), _stream(stream, here))
    return out if residual is None else (out, residual_out)


def quantize_fp8(x, block_rows=1, out=None, stream=None) -> BlockFp8:
    """x (bf16 or fp32, [rows, cols] or [B, H, N, d]) in 8-bit form; block_rows: rows that share a scale, 1 for activations and
    128 for weights.  Up to 16384 columns."""
    here = _current_device()
    rows, cols, xr = _rows(x, here, "quantize_fp8", "x")
    if out is None:
        out = empty_fp8(rows, cols, x.device)
    r, c, om = _matrix(out, here, "quantize_fp8", "out")
    if r != rows or c != cols:
        _refuse("quantize_fp8", "out is %d x %d" % (rows, cols))
    if rows and cols:
        binding.as_quantize_fp8(_QUANT.pack(_QUANT.size, cols, rows, *xr, *om, block_rows, 0), _stream(stream, here))
    return out


_contexts = {}
_lock = threading.Lock()


def _context(here):
    ctx = _contexts.get(here)
    if ctx is None:
        with _lock:
            ctx = _contexts.get(here)
            if ctx is None:
                ctx = _contexts[here] = binding.as_fp8_create()
    return ctx


def matmul_fp8(a, w, bias=None, out=None, stream=None):
    """a [M, K] times the transpose of w [N, K], both in 8-bit form, plus bias [N] (bf16): bf16 [M, N], or what `out` is
    ([M, N] with any row stride, [B, H, tokens, d] with B * tokens = M and H * d = N).

    The first call on a device sets the device's context up (it allocates 256 bytes and synchronises): make it outside of a
    stream capture."""
    here = _current_device()
    m, k, am = _matrix(a, here, "matmul_fp8", "a")
    n, wk, wm = _matrix(w, here, "matmul_fp8", "w")
    if wk != k:
        _refuse("matmul_fp8", "a has %d columns, w %d" % (k, wk))
    bp = 0 if bias is None else _vector(bias, n, _BF16_ONLY, here, "matmul_fp8", "bias")
    if out is None:
        out = torch.empty_strided((m, n), (n, 1), dtype=_BF16, device=a[0].device)
    r, c, orow = _rows(out, here, "matmul_fp8", "out")
    if r != m or c != n or out.dtype != _BF16:
        _refuse("matmul_fp8", "out stands for %d x %d in bf16" % (m, n))
    if m and n:
        if k == 0:
            _refuse("matmul_fp8", "there are no columns to sum over")
        binding.as_matmul_fp8(_context(here), _MATMUL.pack(_MATMUL.size, k, m, n, *am, *wm, bp, *orow), _stream(stream, here))
    return out


def fp8_last_status(stream=None) -> int:
    """AS_OK, or AS_ERR_DEVICE_TIMEOUT if a wait inside a product on this device ran out since the last call; synchronises."""
    here = _current_device()
    return binding.as_fp8_last_status(_context(here), _stream(stream, here))
