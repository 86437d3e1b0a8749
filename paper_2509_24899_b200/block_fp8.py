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

_BF16, _F32, _E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
_DTYPES = {_BF16: binding.AS_DTYPE_BF16, _F32: binding.AS_DTYPE_F32}
# as_rows_t is QiiqqqQ-like: address, dtype, head_dim, tokens, strides of batch, head, token; as_fp8_matrix_t: address, pitch, scales, scale_rows
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
    pitch = (cols + 15) & -16
    data = torch.empty((rows, pitch), dtype=_E4M3, device=device or "cuda")
    scales = torch.empty(((cols + 511) // 512, rows, 4), dtype=torch.uint8, device=device or "cuda")
    return BlockFp8(data if pitch == cols else data[:, :cols], scales)


def _refuse(where, what):
    raise ValueError("%s: %s" % (where, what))


def _rows(t, where, name):
    """((rows, cols), as_rows_t's fields) of a tensor."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None or not t.is_cuda:
        _refuse(where, "%s is a bf16 or fp32 CUDA tensor, not %s on %s" % (name, t.dtype, t.device))
    if t.dim() == 2:
        (rows, cols), (st, one) = t.shape, t.stride()
        # a single row or column leaves its stride open
        if one != 1 and cols > 1:
            _refuse(where, "%s's columns lie next to each other; strides are %s" % (name, t.stride()))
        return (rows, cols), (t.data_ptr(), dtype, cols, rows, 0, 0, st if rows > 1 else 0)
    if t.dim() != 4:
        _refuse(where, "%s is [rows, cols] or [B, H, N, d], not %s" % (name, tuple(t.shape)))
    (b, h, n, d), (sb, sh, st, one) = t.shape, t.stride()
    if one != 1 and d > 1:
        _refuse(where, "%s's columns of a head lie next to each other; strides are %s" % (name, t.stride()))
    return (b * n, h * d), (t.data_ptr(), dtype, d, n, sb if b > 1 else 0, sh if h > 1 else 0, st if n > 1 else 0)


def _matrix(m, where, name):
    """((rows, cols), as_fp8_matrix_t's fields) of a pair."""
    data, scales = m
    if data.dtype != _E4M3 or scales.dtype != torch.uint8 or not data.is_cuda or not scales.is_cuda or data.dim() != 2:
        _refuse(where, "%s is a pair of CUDA tensors, float8_e4m3fn [rows, cols] and uint8 scales" % name)
    rows, cols = data.shape
    st, one = data.stride()
    groups, srows, four = scales.shape if scales.dim() == 3 else (0, 0, 0)
    sg, sr, s1 = scales.stride() if scales.dim() == 3 else (0, 0, 0)
    if groups != (cols + 511) // 512 or srows != rows or four != 4:
        _refuse(where, "%s's scales for %s are [%d, %d, 4], not %s" % (name, tuple(data.shape), (cols + 511) // 512, rows, tuple(scales.shape)))
    if rows == 0:
        return (0, cols), (data.data_ptr() or 16, (cols + 15) & -16, scales.data_ptr() or 16, 0)
    if (one != 1 and cols > 1) or s1 != 1 or (sr != 4 and rows > 1) or (groups > 1 and (sg % 4 or sg < 4 * rows)):
        _refuse(where, "%s's strides are %s and %s: values and the four bytes of a row lie next to each other" % (name, data.stride(), scales.stride()))
    return (rows, cols), (data.data_ptr(), st if rows > 1 else (cols + 15) & -16, scales.data_ptr(), sg // 4 if groups > 1 else rows)


def _stream(stream):
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _same_device(where, *tensors):
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here:
            _refuse(where, "all tensors are on the current device, cuda:%d" % here)


def rms_norm(x, weight=None, residual=None, eps=1e-6, fp8=False, out=None, residual_out=None, stream=None):
    """y = t * rsqrt(mean(t^2) + eps) * weight over the columns of t = x + residual, in fp32, rounded once.

    x, residual   bf16 or fp32 (residual in fp32 if x is); weight: [cols], bf16 or fp32, or None
    fp8           y in 8-bit form (a BlockFp8, a scale for each row and 128 columns) instead of bf16
    out           where y goes: a tensor [rows, cols] or [B, H, N, d] (its layout need not be x's), with fp8 a BlockFp8
    residual_out  where t goes, in the residual's type; may be `residual` itself

    Returns y, or (y, t) with a residual.  Up to 16384 columns."""
    (rows, cols), xr = _rows(x, "rms_norm", "x")
    rr = tr = _NONE_ROWS
    if residual is not None:
        shape, rr = _rows(residual, "rms_norm", "residual")
        if residual_out is None:
            residual_out = torch.empty(residual.shape, dtype=residual.dtype, device=residual.device)
        to, tr = _rows(residual_out, "rms_norm", "residual_out")
        if shape != (rows, cols) or to != shape or residual_out.dtype != residual.dtype:
            _refuse("rms_norm", "residual and residual_out are %d x %d of one type" % (rows, cols))
    elif residual_out is not None:
        _refuse("rms_norm", "residual_out needs a residual")
    wp = wd = 0
    if weight is not None:
        wd = _DTYPES.get(weight.dtype, -1)
        if wd < 0 or weight.shape != (cols,) or (weight.stride(0) != 1 and cols > 1):
            _refuse("rms_norm", "weight is %d bf16 or fp32 values next to each other" % cols)
        wp = weight.data_ptr()
    yr, ym = _NONE_ROWS, _NONE_MATRIX
    if fp8:
        if out is None:
            out = empty_fp8(rows, cols)
        shape, ym = _matrix(out, "rms_norm", "out")
        _same_device("rms_norm", x, weight, residual, residual_out, *out)
    else:
        if out is None:
            out = torch.empty(x.shape, dtype=_BF16, device=x.device)
        shape, yr = _rows(out, "rms_norm", "out")
        _same_device("rms_norm", x, weight, residual, residual_out, out)
    if shape != (rows, cols):
        _refuse("rms_norm", "out stands for %d x %d" % (rows, cols))
    if rows and cols:
        binding.as_rms_norm(_NORM.pack(_NORM.size, cols, rows, *xr, *rr, *tr, *yr, *ym, wp, wd, eps), _stream(stream))
    return out if residual is None else (out, residual_out)


def quantize_fp8(x, block_rows=1, out=None, stream=None) -> BlockFp8:
    """x (bf16 or fp32, [rows, cols] or [B, H, N, d]) in 8-bit form; block_rows: rows that share a scale, 1 for activations and
    128 for weights."""
    (rows, cols), xr = _rows(x, "quantize_fp8", "x")
    if out is None:
        out = empty_fp8(rows, cols)
    shape, om = _matrix(out, "quantize_fp8", "out")
    if shape != (rows, cols):
        _refuse("quantize_fp8", "out is %d x %d" % (rows, cols))
    _same_device("quantize_fp8", x, *out)
    if rows and cols:
        binding.as_quantize_fp8(_QUANT.pack(_QUANT.size, cols, rows, *xr, *om, block_rows, 0), _stream(stream))
    return out


_contexts = {}
_lock = threading.Lock()


def _context():
    dev = torch._C._cuda_getDevice()
    ctx = _contexts.get(dev)
    if ctx is None:
        with _lock:
            ctx = _contexts.get(dev)
            if ctx is None:
                ctx = _contexts[dev] = binding.as_fp8_create()
    return ctx


def matmul_fp8(a, w, bias=None, out=None, stream=None):
    """a [M, K] times the transpose of w [N, K], both in 8-bit form, plus bias [N] (bf16): bf16 [M, N], or what `out` is
    ([M, N] with any row stride, [B, H, tokens, d] with B * tokens = M and H * d = N).

    The first call on a device sets the device's context up (it allocates 256 bytes and synchronises): make it outside of a
    stream capture."""
    (m, k), am = _matrix(a, "matmul_fp8", "a")
    (n, wk), wm = _matrix(w, "matmul_fp8", "w")
    if wk != k:
        _refuse("matmul_fp8", "a has %d columns, w %d" % (k, wk))
    bp = 0
    if bias is not None:
        if bias.dtype != _BF16 or bias.shape != (n,) or (bias.stride(0) != 1 and n > 1):
            _refuse("matmul_fp8", "bias is %d bf16 values next to each other" % n)
        bp = bias.data_ptr()
    if out is None:
        out = torch.empty((m, n), dtype=_BF16, device=a[0].device)
    shape, orow = _rows(out, "matmul_fp8", "out")
    if shape != (m, n) or out.dtype != _BF16:
        _refuse("matmul_fp8", "out stands for %d x %d in bf16" % (m, n))
    _same_device("matmul_fp8", a[0], a[1], w[0], w[1], bias, out)
    if m and n:
        if k == 0:
            _refuse("matmul_fp8", "there are no columns to sum over")
        binding.as_matmul_fp8(_context(), _MATMUL.pack(_MATMUL.size, k, m, n, *am, *wm, bp, *orow), _stream(stream))
    return out


def fp8_last_status(stream=None) -> int:
    """AS_OK, or AS_ERR_DEVICE_TIMEOUT if a wait inside a product on this device ran out since the last call; synchronises."""
    return binding.as_fp8_last_status(_context(), _stream(stream))
