"""Linear layers in bf16 with what follows them: PyTorch tensors in, the library's kernels behind them (include/as_layer.h).

    h = linear(x, w1, bias=b1, activation="gelu_tanh")                   # the feed-forward half's first layer
    t = linear(h, w2, bias=b2, gate=g, residual=t, out=t)                # its second one, gated onto the residual stream in place
    t = linear(o, wo, bias=bo, gate=g, residual=t)                       # the output projection, from the attention's [B, H, N, d] as it lies

A matrix is a tensor [rows, cols], or [B, H, N, d] as the attention has it, which stands for [B * N, H * d].  Any strides are taken whose innermost one is 1; operands whose strides and
addresses are no multiples of 16 bytes, or whose heads are no multiples of 64, are copied first.  Tensors that require gradients are refused unless gradients are off or they are
detached, and so are those with a forward-mode tangent: a program that trains keeps `pre` and calls `linear_backward`.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from .block_fp8 import _calls, _on
from .rotation import _choice

_ACTIVATIONS = {None: -1, "relu": 0, "silu": 1, "gelu": 2, "gelu_tanh": 3}


class LinearGradients(NamedTuple):
    """Gradients of a linear layer's inputs; None where there is no such input, or none was asked for.  (The residual's is that of the result.)"""
    x: torch.Tensor | None
    w: torch.Tensor | None
    bias: torch.Tensor | None
    gate: torch.Tensor | None


def linear(x, w, bias=None, activation=None, gate=None, residual=None, out=None, keep_pre=False, stream=None):
    """residual + gate * act(x w^T + bias), products of bf16 values summed in fp32, one rounding at the end.

    x           [M, K] or [B, H, N, d], bf16; w: [N, K], bf16
    bias        [N]; gate: [N], or [entries, N] where each entry's rows (M / entries in turn) have their own (up to 65534 of them); bf16 or fp32
    activation  None, "relu", "silu", "gelu" (by the error function) or "gelu_tanh"
    residual    [M, N] or heads, bf16 or fp32
    out         where the result goes, bf16 or fp32, rows or heads; may be `residual` itself, and overlaps nothing else.  None: a new tensor in the residual's shape and type, else bf16 [M, N]
    keep_pre    True, or a bf16 tensor to put it in: x w^T + bias as well, rounded to bf16, for `linear_backward`

    Returns the result, or (result, pre).  The first call on a device sets the device's context up (it allocates 256 bytes and synchronises): make it outside of a stream capture.  A
    wait inside that ran out is reported by `fp8_last_status`."""
    return _on(stream, _calls.linear, x, w, bias, _choice(_ACTIVATIONS, activation, "linear", "activation"), gate, residual, out, keep_pre)


def linear_backward(dy, x, w, pre=None, activation=None, gate=None, bias=None, x_grad=True, w_grad=True, gate_grad=True, stream=None) -> LinearGradients:
    """From the gradient dy [M, N] (bf16 or fp32, rows or heads) of `linear`'s result and its arguments: the gradients of its inputs, in their types; dx in x's shape.

    The gradient of x w^T + bias, dy * gate * act'(pre), is rounded to bf16 as an operand of the products behind dx and dw, in fp32 dy's as well; the gradients of bias and gate come from its unrounded values.

    pre   what `linear` kept; needed with an activation, and for the gate's gradient
    bias  the bias, or any vector of its size and type: its gradient is wanted.  x_grad, w_grad, gate_grad: whether those are"""
    return LinearGradients(*_on(stream, _calls.linear_backward, dy, x, w, pre, _choice(_ACTIVATIONS, activation, "linear_backward", "activation"), gate, bias, x_grad, w_grad, gate_grad))
