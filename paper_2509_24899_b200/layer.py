"""A converted layer in bf16: the steps around the attention together with `HybridAttention`, and the two parts of it that a program may train, with their gradients.

    x = norm(t);  q, k = R norm_q(x Wq + bq), R norm_k(x Wk + bk);  v = x Wv + bv     rms_norm; linear (q and k in one product, v into heads); qk_norm_rotary
    t = t + g_o (hybrid attention(q, k, v) Wo + bo)                                    HybridAttention.forward; linear, from the attention's layout
    x = norm(t);  t = t + g_f (act(x W1 + b1) W2 + b2)                                 rms_norm; linear, linear

No tensor is copied or permuted between the calls.  `QkProjection` and `FeedForward` have backward passes; what stands between them in a layer, the attention, has its own gradients for the
feature maps alone, so a layer as a whole has none.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import HybridAttention
from .block_fp8 import rms_norm
from .projection import linear, linear_backward
from .rotation import _where, qk_norm_rotary, qk_norm_rotary_backward


def _frozen(weights, name):
    return None if weights.get(name) is None else weights[name].detach()


class QkProjection:
    """Queries and keys from a layer's input: one product for both, norms (over a token's heads, `norm="row"`, or for each head) and rotation.

    shape    (B, H, N, d);  w: [2 H d, K] bf16, queries' rows first, bias: [2 H d] or None
    norm_q, norm_k: [H d] ([d] with norm="head"), or None;  table, layout, first, positions: as for `qk_norm_rotary`; table=None: no rotation.  A range of a clip's tokens has the clip's table and its
    own `first`
    """

    class Gradients(NamedTuple):
        x: torch.Tensor
        w: torch.Tensor
        bias: torch.Tensor | None
        norm_q: torch.Tensor | None
        norm_k: torch.Tensor | None

    def __init__(self, shape, w, bias=None, norm_q=None, norm_k=None, table=None, norm="row", eps=1e-6, layout="interleaved", first=0, positions=None):
        B, H, N, d = shape
        if w.shape[0] != 2 * H * d:
            raise ValueError("QkProjection: w has %d rows, not %d" % (w.shape[0], 2 * H * d))
        self.shape, self.w, self.bias, self.norms = tuple(shape), w, bias, (norm_q, norm_k)
        self._how = dict(table=table, norm=norm, eps=eps, layout=layout, first=first, positions=positions)

    def _heads(self, rows):
        """The queries' and the keys' part of rows [B N, 2 H d], each as [B, H, N, d]."""
        B, H, N, d = self.shape
        parts = rows.view(B, N, 2, H, d).permute(2, 0, 3, 1, 4)
        return parts[0], parts[1]

    def forward(self, x, keep=False):
        """x [B N, K] -> (q, k), or ((q, k), what `backward` takes) with `keep`."""
        rows = linear(x, self.w, bias=self.bias)
        qk = qk_norm_rotary(*self._heads(rows), *self.norms, **self._how)
        return (qk, (x, rows)) if keep else qk

    def backward(self, dq, dk, kept) -> "QkProjection.Gradients":
        x, rows = kept
        drows = torch.empty_like(rows)
        dq_out, dk_out = self._heads(drows)
        g = qk_norm_rotary_backward(dq, dk, *self._heads(rows), *self.norms, dq_out=dq_out, dk_out=dk_out, **self._how)
        f = linear_backward(drows, x, self.w, bias=self.bias)
        return self.Gradients(f.x, f.w, f.bias, g.q_weight, g.k_weight)


class FeedForward:
    """act(x w1^T + b1) w2^T + b2, gated onto a residual."""

    class Gradients(NamedTuple):
        x: torch.Tensor
        w1: torch.Tensor
        b1: torch.Tensor | None
        w2: torch.Tensor
        b2: torch.Tensor | None
        gate: torch.Tensor | None

    def __init__(self, w1, w2, b1=None, b2=None, activation="gelu_tanh"):
        if w1.shape[0] != w2.shape[1]:
            raise ValueError("FeedForward: w2 takes %d columns, w1 gives %d" % (w2.shape[1], w1.shape[0]))
        self.w1, self.w2, self.b1, self.b2, self.activation = w1, w2, b1, b2, activation

    def forward(self, x, gate=None, residual=None, out=None, keep=False):
        """x [rows, K] -> the result, in the residual's type, or (result, what `backward` takes) with `keep`."""
        if not keep:
            h = linear(x, self.w1, bias=self.b1, activation=self.activation)
            return linear(h, self.w2, bias=self.b2, gate=gate, residual=residual, out=out)
        h, pre1 = linear(x, self.w1, bias=self.b1, activation=self.activation, keep_pre=True)
        got = linear(h, self.w2, bias=self.b2, gate=gate, residual=residual, out=out, keep_pre=gate is not None)
        y, pre2 = got if gate is not None else (got, None)
        return y, (x, pre1, h, pre2, gate)

    def backward(self, dy, kept) -> "FeedForward.Gradients":
        """From the result's gradient, which is the residual's as well."""
        x, pre1, h, pre2, gate = kept
        second = linear_backward(dy, h, self.w2, pre=pre2, gate=gate, bias=self.b2)
        first = linear_backward(second.x, x, self.w1, pre=pre1, activation=self.activation, bias=self.b1)
        return self.Gradients(first.x, first.w, first.bias, second.w, second.bias, second.gate)


class AttentionLayer:
    """`attention`: the layer's HybridAttention, of B x H x N x d.  `weights`: name -> bf16 CUDA tensor: "q", "k", "v", "o" [H d, H d], "up" [F, H d], "down" [H d, F] and optionally "bias_q", ...,
    "bias_down", "norm", "norm_ff" [H d], "norm_q", "norm_k" [H d] ([d] with norm="head"); `phi`: the keyword arguments that `HybridAttention.forward` takes (wq, wk, ...); `table`: a
    RotaryTable of the layer's grid, or None; `first`, `positions`: as for `qk_norm_rotary`, with None the attention's tokens begin at its `n0` (a SeqShardedAttention's range of them), or at 0.
    Weights are taken when the layer is made (queries' and keys' are put together, the others stay where they are): one that they change for is made again."""

    def __init__(self, attention: HybridAttention, weights, phi, table=None, norm="row", eps=1e-6, activation="gelu_tanh", layout="interleaved", first=None, positions=None):
        self.attention, self.phi, self.eps = attention, phi, eps
        B, H, N, d = attention.shape
        w = {name: _frozen(weights, name) for name in ("q", "k", "v", "o", "up", "down", "norm", "norm_ff", "norm_q", "norm_k")}
        b = {name: _frozen(weights, "bias_" + name) for name in ("q", "k", "v", "o", "up", "down")}
        if (b["q"] is None) != (b["k"] is None):
            raise ValueError("AttentionLayer: a bias of queries goes with one of keys")
        qk_bias = None if b["q"] is None else torch.cat((b["q"], b["k"]))
        self.qk = QkProjection(attention.shape, torch.cat((w["q"], w["k"])), qk_bias, w["norm_q"], w["norm_k"], table, norm, eps, layout, **_where(attention, first, positions))
        self.feed_forward = FeedForward(w["up"], w["down"], b["up"], b["down"], activation)
        self._w, self._b = w, b

    def forward(self, stream, gate_o=None, gate_f=None):
        """stream [B N, H d] bf16 or fp32, gates [H d] or [B, H d] -> the stream behind the layer, a new tensor of its type."""
        x = rms_norm(stream, self._w["norm"], eps=self.eps)
        q, k = self.qk.forward(x)
        v = linear(x, self._w["v"], bias=self._b["v"], out=torch.empty_like(q))
        o = self.attention.forward(q, k, v, **self.phi)
        t = linear(o, self._w["o"], bias=self._b["o"], gate=gate_o, residual=stream)
        x = rms_norm(t, self._w["norm_ff"], eps=self.eps)
        return self.feed_forward.forward(x, gate=gate_f, residual=t, out=t)
