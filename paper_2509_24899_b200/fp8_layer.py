"""The attention half of a converted layer, its linear layers in 8 bits: what `HybridAttention` and the 8-bit projections do together.

    t = hidden + residual;  x = norm(t)                                  rms_norm: x in 8-bit form, t is the next residual
    q, k = norm_q(x Wq + bq), norm_k(x Wk + bk);  v = x Wv + bv          matmul_fp8; the norms and v land in heads
    o = hybrid attention of q, k, v                                      HybridAttention.forward
    y = o Wo + bo                                                        quantize_fp8 from heads, matmul_fp8

No tensor is copied or permuted between the calls.  Weights are frozen: they are brought to their 8-bit form once.

Nothing stands between the norms of q and k and the attention: a model that turns them there (a rotary embedding) makes the same calls itself, with its own step in between.  q, k and
v come from three products, each of which lands where it is needed; one product with the three weights on top of each other gives rows [B N, 3 H d], of which the norms take their
thirds as they lie, but v would be copied into heads (the attention takes contiguous ones).
"""
from __future__ import annotations

import torch

from . import HybridAttention
from .block_fp8 import matmul_fp8, quantize_fp8, rms_norm


class Fp8AttentionLayer:
    """`attention`: the layer's HybridAttention, of B x H x N x d.  `weights`: name -> bf16 CUDA tensor: "q", "k", "v", "o" [H d, H d] and
    optionally "bias_q", ..., "bias_o" [H d], "norm", "norm_q", "norm_k" [H d], all on the current device; `phi`: the feature maps' weights, the
    keyword arguments that `HybridAttention.forward` takes (wq, wk, ...)."""

    def __init__(self, attention: HybridAttention, weights, phi, eps=1e-6):
        self.attention, self.phi, self.eps = attention, phi, eps
        B, H, N, d = attention.shape
        for name in "qkvo":
            if tuple(weights[name].shape) != (H * d, H * d):
                raise ValueError("Fp8AttentionLayer: weight %r is %d x %d, not %s" % (name, H * d, H * d, tuple(weights[name].shape)))

        def frozen(name):
            return None if weights.get(name) is None else weights[name].detach()

        self._w8 = {name: quantize_fp8(frozen(name), block_rows=128) for name in "qkvo"}
        self._bias = {name: frozen("bias_" + name) for name in "qkvo"}
        self._norm = {name: frozen(name) for name in ("norm", "norm_q", "norm_k")}

    def forward(self, hidden, residual):
        """hidden [B N, H d] bf16, residual [B N, H d] bf16 or fp32 -> (y [B N, H d] bf16, the next residual)."""
        x8, residual = rms_norm(hidden, self._norm["norm"], residual=residual, eps=self.eps, fp8=True)
        shape = self.attention.shape
        q, k, v = (torch.empty(shape, dtype=torch.bfloat16, device=hidden.device) for _ in range(3))
        for name, out in (("q", q), ("k", k)):
            rows = matmul_fp8(x8, self._w8[name], bias=self._bias[name])
            rms_norm(rows, self._norm["norm_" + name], eps=self.eps, out=out)
        matmul_fp8(x8, self._w8["v"], bias=self._bias["v"], out=v)
        o = self.attention.forward(q, k, v, **self.phi)
        return matmul_fp8(quantize_fp8(o), self._w8["o"], bias=self._bias["o"]), residual
