"""The attention half of a converted layer, its linear layers in 8 bits: what `HybridAttention` and the 8-bit projections do together.

    t = hidden + residual;  x = norm(t)                                  rms_norm: x in 8-bit form, t is the next residual
    q, k = norm_q(x Wq + bq), norm_k(x Wk + bk);  v = x Wv + bv          matmul_fp8; the norms and v land in heads; with a table, turned by the tokens' positions in the same pass (qk_norm_rotary)
    o = hybrid attention of q, k, v                                      HybridAttention.forward
    y = o Wo + bo                                                        quantize_fp8 from heads, matmul_fp8

No tensor is copied or permuted between the calls.  Weights are frozen: they are brought to their 8-bit form once.

q, k and v come from three products, each of which lands where it is needed; one product with the three weights on top of each other gives rows [B N, 3 H d], of which the norms take their
thirds as they lie, but v would be copied into heads (the attention takes contiguous ones).
"""
from __future__ import annotations

import torch

from . import HybridAttention
from .block_fp8 import matmul_fp8, quantize_fp8, rms_norm
from .rotation import _where, qk_norm_rotary


class Fp8AttentionLayer:
    """`attention`: the layer's HybridAttention, of B x H x N x d.  `weights`: name -> bf16 CUDA tensor: "q", "k", "v", "o" [H d, H d] and
    optionally "bias_q", ..., "bias_o" [H d], "norm", "norm_q", "norm_k" [H d], all on the current device; `phi`: the feature maps' weights, the
    keyword arguments that `HybridAttention.forward` takes (wq, wk, ...); `table`: a RotaryTable of the layer's grid, by which q and k are turned, in `layout`;
    `first`, `positions`: as for `qk_norm_rotary`, with None the attention's tokens begin at its `n0` (a SeqShardedAttention's range of them), or at 0."""

    def __init__(self, attention: HybridAttention, weights, phi, eps=1e-6, table=None, layout="interleaved", first=None, positions=None):
        self.attention, self.phi, self.eps, self.table, self.layout = attention, phi, eps, table, layout
        self._where = _where(attention, first, positions)
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
        if self.table is None:                               # one after the other: the rows of one product are held at a time
            for name, out in (("q", q), ("k", k)):
                rms_norm(matmul_fp8(x8, self._w8[name], bias=self._bias[name]), self._norm["norm_" + name], eps=self.eps, out=out)
        else:
            B, H, N, d = shape
            qk_norm_rotary(*[matmul_fp8(x8, self._w8[name], bias=self._bias[name]).view(B, N, H, d).permute(0, 2, 1, 3) for name in "qk"], self._norm["norm_q"], self._norm["norm_k"], self.table,
                           norm="row", eps=self.eps, layout=self.layout, q_out=q, k_out=k, **self._where)
        matmul_fp8(x8, self._w8["v"], bias=self._bias["v"], out=v)
        o = self.attention.forward(q, k, v, **self.phi)
        return matmul_fp8(quantize_fp8(o), self._w8["o"], bias=self._bias["o"]), residual
