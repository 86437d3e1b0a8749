"""Rotation of heads by their tokens' positions, and the norms of queries and keys with it: PyTorch tensors in, the library's kernels behind them (include/as_layer.h).

    table = rotary_table((21, 30, 52), (22, 21, 21))                     # a latent grid's three axes, once per clip size
    q, k = qk_norm_rotary(q, k, wq, wk, table, norm="row")               # [B, H, N, d], any strides: as the projection left them
    y = rotary(x, table, layout="half", positions=positions)             # single tokens at positions of their own

Tensors are [B, H, N, d] in bf16 or fp32 with any strides whose innermost one is 1; where sizes, strides and addresses are multiples of 16 bytes (and the pairs of 8), rows move
faster.  Outputs are new tensors in [B, H, N, d] order unless they are given; one may be its input itself, and overlaps no other tensor.  Tensors that require gradients are refused unless gradients are off or they are
detached, and so are those with a forward-mode tangent: a program that trains calls the `_backward` functions.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from .block_fp8 import _calls, _on

_SCALINGS = {None: 0, "linear": 1, "ntk": 2, "yarn": 3}
_NORMS = {None: 0, "head": 1, "row": 2}
_LAYOUTS = {"interleaved": False, "half": True}


class RotaryTable(NamedTuple):
    """cos and sin of the positions of up to four axes.  Any triple laid out like this will do in its place.

    factors  fp32 [sum(sizes), sum(pairs), 2]: an axis's positions are the rows behind those of the axes before it, in which its own pairs are filled and the others 0
    sizes    positions of each axis
    pairs    pairs of a head that each axis turns, in turn
    """
    factors: torch.Tensor
    sizes: tuple
    pairs: tuple


class QkGradients(NamedTuple):
    """Gradients of queries, keys and their weights; None where there is no such input."""
    q: torch.Tensor
    k: torch.Tensor | None
    q_weight: torch.Tensor | None
    k_weight: torch.Tensor | None


def _where(attention, first, positions):
    """`first` and `positions` of a layer's tokens for the calls: where `first` is None, the tokens begin where the attention's do."""
    if first is None:
        first = 0 if positions is not None else getattr(attention, "n0", 0)
    return dict(first=first, positions=positions)


def _choice(table, key, where, name):
    try:
        return table[key]
    except (KeyError, TypeError):
        raise ValueError("%s: %s is none of %s" % (where, name, ", ".join(repr(k) for k in table))) from None


def rotary_table(sizes, pairs, base=10000.0, scaling=None, factor=1.0, original=0.0, stream=None) -> RotaryTable:
    """The table of axes with `sizes` positions, of which each turns its number of `pairs`: pair i of n by position * base^(-i / n).

    scaling   for positions beyond those that a model was trained on: None, "linear" (positions over `factor`), "ntk" (the base times factor^(n / (n - 1))) or "yarn" (pairs of few turns over
              `original` positions over `factor`, those of 32 and more left alone, a ramp over turns between them; cos and sin times 0.1 ln(factor) + 1).  A model whose ramp goes over the pairs' indices, or whose angles are others, makes
              a table of its own
    base, scaling, factor, original: one for all axes, or a tuple with one for each."""
    sizes, pairs = tuple(sizes), tuple(pairs)

    def each(v):
        return v if isinstance(v, tuple) else (v,) * len(sizes)

    codes = tuple(_choice(_SCALINGS, s, "rotary_table", "scaling") for s in each(scaling))
    return RotaryTable(_on(stream, _calls.rotary_table, sizes, pairs, each(base), codes, each(factor), each(original)), sizes, pairs)


def rotary(x, table, layout="interleaved", positions=None, first=0, inverse=False, out=None, stream=None):
    """x [B, H, N, d] with the first 2 P elements of each head turned pair by pair, (a, b) -> (a cos - b sin, a sin + b cos); the rest is copied.

    table      a RotaryTable of P pairs
    layout     "interleaved": pair i is elements 2 i and 2 i + 1; "half": i and i + P
    positions  int32 or int64, [N] or [B, N] (with several axes [N, axes] or [B, N, axes]); a token outside of an axis has NaN where it would be turned.  None: token t is at `first` + t in
               the axes' raster order, the last axis fastest, which has to lie in the grid
    inverse    the transposed rotation: what the gradient of the result goes through to become that of x"""
    return _on(stream, _calls.qk_norm_rotary, x, None, None, None, table, 0, 0.0, _choice(_LAYOUTS, layout, "rotary", "layout"), inverse, positions, first, out, None)


def qk_norm_rotary(q, k, q_weight=None, k_weight=None, table=None, norm="head", eps=1e-6, layout="interleaved", positions=None, first=0, q_out=None, k_out=None, stream=None):
    """(q, k), each R(x * rsqrt(mean(x^2) + eps) * weight), in fp32, rounded once.

    q, k    [B, H, N, d] and [B, H', N, d]; k may be None, and is then left out of what is returned
    norm    "head": the mean over a head's d elements, weights [d]; "row": over all heads of a token, weights [H d] (up to 16384 columns); None: no norm
    weights bf16 or fp32, of one type, or None
    table, layout, positions, first: as for `rotary`; table=None: norms alone"""
    return _on(stream, _calls.qk_norm_rotary, q, k, q_weight, k_weight, table, _choice(_NORMS, norm, "qk_norm_rotary", "norm"), eps, _choice(_LAYOUTS, layout, "qk_norm_rotary", "layout"), False,
               positions, first, q_out, k_out)


def qk_norm_rotary_backward(dq, dk, q, k, q_weight=None, k_weight=None, table=None, norm="head", eps=1e-6, layout="interleaved", positions=None, first=0, dq_out=None, dk_out=None,
                            stream=None) -> QkGradients:
    """From the gradients dq, dk of `qk_norm_rotary`'s results (the types and shapes of q and k) and its arguments, with a norm: the gradients of its inputs.  dq_out may be dq itself."""
    code = _choice({"head": 1, "row": 2}, norm, "qk_norm_rotary_backward", "norm")
    return QkGradients(*_on(stream, _calls.qk_norm_rotary_backward, dq, dk, q, k, q_weight, k_weight, table, code, eps, _choice(_LAYOUTS, layout, "qk_norm_rotary_backward", "layout"), False, positions,
                            first, dq_out, dk_out))
