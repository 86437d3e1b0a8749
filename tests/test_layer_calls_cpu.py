"""Which calls the layers make, in which order and with what: their modules' calls are replaced by ones that write down what they are given.  No GPU."""
import pytest
import torch

from paper_2509_24899_b200 import build

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


class Attention:
    """What a layer asks of its attention: a shape, and `forward`."""

    def __init__(self, shape, **kw):
        self.shape = shape
        self.__dict__.update(kw)

    def forward(self, q, k, v):
        return q


def fp8_layer(monkeypatch, log, shape, attention=None, **how):
    from paper_2509_24899_b200 import fp8_layer as module
    B, H, N, d = shape

    def rms_norm(x, weight, eps=1e-6, out=None, residual=None, fp8=False):
        log.append(("norm", None if weight is None else chr(int(weight[0]))))
        return (x, residual) if residual is not None else x

    def matmul_fp8(a, w, bias=None, out=None):
        log.append(("product", chr(int(w[0, 0]))))
        return out if out is not None else torch.zeros(B * N, H * d, dtype=BF16)

    def qk_norm_rotary(*args, **kw):
        log.append(("turn", args[4], kw))

    monkeypatch.setattr(module, "quantize_fp8", lambda x, block_rows=1: x)
    for f in (rms_norm, matmul_fp8, qk_norm_rotary):
        monkeypatch.setattr(module, f.__name__, f)
    w = {n: torch.full((H * d, H * d), float(ord(n)), dtype=BF16) for n in "qkvo"}
    w.update({"norm_" + n: torch.full((H * d,), float(ord(n)), dtype=BF16) for n in "qk"})
    return module.Fp8AttentionLayer(attention or Attention(shape), w, {}, **how)


def test_the_8_bit_layer_holds_one_product_at_a_time(monkeypatch):
    shape, log = (1, 2, 3, 4), []
    layer = fp8_layer(monkeypatch, log, shape)
    layer.forward(torch.zeros(3, 8, dtype=BF16), torch.zeros(3, 8, dtype=BF16))
    assert log == [("norm", None), ("product", "q"), ("norm", "q"), ("product", "k"), ("norm", "k"), ("product", "v"), ("product", "o")]


@pytest.mark.parametrize("attention,how,want", [({}, {}, (0, None)), ({}, dict(first=7), (7, None)), (dict(n0=5), {}, (5, None)), (dict(n0=5), dict(first=0), (0, None)), (dict(n0=5), dict(positions="here"), (0, "here"))])
def test_where_a_layers_tokens_begin(monkeypatch, attention, how, want):
    """In the grid of the layer's table: where it is said, else where the attention's range of a clip begins."""
    from paper_2509_24899_b200 import layer as module
    shape, log = (1, 2, 3, 4), []
    fp8_layer(monkeypatch, log, shape, Attention(shape, **attention), table="table", **how).forward(torch.zeros(3, 8, dtype=BF16), torch.zeros(3, 8, dtype=BF16))
    turns = [e for e in log if e[0] == "turn"]

    def linear(x, w, bias=None, out=None, **kw):
        return torch.zeros(x.shape[0] if x.dim() == 2 else 3, w.shape[0], dtype=BF16) if out is None else out

    def qk_norm_rotary(q, k, wq, wk, table=None, **kw):
        turns.append(("turn", table, kw))
        return q, k

    def qk_norm_rotary_backward(dq, dk, q, k, wq, wk, table=None, **kw):
        turns.append(("turn", table, kw))
        raise InterruptedError

    for f in (linear, qk_norm_rotary, qk_norm_rotary_backward):
        monkeypatch.setattr(module, f.__name__, f)
    monkeypatch.setattr(module, "rms_norm", lambda x, w, eps: x)
    w = {n: torch.zeros(8, 8, dtype=BF16) for n in ("q", "k", "v", "o", "up", "down")}
    layer = module.AttentionLayer(Attention(shape, **attention), w, {}, "table", **how)
    layer.forward(torch.zeros(3, 8, dtype=BF16))
    _, kept = layer.qk.forward(torch.zeros(3, 8, dtype=BF16), keep=True)
    with pytest.raises(InterruptedError):
        layer.qk.backward(None, None, kept)
    assert [(t[1], t[2]["first"], t[2]["positions"]) for t in turns] == [("table", *want)] * 4
