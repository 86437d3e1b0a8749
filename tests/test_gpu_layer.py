"""The steps around the attention run together, as a layer runs them: the bf16 layer, the 8-bit one with a rotation, and the gradients of the parts that have some."""
import pytest
import torch

from tests import _layer as R

pytestmark = pytest.mark.gpu

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
# A chain of products whose operands are rounded to bf16, each rounding independent and at most 2^-8 relative, 2^-8 / sqrt 3 in the mean: nine of them, the deepest chain here, stay below 2^-8 * 3 ** 0.5,
# and norms, gates and activations change a relative error by less than twice.
CHAIN = 2.0 ** -6


@pytest.fixture(scope="module", autouse=True)
def ops():
    import paper_2509_24899_b200 as pkg
    yield pkg
    torch.cuda.synchronize()
    assert pkg.fp8_last_status() == 0


def randn(*shape, dtype=BF16, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * gain).to(dtype)


def near(got, want, what, tol=CHAIN):
    got, want = got.to(F64), want.to(F64)
    assert got.shape == want.shape and bool(got.isfinite().all())
    off = float((got - want).norm() / want.norm())
    assert off <= tol, (what, off)


def table_of(ops, sizes, d):
    third = d // 6
    return ops.rotary_table(sizes, (d // 2 - 2 * third, third, third))


def qk64(x, w, bias, norms, table, shape, norm, layout):
    B, H, N, d = shape
    rows = x @ w.T + bias
    out = []
    for part, weight in zip((rows[:, :H * d], rows[:, H * d:]), norms):
        n, _, s = R.normed64(R.heads_of(part, B, d), weight, norm, 1e-6)
        out.append(R.turn64(n * s, R.factors64(table, B, N), layout))
    return out


@pytest.mark.parametrize("norm,layout,shape,sizes", [("row", "interleaved", (2, 4, 24, 64), (2, 3, 4)), ("head", "half", (1, 3, 130, 128), (5, 2, 13)), ("row", "half", (1, 5, 20, 40), (20,))])
def test_projection_of_queries_and_keys(ops, norm, layout, shape, sizes):
    from paper_2509_24899_b200.layer import QkProjection
    B, H, N, d = shape
    K = 96
    table = table_of(ops, sizes, d) if len(sizes) == 3 else ops.rotary_table(sizes, (d // 2,))
    x, w, bias = randn(B * N, K, seed=1), randn(2 * H * d, K, seed=2, gain=K ** -0.5), randn(2 * H * d, seed=3, gain=0.1)
    n = H * d if norm == "row" else d
    norms = [1 + 0.2 * randn(n, dtype=F32, seed=4 + i) for i in range(2)]
    p = QkProjection(shape, w, bias, *norms, table, norm=norm, layout=layout)
    (q, k), kept = p.forward(x, keep=True)
    leaves = [t.to(F64).requires_grad_() for t in (x, w, bias, *norms)]
    want = qk64(leaves[0], leaves[1], leaves[2], leaves[3:], table, shape, norm, layout)
    near(q, want[0].detach(), "q")
    near(k, want[1].detach(), "k")
    plain = p.forward(x)
    assert torch.equal(plain[0], q) and torch.equal(plain[1], k)
    dq, dk = randn(*shape, seed=8), randn(*shape, seed=9)
    got = p.backward(dq, dk, kept)
    for name, g, ref in zip(got._fields, got, torch.autograd.grad(want, leaves, (dq.to(F64), dk.to(F64)))):
        near(g, ref, name)


@pytest.mark.parametrize("act", ["gelu_tanh", "silu"])
@pytest.mark.parametrize("gates", [0, 2])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_feed_forward(ops, act, gates, dtype):
    from paper_2509_24899_b200.layer import FeedForward
    m, k, f = 300, 128, 320
    x, w1, w2 = randn(m, k, seed=1), randn(f, k, seed=2, gain=k ** -0.5), randn(k, f, seed=3, gain=f ** -0.5)
    b1, b2, r = randn(f, seed=4, gain=0.1), randn(k, seed=5, gain=0.1), randn(m, k, dtype=dtype, seed=6)
    gate = randn(gates, k, dtype=F32, seed=7) if gates else None
    ff = FeedForward(w1, w2, b1, b2, act)
    y, kept = ff.forward(x, gate, r, keep=True)
    leaves = [t.to(F64).requires_grad_() for t in (x, w1, b1, w2, b2)] + ([gate.to(F64).requires_grad_()] if gates else [])
    h, _ = R.act64(leaves[0] @ leaves[1].T + leaves[2], act)
    z = h @ leaves[3].T + leaves[4]
    want = (z * leaves[5].repeat_interleave(m // gates, 0) if gates else z) + r.to(F64)
    assert y.dtype == dtype
    near(y, want.detach(), "y")
    assert torch.equal(ff.forward(x, gate, r), y)
    dy = randn(m, k, dtype=dtype, seed=8)
    got = ff.backward(dy, kept)
    refs = torch.autograd.grad(want, leaves, dy.to(F64))
    for name, g, ref in zip(got._fields, got, refs):
        near(g, ref, name)
    if not gates:
        assert got.gate is None


def layer_weights(H, d, F, seed=0):
    hd = H * d
    w = {n: randn(hd, hd, seed=seed + i, gain=hd ** -0.5) for i, n in enumerate("qkvo")}
    w["up"], w["down"] = randn(F, hd, seed=seed + 5, gain=hd ** -0.5), randn(hd, F, seed=seed + 6, gain=F ** -0.5)
    for i, n in enumerate(("q", "k", "v", "o", "up", "down")):
        w["bias_" + n] = randn(w[n].shape[0], seed=seed + 10 + i, gain=0.1)
    for i, n in enumerate(("norm", "norm_ff", "norm_q", "norm_k")):
        w[n] = (1 + 0.2 * randn(hd, dtype=F32, seed=seed + 20 + i)).to(BF16)
    return w


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_bf16_layer(ops, dtype):
    """The layer's calls against their formulas, with the attention's own results in between."""
    import numpy as np
    from paper_2509_24899_b200 import HybridAttention, workloads as W
    from paper_2509_24899_b200.layer import AttentionLayer
    wl = W.CONFIGS["tiny"]
    data = W.generate(wl, wq_gain=2e-3)
    phi = {n: torch.from_numpy(data[n].view(np.int16)).cuda().view(BF16) for n in ("wq", "wk")}
    B, H, N, d = wl.B, wl.H, wl.N, wl.d
    w, table = layer_weights(H, d, 256), table_of(ops, wl.grid, d)
    attention = HybridAttention.from_workload(wl)
    layer = AttentionLayer(attention, w, phi, table)
    stream, go, gf = randn(B * N, H * d, dtype=dtype, seed=30), randn(H * d, dtype=F32, seed=31), randn(B, H * d, dtype=F32, seed=32)
    before = stream.clone()
    got = layer.forward(stream, go, gf)
    assert got.dtype == dtype and torch.equal(stream, before) and attention.last_status() == 0

    def norm(t, weight):
        return t / torch.sqrt(t.square().mean(1, keepdim=True) + 1e-6) * weight.to(F64)

    u = {n: t.to(F64) for n, t in w.items()}
    x = norm(stream.to(F64), u["norm"])
    q, k = qk64(x, torch.cat((u["q"], u["k"])), torch.cat((u["bias_q"], u["bias_k"])), (u["norm_q"], u["norm_k"]), table, (B, H, N, d), "row", "interleaved")
    v = R.heads_of(x @ u["v"].T + u["bias_v"], B, d)
    o = attention.forward(q.to(BF16).contiguous(), k.to(BF16).contiguous(), v.to(BF16).contiguous(), **phi)
    t = stream.to(F64) + go.to(F64) * (R.rows_of(o.to(F64)) @ u["o"].T + u["bias_o"])
    h, _ = R.act64(norm(t, u["norm_ff"]) @ u["up"].T + u["bias_up"], "gelu_tanh")
    want = t + gf.to(F64).repeat_interleave(N, 0) * (h @ u["down"].T + u["bias_down"])
    near(got, want, "stream")
    # two calls on one stream, and captured
    again = layer.forward(stream, go, gf)
    assert torch.equal(again, got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = layer.forward(stream, go, gf)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, got)


def test_the_8_bit_layer_with_a_rotation(ops):
    """Turned queries and keys reach the attention: the layer's result is that of its own calls made one by one; without a table, as it was."""
    import numpy as np
    from paper_2509_24899_b200 import HybridAttention, workloads as W
    from paper_2509_24899_b200.fp8_layer import Fp8AttentionLayer
    wl = W.CONFIGS["tiny"]
    data = W.generate(wl, wq_gain=2e-3)
    phi = {n: torch.from_numpy(data[n].view(np.int16)).cuda().view(BF16) for n in ("wq", "wk")}
    B, H, N, d = wl.B, wl.H, wl.N, wl.d
    w = {n: t for n, t in layer_weights(H, d, 256).items() if "up" not in n and "down" not in n and n != "norm_ff"}
    table = table_of(ops, wl.grid, d)
    attention = HybridAttention.from_workload(wl)
    hidden, residual = randn(B * N, H * d, seed=1), randn(B * N, H * d, dtype=F32, seed=2)
    turned, r1 = Fp8AttentionLayer(attention, w, phi, table=table).forward(hidden, residual)
    plain, r2 = Fp8AttentionLayer(attention, w, phi).forward(hidden, residual)
    assert torch.equal(r1, r2) and not torch.equal(turned, plain)
    x8, _ = ops.rms_norm(hidden, w["norm"], residual=residual, fp8=True)
    w8 = {n: ops.quantize_fp8(w[n], block_rows=128) for n in "qkvo"}
    q, k = (ops.matmul_fp8(x8, w8[n], bias=w["bias_" + n]) for n in "qk")
    v = ops.matmul_fp8(x8, w8["v"], bias=w["bias_v"], out=torch.empty(B, H, N, d, dtype=BF16, device="cuda"))
    cs = R.factors64(table, B, N)
    for rows, weight in ((q, w["norm_q"]), (k, w["norm_k"])):
        heads = R.heads_of(rows, B, d)
        R.check_forward(ops.qk_norm_rotary(heads, None, weight, None, table, norm="row"), heads, weight, cs, "row", 1e-6, "interleaved")
    q, k = (ops.qk_norm_rotary(R.heads_of(r, B, d), None, n, None, table, norm="row") for r, n in ((q, w["norm_q"]), (k, w["norm_k"])))
    o = attention.forward(q, k, v, **phi)
    assert torch.equal(ops.matmul_fp8(ops.quantize_fp8(o), w8["o"], bias=w["bias_o"]), turned)


@pytest.mark.parametrize("way", ["first", "positions"])
def test_ranges_of_a_clips_tokens(ops, way):
    """Two ranges of a clip's tokens, as two ranks have them, turned by the clip's table: queries, keys and gradients are the whole clip's; so are the results of both layers."""
    from paper_2509_24899_b200.fp8_layer import Fp8AttentionLayer
    from paper_2509_24899_b200.layer import AttentionLayer, QkProjection
    H, d, sizes = 3, 64, (3, 5, 6)
    N, hd = 90, H * d
    table = table_of(ops, sizes, d)
    grid = torch.stack(torch.meshgrid(*(torch.arange(s) for s in sizes), indexing="ij"), -1).reshape(N, 3).int().cuda()
    ranges = ((0, 37), (37, N))

    def where(a, b):
        return dict(first=a) if way == "first" else dict(positions=grid[a:b])

    x, w = randn(N, 96, seed=1), randn(2 * hd, 96, seed=2, gain=96 ** -0.5)
    norms = [1 + 0.2 * randn(hd, dtype=F32, seed=4 + i) for i in range(2)]
    dq, dk = randn(1, H, N, d, seed=8), randn(1, H, N, d, seed=9)

    def parts(shape, x, dq, dk, **how):
        p = QkProjection(shape, w, None, *norms, table, **how)
        qk, kept = p.forward(x, keep=True)
        return qk, p.backward(dq, dk, kept)

    qk, g = parts((1, H, N, d), x, dq, dk)
    some = [parts((1, H, b - a, d), x[a:b], dq[:, :, a:b], dk[:, :, a:b], **where(a, b)) for a, b in ranges]
    for i in range(2):
        near(torch.cat([s[0][i] for s in some], 2), qk[i], "qk"[i])
    near(torch.cat([s[1].x for s in some]), g.x, "x")
    for name in ("w", "norm_q", "norm_k"):
        near(sum(getattr(s[1], name).to(F64) for s in some), getattr(g, name), name)

    class Attention:                                          # of a range: its queries, keys and values for the results
        def __init__(self, a, b):
            self.shape, self.n0 = (1, H, b - a, d), a

        def forward(self, q, k, v):
            return q + k + v

    weights, rows = layer_weights(H, d, 128), randn(N, hd, seed=10)
    for make, call in ((AttentionLayer, lambda l, r: l.forward(r)), (Fp8AttentionLayer, lambda l, r: l.forward(r, r)[0])):
        def result(a, b, **how):
            return call(make(Attention(a, b), weights, {}, table=table, **how), rows[a:b])
        whole = result(0, N)
        near(torch.cat([result(a, b, **(where(a, b) if way == "positions" else {})) for a, b in ranges]), whole, make.__name__)
        assert float((result(37, N, first=0).to(F64) - whole[37:].to(F64)).norm() / whole[37:].to(F64).norm()) > 2 * CHAIN      # (what a range at another place gives)
