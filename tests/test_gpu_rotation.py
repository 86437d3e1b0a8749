"""Rotation and the norms of queries and keys on a GPU against their formulas in 64 bits: layouts, sizes and strides where they can go wrong, positions, ranges of values, gradients."""
import math

import pytest
import torch

from tests import _layer as R
from tests._util import Guarded

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def ops():
    import paper_2509_24899_b200 as pkg
    yield pkg
    torch.cuda.synchronize()


def randn(*shape, dtype=BF16, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * gain).to(dtype)


def plain_table(sizes, pairs, **how):
    return (R.table64(sizes, pairs, **how).to(F32).cuda(), tuple(sizes), tuple(pairs))


# ------------------------------------------------------------------------------------------------ the table
@pytest.mark.parametrize("sizes,pairs,how", [
    ((1,), (1,), {}), ((7,), (1,), dict(scaling="ntk", factor=4.0)), ((5, 6, 7), (22, 21, 21), {}), ((300, 1), (3, 65), dict(base=500000.0)), ((2, 3, 4, 5), (1, 2, 3, 4), {}),
    ((20000,), (32,), dict(scaling="yarn", factor=8.0, original=4096.0)), ((20000,), (64,), dict(scaling="linear", factor=3.0)), ((20000,), (64,), dict(scaling="ntk", factor=16.0)),
    ((1 << 20,), (2,), {})])
def test_table(ops, sizes, pairs, how):
    got = ops.rotary_table(sizes, pairs, **how)
    assert got.sizes == sizes and got.pairs == pairs and got.factors.shape == (sum(sizes), sum(pairs), 2)
    # an angle: 2^-53 of the position's turns a few times over (below 2^20: 2^-30 of a turn); a value: a rounding of its argument, 2 ulp of sinpi and cospi and the result's rounding, 2^-21
    ref = R.table64(sizes, pairs, **how)
    R.within(got.factors.cpu(), ref, ref.abs() * 2.0 ** -21 + math.tau * 2.0 ** -30 * 1.5)


def test_table_of_one_choice_for_each_axis(ops):
    got = ops.rotary_table((9, 10), (4, 6), base=(100.0, 10000.0), scaling=("linear", None), factor=(2.0, 1.0))
    ref = torch.zeros(19, 10, 2, dtype=R.F64)
    ref[:9, :4] = R.table64((9,), (4,), base=100.0, scaling="linear", factor=2.0)
    ref[9:, 4:] = R.table64((10,), (6,))
    R.within(got.factors.cpu(), ref, ref.abs() * 2.0 ** -21 + 1e-8)


# ------------------------------------------------------------------------------------------------ rotation
SHAPES = [(1, 1, 1, 2), (1, 2, 33, 64), (2, 12, 50, 128), (3, 5, 7, 40), (2, 3, 31, 8), (1, 9, 20, 17), (2, 4, 9, 96), (1, 3, 70, 256), (1, 2, 5, 512), (1, 1, 3, 1000), (1, 40, 300, 80),
          (4, 6, 1, 128), (1, 1, 2000, 64), (1, 7, 3, 1024), (1, 5, 9, 144), (2, 3, 11, 176), (1, 3, 40, 24), (2, 9, 30, 72), (1, 2, 7, 272), (1, 3, 300, 384), (1, 4, 5, 248)]


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,H,N,d", SHAPES)
def test_rotary(ops, B, H, N, d, dtype, layout):
    x = randn(B, H, N, d, dtype=dtype, seed=N)
    for pairs in sorted({d // 2, d // 4 // 8 * 8, max(1, d // 3)} - {0}):
        if pairs > d // 2:
            continue
        table = plain_table((N + 3,), (pairs,))
        cs = R.factors64(table, B, N, first=2)
        R.check_forward(ops.rotary(x, table, layout=layout, first=2), x, None, cs, None, 0, layout, "all")
        R.check_forward(ops.rotary(x, table, layout=layout, first=2, inverse=True), x, None, cs, None, 0, layout, "inverse", inverse=True)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("sizes,pairs,d", [((3, 4, 5), (22, 21, 21), 128), ((60, 1, 1), (8, 8, 16), 64), ((2, 5, 6), (3, 3, 4), 20), ((3, 4, 5), (10, 11, 11), 96), ((2, 2, 3, 5), (8, 3, 2, 11), 64),
                                           ((10, 6), (31, 33), 130)])
def test_rotary_on_grids(ops, sizes, pairs, d, layout):
    N = math.prod(sizes)
    x = randn(2, 3, N, d, seed=d)
    table = plain_table(sizes, pairs)
    for n, first in ((N, 0), (N - 7, 7), (1, N - 1)):
        y = ops.rotary(x[:, :, :n], table, layout=layout, first=first)
        R.check_forward(y, x[:, :, :n], None, R.factors64(table, 2, n, first=first), None, 0, layout)


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_positions_of_tokens(ops, kind):
    g = torch.Generator(device="cuda").manual_seed(3)
    for B, N, sizes, pairs, d in ((16, 1, (50,), (64,), 128), (2, 30, (50,), (9,), 40), (2, 9, (4, 5, 6), (22, 21, 21), 128)):
        x, table = randn(B, 3, N, d, seed=B), plain_table(sizes, pairs)
        shape = (B, N) if len(sizes) == 1 else (B, N, len(sizes))
        p = torch.stack([torch.randint(0, s, (B, N), generator=g, device="cuda") for s in sizes], -1).reshape(shape).to(kind)
        for layout in ("interleaved", "half"):
            R.check_forward(ops.rotary(x, table, layout=layout, positions=p), x, None, R.factors64(table, B, N, p), None, 0, layout)
            one = p[0].contiguous()
            R.check_forward(ops.rotary(x, table, layout=layout, positions=one), x, None, R.factors64(table, B, N, one), None, 0, layout)
        wide = torch.full((B, N + 4) + shape[2:], 77, dtype=kind, device="cuda")          # entries that lie in a wider tensor
        wide[:, 1:N + 1] = p
        assert torch.equal(ops.rotary(x, table, positions=wide[:, 1:N + 1]), ops.rotary(x, table, positions=p))


def test_positions_that_are_not_there_are_nan(ops):
    table = plain_table((10,), (8,))
    for d in (32, 18):                                     # vectors, and pair by pair
        x = randn(1, 2, 6, d, seed=d)
        for p in (torch.tensor([0, 9, 10, -1, 2 ** 31 - 1, -2 ** 31], device="cuda", dtype=torch.int32), torch.tensor([0, 9, 10, -1, 2 ** 62, -2 ** 62], device="cuda")):
            y = ops.rotary(x, table, positions=p)
            assert bool(y[:, :, 2:, :16].isnan().all()) and not bool(y[:, :, :2].isnan().any()) and torch.equal(y[..., 16:], x[..., 16:])
            R.check_forward(y, x, None, R.factors64(table, 1, 6, p), None, 0, "interleaved")


def test_rotary_strides_and_in_place(ops):
    B, H, N, d = 2, 6, 21, 64
    table = plain_table((N,), (32,))
    cs = R.factors64(table, B, N)
    wide = randn(B * N, 3 * H * d + 1, seed=5)
    for shift in (0, 1, 8, H * d):
        x = wide[:, shift:shift + H * d].reshape(B, N, H, d).permute(0, 2, 1, 3) if shift == 0 else wide[:, shift:shift + H * d].unflatten(1, (H, d)).unflatten(0, (B, N)).permute(0, 2, 1, 3)
        R.check_forward(ops.rotary(x, table), x, None, cs, None, 0, "interleaved")
    even = randn(B, N, 2 * H, d, seed=6)
    x = even[:, :, ::2].permute(0, 2, 1, 3)
    want = ops.rotary(x, table, layout="half")
    out = torch.full((B, N, H, d), 3.0, dtype=BF16, device="cuda").permute(0, 2, 1, 3)
    assert ops.rotary(x, table, layout="half", out=out) is out and torch.equal(out, want)
    keep = even[:, :, 1::2].clone()
    assert ops.rotary(x, table, layout="half", out=x) is x and torch.equal(x, want) and torch.equal(even[:, :, 1::2], keep)
    alike = randn(1, 1, 1, d, seed=7).expand(B, H, N, d)       # one head for all
    R.check_forward(ops.rotary(alike, table), alike, None, cs, None, 0, "interleaved")


@pytest.mark.parametrize("d,pairs", [(64, 32), (50, 11)])
def test_nothing_is_written_beside_the_output(ops, d, pairs):
    B, H, N = 2, 3, 37
    x = randn(B, H, N, d, seed=1)
    buf = Guarded(B * H * N * d * 2)
    out = buf.view(BF16, (B, H, N, d))
    ops.qk_norm_rotary(x, None, randn(d, seed=2), None, plain_table((N,), (pairs,)), q_out=out)
    torch.cuda.synchronize()
    buf.check()


def test_turned_and_turned_back(ops):
    """Of powers of two in fp32 with a table of quarter turns everything is exact."""
    table = (torch.tensor([[1., 0.], [0., 1.], [-1., 0.], [0., -1.]], device="cuda").reshape(4, 1, 2).expand(4, 16, 2).contiguous(), (4,), (16,))
    x = torch.exp2(torch.randint(-20, 20, (1, 2, 4, 48), device="cuda").float())
    for layout in ("interleaved", "half"):
        y = ops.rotary(x, table, layout=layout)
        assert torch.equal(y.to(R.F64), R.turn64(x, R.factors64(table, 1, 4), layout))
        assert torch.equal(ops.rotary(y, table, layout=layout, inverse=True), x)


# ------------------------------------------------------------------------------------------------ norms
QK = [(1, 1, 1, 1, 2), (1, 12, 12, 5, 128), (2, 12, 3, 50, 128), (3, 5, 2, 7, 40), (1, 24, 24, 19, 64), (1, 9, 9, 20, 17), (2, 4, 1, 9, 96), (1, 3, 3, 30, 256), (1, 2, 2, 5, 512),
      (1, 64, 8, 11, 128), (1, 128, 128, 3, 128), (1, 1, 1, 700, 1000), (4, 6, 6, 1, 128), (1, 12, 12, 700, 128), (1, 1, 7, 33, 80), (1, 5, 2, 9, 144), (2, 3, 3, 11, 176), (1, 9, 9, 40, 24), (2, 12, 4, 300, 72), (1, 30, 30, 9, 248), (1, 2, 1, 30, 384)]


@pytest.mark.parametrize("norm", ["head", "row"])
@pytest.mark.parametrize("dtype,wd", [(BF16, BF16), (BF16, F32), (F32, F32), (BF16, None)])
@pytest.mark.parametrize("B,H,Hk,N,d", QK)
def test_norm_and_rotation(ops, B, H, Hk, N, d, dtype, wd, norm):
    q, k = randn(B, H, N, d, dtype=dtype, seed=N), randn(B, Hk, N, d, dtype=dtype, seed=N + 1, gain=3.0)
    wq, wk = (None if wd is None else (1 + 0.3 * randn(d * (h if norm == "row" else 1), dtype=F32, seed=h)).to(wd) for h in (H, Hk))
    for layout, pairs in (("interleaved", d // 2), ("half", d // 2), ("half", max(1, d // 4 // 8 * 8)), (None, 0)):
        table = plain_table((N,), (pairs,)) if layout else None
        cs = R.factors64(table, B, N) if layout else None
        gq, gk = ops.qk_norm_rotary(q, k, wq, wk, table, norm=norm, eps=1e-5, layout=layout or "half")
        R.check_forward(gq, q, wq, cs, norm, 1e-5, layout, "q")
        R.check_forward(gk, k, wk, cs, norm, 1e-5, layout, "k")
        assert torch.equal(ops.qk_norm_rotary(k, None, wk, None, table, norm=norm, eps=1e-5, layout=layout or "half"), gk)


@pytest.mark.parametrize("norm", ["head", "row"])
@pytest.mark.parametrize("dtype,wd", [(BF16, BF16), (BF16, F32), (F32, F32), (BF16, None)])
@pytest.mark.parametrize("B,H,Hk,N,d", QK)
def test_gradients(ops, B, H, Hk, N, d, dtype, wd, norm):
    q, k = randn(B, H, N, d, dtype=dtype, seed=N), randn(B, Hk, N, d, dtype=dtype, seed=N + 1, gain=3.0)
    dq, dk = randn(B, H, N, d, dtype=dtype, seed=N + 2), randn(B, Hk, N, d, dtype=dtype, seed=N + 3, gain=1e-3)
    wq, wk = (None if wd is None else (1 + 0.3 * randn(d * (h if norm == "row" else 1), dtype=F32, seed=h)).to(wd) for h in (H, Hk))
    for layout, pairs in (("interleaved", d // 2), ("half", max(1, d // 4 // 8 * 8)), (None, 0)):
        table = plain_table((N,), (pairs,)) if layout else None
        cs = R.factors64(table, B, N) if layout else None
        got = ops.qk_norm_rotary_backward(dq, dk, q, k, wq, wk, table, norm=norm, eps=1e-5, layout=layout or "half")
        assert (got.q_weight is None) == (wd is None) == (got.k_weight is None)
        R.check_backward(got.q, dq, q, wq, cs, norm, 1e-5, layout, got.q_weight, "q")
        R.check_backward(got.k, dk, k, wk, cs, norm, 1e-5, layout, got.k_weight, "k")
        alone = ops.qk_norm_rotary_backward(dk, None, k, None, wk, None, table, norm=norm, eps=1e-5, layout=layout or "half")
        assert torch.equal(alone.q, got.k) and alone.k is None and alone.k_weight is None


def test_gradients_against_differences(ops):
    """The forward call's own results along a direction, in fp32, against the gradients along it."""
    for norm in ("head", "row"):
        q, w = randn(1, 2, 3, 32, dtype=F32, seed=1), 1 + 0.3 * randn(64 if norm == "row" else 32, dtype=F32, seed=2)
        dy, table = randn(1, 2, 3, 32, dtype=F32, seed=3), plain_table((3,), (16,))
        got = ops.qk_norm_rotary_backward(dy, None, q, None, w, None, table, norm=norm)
        h = 2.0 ** -8
        for v, u, name in ((randn(1, 2, 3, 32, dtype=F32, seed=4), 0 * w, "x"), (0 * q, randn(w.numel(), dtype=F32, seed=5), "w")):
            y = [(ops.qk_norm_rotary(q + s * h * v, None, w + s * h * u, None, table, norm=norm).to(R.F64) * dy.to(R.F64)).sum() for s in (1, -1)]
            along = (got.q.to(R.F64) * v.to(R.F64)).sum() + (got.q_weight.to(R.F64) * u.to(R.F64)).sum()
            # a difference of values that are 2^-20 off, over 2 h: 192 terms of up to 10 in size; and h^2 of third derivatives of size 10
            assert abs(float((y[0] - y[1]) / (2 * h) - along)) <= 192 * 10 * 2.0 ** -20 / (2 * h) / 8 + 200 * h * h, name


@pytest.mark.parametrize("d,pairs", [(64, 32), (34, 10)])
@pytest.mark.parametrize("norm", ["head", "row"])
def test_range(ops, norm, d, pairs):
    """Tokens of zeros, of huge and of tiny values, each beside ordinary ones; infinities and NaN stay in their head (row)."""
    x = randn(1, 3, 9, d, dtype=F32, seed=8)
    x[:, :, 1] = 0
    x[:, :, 2] *= 1e-25
    x[:, :, 3] *= 1e30
    x[:, :, 4] = x[:, :, 4].clamp(-1, 1) * 3e38
    x[:, :, 5] *= 1e-38
    x[:, 1, 6, 3] = float("nan")
    x[:, 1, 7, 4] = float("inf")
    table = plain_table((9,), (pairs,))
    cs = R.factors64(table, 1, 9)
    w = 1 + 0.3 * randn(3 * d if norm == "row" else d, dtype=F32, seed=1)
    hit = (slice(None), slice(None) if norm == "row" else slice(1, 2), slice(6, 8))
    for eps in (1e-6, 0.0):
        y = ops.qk_norm_rotary(x, None, w, None, table, norm=norm, eps=eps)
        dy = randn(1, 3, 9, d, dtype=F32, seed=9)
        back = ops.qk_norm_rotary_backward(dy, None, x, None, w, None, table, norm=norm, eps=eps).q
        ok = torch.ones(1, 3, 9, 1, dtype=torch.bool, device="cuda")
        ok[hit] = False
        if eps == 0.0:
            assert bool(y[:, :, 1].isnan().all())
            ok[:, :, 1] = False
        n, r, scale = R.normed64(x, w, norm, eps)
        ref, size = R.turn64(n * scale, cs, "interleaved"), R.size_of_turn(n * scale, cs, "interleaved")
        ok4 = ok.expand_as(y)
        R.within(y[ok4], ref[ok4], ref[ok4].abs() * 2.0 ** -24 + size[ok4] * R.SLACK + 1e-37)
        for t in range(9):
            if bool(ok[0, :, t].all()) and not (eps == 0.0 and t == 5):                # (there the gradient itself lies beyond fp32)
                x1 = x[:, :, t:t + 1]
                d1 = R.turn64(dy[:, :, t:t + 1], tuple(v[:, :, t:t + 1] for v in cs), "interleaved", inverse=True)
                s1 = R.size_of_turn(dy[:, :, t:t + 1], tuple(v[:, :, t:t + 1] for v in cs), "interleaved")
                n1, r1, w1 = R.normed64(x1, w, norm, eps)
                dims = (3,) if norm == "head" else (1, 3)
                ref1 = r1 * (d1 * w1 - n1 * (d1 * w1 * n1).mean(dims, keepdim=True))
                reach = r1 * (s1 * w1.abs() + n1.abs() * (s1 * w1.abs() * n1.abs()).mean(dims, keepdim=True))
                R.within(back[:, :, t:t + 1], ref1, ref1.abs() * 2.0 ** -24 + reach * 2 * R.SLACK + 1e-37, "gradient of token %d" % t)
        assert bool(y[:, 1, 6].isnan().all())


def test_many_rows_and_heads(ops):
    """Turns of several rows a CTA, partial sums of many CTAs; the same bits from run to run."""
    q, dq, w = randn(1, 12, 7000, 128, seed=1), randn(1, 12, 7000, 128, seed=2), 1 + 0.2 * randn(128, seed=3)
    table = plain_table((5, 35, 40), (22, 21, 21))
    cs = R.factors64(table, 1, 7000)
    R.check_forward(ops.qk_norm_rotary(q, None, w, None, table), q, w, cs, "head", 1e-6, "interleaved")
    one, two = (ops.qk_norm_rotary_backward(dq, None, q, None, w, None, table) for _ in range(2))
    assert torch.equal(one.q, two.q) and torch.equal(one.q_weight, two.q_weight)
    R.check_backward(one.q, dq, q, w, cs, "head", 1e-6, "interleaved", one.q_weight)


def test_offsets_past_32_bits(ops):
    """Tokens that lie 2^32 elements and more into their tensor."""
    need = (1 << 32) + 4096
    if torch.cuda.mem_get_info()[0] < need * 2 + (1 << 30):
        pytest.skip("not enough memory")
    flat = torch.empty(need, dtype=BF16, device="cuda")
    x = flat.as_strided((1, 2, 2, 64), (0, 64, 1 << 32, 1))
    x.copy_(randn(1, 2, 2, 64, seed=1))
    table = plain_table((2,), (32,))
    R.check_forward(ops.qk_norm_rotary(x, None, None, None, table), x, None, R.factors64(table, 1, 2), "head", 1e-6, "interleaved")
    ops.rotary(x, table, out=x)


def test_no_tokens(ops):
    q, w = randn(2, 3, 0, 64), randn(64, seed=1)
    table = plain_table((4,), (32,))
    a, b = ops.qk_norm_rotary(q, q, w, w, table)
    assert a.shape == b.shape == q.shape and ops.rotary(q, table).shape == q.shape
    got = ops.qk_norm_rotary_backward(q, q, q, q, w, w, table)
    assert bool((got.q_weight == 0).all()) and bool((got.k_weight == 0).all()) and got.q.shape == q.shape


def test_streams_and_graphs(ops):
    q, k, w = randn(1, 4, 100, 64, seed=1), randn(1, 4, 100, 64, seed=2), randn(64, seed=3)
    table = plain_table((100,), (32,))
    want = ops.qk_norm_rotary(q, k, w, w, table)
    grads = ops.qk_norm_rotary_backward(q, k, q, k, w, w, table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.qk_norm_rotary(q, k, w, w, table, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = ops.qk_norm_rotary(q, k, w, w, table)
            d = ops.qk_norm_rotary_backward(q, k, q, k, w, w, table)
        graphs.append((g, y, d))
    for t in (q, k):
        t.neg_()
    for g, _, _ in graphs:
        g.replay()
    for t in (q, k):
        t.neg_()
    for g, y, d in graphs:
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y[0], want[0]) and torch.equal(y[1], want[1])
        assert all(torch.equal(a, b) for a, b in zip(d, grads))


def test_refusals(ops):
    q, w = randn(2, 3, 5, 64), randn(64, seed=1)
    table = plain_table((5,), (32,))
    f, s, p = table
    bad = [lambda: ops.rotary(q[0], table), lambda: ops.rotary(q.half(), table), lambda: ops.rotary(q.cpu(), table), lambda: ops.rotary(q, (f, s)), lambda: ops.rotary(q, (f, (6,), p)),
           lambda: ops.rotary(q, (f.double(), s, p)), lambda: ops.rotary(q, (f, s, (16, 16))), lambda: ops.rotary(q, (f[::2], (3,), p)), lambda: ops.rotary(q, table, layout="both"),
           lambda: ops.rotary(q, table, positions=torch.zeros(5, device="cuda")), lambda: ops.rotary(q, table, positions=torch.zeros(4, dtype=torch.int32, device="cuda")),
           lambda: ops.rotary(q, table, positions=torch.zeros(3, 5, dtype=torch.int32, device="cuda")), lambda: ops.rotary(q, table, positions=torch.zeros(10, dtype=torch.int32, device="cuda")[::2]),
           lambda: ops.rotary(q, table, first=1, positions=torch.zeros(5, dtype=torch.int32, device="cuda")), lambda: ops.rotary(q, table, out=torch.empty(2, 3, 5, 64, device="cuda")),
           lambda: ops.rotary(q, table, out=q[:, :, :4]), lambda: ops.rotary(q.transpose(2, 3), plain_table((64,), (2,))), lambda: ops.rotary(q.clone().requires_grad_(), table),
           lambda: ops.qk_norm_rotary(q, q[:, :, :4], w, w, table), lambda: ops.qk_norm_rotary(q, q.float(), w, w, table), lambda: ops.qk_norm_rotary(q, q, w[:32], w, table),
           lambda: ops.qk_norm_rotary(q, q, w, w.float(), table), lambda: ops.qk_norm_rotary(q, q, w, w, table, norm="row"), lambda: ops.qk_norm_rotary(q, q, w, w, table, norm="token"),
           lambda: ops.qk_norm_rotary(q, q, w, None, table, norm=None), lambda: ops.qk_norm_rotary(q, None, w, w, table), lambda: ops.qk_norm_rotary(q, None, w, None, None, positions=torch.zeros(5, dtype=torch.int32, device="cuda")),
           lambda: ops.qk_norm_rotary_backward(q, None, q, q, w, w, table), lambda: ops.qk_norm_rotary_backward(q.float(), q, q, q, w, w, table),
           lambda: ops.qk_norm_rotary_backward(q, q, q, q, w, w, table, norm=None), lambda: ops.rotary_table((5,), (1, 2)), lambda: ops.rotary_table((0,), (1,)), lambda: ops.rotary_table((5,), (3,), scaling="more"),
           lambda: ops.rotary_table((5, 5), (1, 1), factor=(1.0,)), lambda: ops.rotary_table((1, 1, 1, 1, 1), (1, 1, 1, 1, 1))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)
    refused = [lambda: ops.rotary(q, table, first=1), lambda: ops.rotary(q, table, first=-1), lambda: ops.rotary(q, plain_table((5,), (33,))), lambda: ops.rotary(q.expand(2, 3, 5, 64), table, out=q[:1].expand(2, 3, 5, 64)),
               lambda: ops.qk_norm_rotary(q, q, w, w, table, eps=-1.0), lambda: ops.qk_norm_rotary(q, q, w, w, table, eps=float("nan")), lambda: ops.qk_norm_rotary(randn(1, 300, 2, 64), None, norm="row"),
               lambda: ops.rotary_table((5,), (3,), base=0.0), lambda: ops.rotary_table((5,), (3,), scaling="linear", factor=0.5), lambda: ops.rotary_table((5,), (3,), scaling="yarn", factor=2.0)]
    for i, call in enumerate(refused):
        with pytest.raises(ops.AsError):
            call()
            print("not refused:", i)
    out = q.clone()
    version = out._version
    ops.rotary(q, table, out=out)
    assert out._version > version
    with torch.no_grad():
        ops.rotary(q.clone().requires_grad_(), table)


def test_refuses_results_over_other_tensors(ops):
    """A result at an input's address, but for its own input's in the same layout."""
    q, k, w, table = randn(1, 2, 2, 64), randn(1, 2, 2, 64, seed=1), randn(64, seed=2), plain_table((2,), (32,))
    crossed = q.transpose(1, 2)                          # [1, 2, 2, 64] again, tokens and heads exchanged
    for f in (lambda: ops.rotary(q, table, out=crossed), lambda: ops.qk_norm_rotary(q, k, w, w, table, q_out=k), lambda: ops.qk_norm_rotary(q, k, w, w, table, k_out=q),
              lambda: ops.qk_norm_rotary(q, q, w, w, table, q_out=q), lambda: ops.qk_norm_rotary(q, k, w, w, table, q_out=torch.empty_like(q), k_out=k.transpose(1, 2)),
              lambda: ops.qk_norm_rotary_backward(q, k, q.clone(), k.clone(), w, w, table, dq_out=k), lambda: ops.qk_norm_rotary_backward(q, k, q.clone(), k.clone(), w, w, table, dk_out=q),
              lambda: ops.qk_norm_rotary_backward(q, k, q.clone(), k.clone(), w, w, table, dq_out=crossed)):
        with pytest.raises(ops.AsError):
            f()
    want = ops.qk_norm_rotary(q, k, w, w, table)
    ops.qk_norm_rotary(q, k, w, w, table, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_host_threads_with_calls_of_different_sizes(ops):
    """Two threads launch the same kernels, one with 64 pairs (52 KB of shared memory and more), one with 32 (50 KB): neither call changes what the other one may take.  Through the C entries, which
    hold no lock (with a limit set by each call, 1566 of 80000 launches failed)."""
    import ctypes as C
    import threading
    from paper_2509_24899_b200 import binding as b
    n, d = 1000, 128
    wrong, turns = [], 8000

    def of(t):
        return b.as_rows_t(t.data_ptr(), b.AS_DTYPE_BF16, d, n, t.stride(0), t.stride(1), t.stride(2))

    def prepare(pairs):
        table = ops.rotary_table((n,), (pairs,))
        q, dq, out = randn(1, 12, n, d, seed=pairs), randn(1, 12, n, d, seed=pairs + 1), torch.empty(1, 12, n, d, dtype=BF16, device="cuda")
        a = b.as_qk_norm_rotary_t(struct_size=C.sizeof(b.as_qk_norm_rotary_t), norm=b.AS_NORM_HEAD, rows=n, head_dim=d, q_heads=12, eps=1e-6, q=of(q), q_out=of(out))
        a.rotation.table, a.rotation.n_axes, a.rotation.size[0], a.rotation.pairs[0] = table.factors.data_ptr(), 1, n, pairs
        back = b.as_qk_norm_rotary_backward_t(struct_size=C.sizeof(b.as_qk_norm_rotary_backward_t), fwd=C.pointer(a), dq=of(dq), dq_out=of(out))
        return a, back, (table, q, dq, out), torch.cuda.Stream()

    def work(a, back, keep, stream):
        for i in range(turns):
            for call, args in ((b.lib().as_qk_norm_rotary, a), (b.lib().as_qk_norm_rotary_backward, back)):
                status = call(C.addressof(args), stream.cuda_stream)
                if status != b.AS_OK:
                    wrong.append(status)

    calls = [prepare(pairs) for pairs in (64, 32, 64, 32)]
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=c) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, (len(wrong), set(wrong))
    for pairs, (_, _, (table, q, dq, out), _) in zip((64, 32, 64, 32), calls):
        assert torch.equal(out, ops.qk_norm_rotary_backward(dq, None, q, None, None, None, table).q)


def test_table_of_the_most_rows(ops):
    """2^31 - 1 positions of a pair: the last ones are there as well.  (An angle of 2^-53 relative over 2^31 / 2 pi turns: 2^-24 of a turn.)"""
    n = (1 << 31) - 1
    if torch.cuda.mem_get_info()[0] < n * 8 + (1 << 30):
        pytest.skip("not enough memory")
    torch.full((n, 1, 2), float("nan"), device="cuda")            # what the next tensor of this size lies over
    last = ops.rotary_table((n,), (1,)).factors[-200:].cpu()
    ref = torch.tensor([[[math.cos(r), math.sin(r)]] for r in range(n - 200, n)], dtype=R.F64)
    R.within(last, ref, ref.abs() * 2.0 ** -21 + math.tau * 2.0 ** -24 * 1.5)


def test_in_place_past_32_bits(ops):
    """Tokens that lie 2^32 elements into their tensor, turned where they are, in vectors and pair by pair."""
    need = (1 << 32) + 4096
    if torch.cuda.mem_get_info()[0] < need * 2 + (1 << 30):
        pytest.skip("not enough memory")
    flat = torch.zeros(need, dtype=BF16, device="cuda")
    for d, pairs in ((64, 32), (50, 11)):
        x = flat.as_strided((1, 2, 2, d), (0, d, 1 << 32, 1))
        was = randn(1, 2, 2, d, seed=d)
        x.copy_(was)
        table = plain_table((2,), (pairs,))
        assert ops.rotary(x, table, out=x) is x
        R.check_forward(x, was, None, R.factors64(table, 1, 2), None, 0, "interleaved")
        flat[:2 * d], flat[1 << 32:(1 << 32) + 2 * d] = 0, 0
        assert not bool(flat.view(torch.int16).any())            # nothing else has been written
