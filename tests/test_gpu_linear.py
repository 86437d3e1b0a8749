"""Linear layers on a GPU against their formulas in 64 bits: tiles, parts and rows where they can go wrong, layouts and strides, what follows the product, gradients."""
import itertools

import pytest
import torch

from tests import _layer as R
from tests._util import Guarded

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module", autouse=True)
def ops():
    import paper_2509_24899_b200 as pkg
    yield pkg
    torch.cuda.synchronize()
    assert pkg.fp8_last_status() == 0


def randn(*shape, dtype=BF16, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * gain).to(dtype)


def weights(n, k, seed=1):
    return randn(n, k, seed=seed, gain=k ** -0.5)


ROWS = [1, 2, 7, 8, 9, 15, 16, 17, 31, 64, 100, 127, 128, 129, 255, 256, 257, 300, 513, 1000]


@pytest.mark.parametrize("m", ROWS)
@pytest.mark.parametrize("n,k", [(8, 8), (40, 64), (256, 128), (200, 72), (512, 192), (1000, 1160), (64, 2048), (33, 65), (1, 1), (130, 200)])
def test_rows_and_widths(ops, m, n, k):
    x, w, b = randn(m, k, seed=m), weights(n, k), randn(n, seed=3)
    R.check_linear(ops.linear(x, w, bias=b), x, w, b)


@pytest.mark.parametrize("m", [3, 12, 40, 200, 700])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [96, 101])
def test_what_follows_the_product(ops, m, act, n):
    """Bias, activation, gate, residual and pre in every type, together and apart."""
    k = 128
    x, w = randn(m, k, seed=m, gain=2.0), weights(n, k)
    for i, (bd, gd, rd, pre) in enumerate(itertools.product((None, BF16, F32), (None, BF16, F32), (None, BF16, F32), (False, True))):
        b, g, r = (None if t is None else randn(*s, dtype=t, seed=i + j) for j, (t, s) in enumerate(((bd, (n,)), (gd, (n,)), (rd, (m, n)))))
        got = ops.linear(x, w, bias=b, activation=act, gate=g, residual=r, keep_pre=pre)
        y, z = got if pre else (got, None)
        assert y.dtype == (rd or BF16)
        R.check_linear(y, x, w, b, act, g, r, z)


@pytest.mark.parametrize("m,k,n", [(2048, 256, 512), (4096, 64, 1536), (1500, 1536, 1536), (300, 4096, 256), (5000, 520, 776), (20, 6144, 1536), (256, 8192, 64)])
def test_larger_products(ops, m, k, n):
    """Several turns of the tiles, parts of long sums; the same bits from run to run."""
    x, w, b, r = randn(m, k, seed=1), weights(n, k), randn(n, seed=3), randn(m, n, dtype=F32, seed=4)
    y = ops.linear(x, w, bias=b, activation="gelu_tanh", residual=r)
    R.check_linear(y, x, w, b, "gelu_tanh", None, r)
    assert torch.equal(y, ops.linear(x, w, bias=b, activation="gelu_tanh", residual=r))


@pytest.mark.parametrize("m", [4, 40, 300, 2000])
@pytest.mark.parametrize("k", [1536, 6144, 20000])
def test_long_sums_in_fp32(ops, m, k):
    """The matrix instructions truncate what they add up, 2^-23 of it at most and half of that in the mean, always towards 0: sums come in runs of 72 instructions at most (18 steps of 64 columns, and
    a third more in a tile's first run), so that the whole is off by less than 96 * 2^-24 in the mean.  (In one run of 384, for 6144 columns, it was 7e-6, of 1250, for 20000, 2e-5.)"""
    x, w = randn(m, k, seed=1).abs(), weights(192, k).abs()
    y = ops.linear(x, w, out=torch.empty(m, 192, dtype=F32, device="cuda"))
    ref = x.to(R.F64) @ w.to(R.F64).T
    assert float((y.to(R.F64) - ref).norm() / ref.norm()) <= 96 * 2.0 ** -24


@pytest.mark.parametrize("B,H,N,d", [(1, 2, 300, 64), (2, 12, 150, 128), (3, 5, 7, 40), (2, 3, 31, 8), (1, 9, 20, 17), (40, 4, 1, 64), (2, 4, 1030, 64), (1, 3, 9, 128), (5, 2, 3, 128)])
def test_heads(ops, B, H, N, d):
    """x, residual, out and pre in heads, each beside rows of the others; a gate for each entry."""
    x, w, b, g = randn(B, H, N, d, seed=N), weights(H * d, H * d), randn(H * d, seed=2), randn(B, H * d, dtype=F32, seed=3)
    R.check_linear(ops.linear(x, w, bias=b, gate=g), x, w, b, None, g)
    r = randn(B, H, N, d, dtype=F32, seed=4)
    y = ops.linear(x, w, bias=b, activation="silu", gate=g, residual=r)
    assert y.shape == r.shape and y.dtype == F32
    R.check_linear(y, x, w, b, "silu", g, r)
    flat = R.rows_of(x).contiguous()
    out, pre = torch.full((B, H, N, d), 7.0, dtype=BF16, device="cuda"), torch.full((B, N, H, d), 7.0, dtype=BF16, device="cuda").permute(0, 2, 1, 3)
    got = ops.linear(flat, w, bias=b, activation="gelu", out=out, keep_pre=pre)
    assert got[0] is out and got[1] is pre
    R.check_linear(out, flat, w, b, "gelu", None, None, pre)
    want = ops.linear(flat, w, bias=b, activation="silu", gate=g, residual=r)
    assert ops.linear(flat, w, bias=b, activation="silu", gate=g, residual=r, out=r) is r and torch.equal(r, want)      # in place


@pytest.mark.parametrize("m", [5, 130, 600])
@pytest.mark.parametrize("shift,stride", [(0, 192), (1, 192), (4, 192), (8, 200), (0, 193), (3, 196), (0, 0)])
def test_strides_and_alignment(ops, m, shift, stride):
    """Operands, results and vectors that begin and go on anywhere; all rows the same one."""
    k, n = 192, 136
    flat = randn(m * 256 + 4096, seed=9)
    x = flat[shift:].as_strided((m, k), (stride, 1), flat.storage_offset() + shift)
    w = randn(n * 256 + 4096, seed=10, gain=0.1)[shift:].as_strided((n, k), (max(stride, 192), 1), shift)
    b, g = randn(n + 16, seed=3)[shift:shift + n], randn(n + 16, seed=4)[shift:shift + n]
    big = torch.zeros(m, n + 30, dtype=F32, device="cuda")
    out = big[:, shift:shift + n]
    R.check_linear(ops.linear(x, w, bias=b, gate=g, out=out), x, w, b, None, g)
    assert not bool(big[:, :shift].any()) and not bool(big[:, shift + n:].any())
    R.check_linear(ops.linear(x, w, bias=b, gate=g), x, w, b, None, g)


@pytest.mark.parametrize("m,n", [(3, 37), (130, 100), (300, 513), (64, 1024)])
def test_nothing_is_written_beside_the_outputs(ops, m, n):
    k = 256
    x, w = randn(m, k, seed=1), weights(n, k)
    a, b = Guarded(m * n * 2), Guarded(m * n * 2)
    ops.linear(x, w, out=a.view(BF16, (m, n)), keep_pre=b.view(BF16, (m, n)))
    torch.cuda.synchronize()
    a.check("out")
    b.check("pre")
    R.check_linear(a.view(BF16, (m, n)), x, w, pre=b.view(BF16, (m, n)))


def test_activations_over_their_range(ops):
    """One column of weights that is 1: z is x; values from tiny to huge, infinities and NaN."""
    z = torch.cat([torch.linspace(-12, 12, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 87.0, -87.0, 200.0, -200.0, 1e4, -1e4, 3e38, -3e38])]).to(BF16).cuda()
    for m in (len(z), 8):
        x = torch.zeros(m, 8, dtype=BF16, device="cuda")
        x[:, 0] = z[-m:]
        w = torch.zeros(8, 8, dtype=BF16, device="cuda")
        w[:, 0] = 1
        for act in ACTS:
            y = ops.linear(x, w, activation=act, out=torch.empty(m, 8, dtype=F32, device="cuda"))
            ref, _ = R.act64(x[:, :1].to(R.F64).expand(m, 8), act)
            # (gelu's erfc of what lies below -13 is below fp32's numbers: its value is within 1e-38 of 0)
            R.within(y, ref, ref.abs() * R.ACT + 1e-37, act)
            got = ops.linear_backward(torch.ones(m, 8, dtype=F32, device="cuda"), x, w, pre=x[:, :1].expand(m, 8).contiguous(), activation=act, bias=torch.empty(8, dtype=F32, device="cuda"), w_grad=False,
                                      x_grad=False)
            _, slope = R.act64(x[:, 0].to(R.F64), act)
            assert abs(float(got.bias[0]) - float(slope.sum())) <= float(slope.abs().sum()) * R.ACT + 1e-30
    x = torch.zeros(4, 8, dtype=BF16, device="cuda")
    x[0, 0], x[1, 0], x[2, 0] = float("inf"), float("-inf"), float("nan")
    one = torch.zeros(8, 8, dtype=BF16, device="cuda")
    one[0, 0] = 1
    for act in ACTS:
        y = ops.linear(x[:, :1].contiguous(), one[:1, :1].contiguous(), activation=act).float().flatten()
        assert y[0] == float("inf") and y[2].isnan() and y[3] == 0 and y[1] == (float("-inf") if act is None else 0), act


def test_values_that_are_no_numbers_stay_in_their_rows(ops):
    for m in (10, 300):
        x, w = randn(m, 128, seed=1), weights(96, 128)
        want = ops.linear(x, w)
        x[3, 5], x[m - 1, 0] = float("nan"), float("inf")
        y = ops.linear(x, w)
        assert bool(y[3].isnan().all()) and not bool(y[m - 1].isfinite().any())
        keep = [i for i in range(m) if i not in (3, m - 1)]
        assert torch.equal(y[keep], want[keep])


# ------------------------------------------------------------------------------------------------ gradients
@pytest.mark.parametrize("m", [1, 5, 16, 64, 65, 130, 300, 1000])
@pytest.mark.parametrize("n,k", [(8, 8), (64, 64), (256, 128), (200, 72), (33, 65), (1000, 264), (1, 1), (96, 520)])
def test_gradients(ops, m, n, k):
    x, w, dy, b = randn(m, k, seed=m), weights(n, k), randn(m, n, seed=2), randn(n, seed=3)
    R.check_linear_backward(ops.linear_backward(dy, x, w, bias=b), dy, x, w, bias=b)
    pre, g = randn(m, n, seed=4, gain=2.0), randn(n, dtype=F32, seed=5)
    R.check_linear_backward(ops.linear_backward(dy.float(), x, w, pre=pre, activation="gelu_tanh", gate=g, bias=b), dy.float(), x, w, pre, "gelu_tanh", g, b)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gates", [0, 1, 3])
def test_gradients_of_what_follows(ops, act, dtype, gates):
    m, n, k = 303, 136, 96
    x, w, dy, pre = randn(m, k, seed=1), weights(n, k), randn(m, n, dtype=dtype, seed=2), randn(m, n, seed=3, gain=2.0)
    for vd in (BF16, F32):
        g = None if gates == 0 else randn(n, dtype=vd, seed=4) if gates == 1 else randn(gates, n, dtype=vd, seed=4)
        b = randn(n, dtype=vd, seed=5)
        got = ops.linear_backward(dy, x, w, pre=pre, activation=act, gate=g, bias=b)
        assert got.bias.dtype == vd and (g is None or (got.gate.dtype == vd and got.gate.shape == g.shape))
        R.check_linear_backward(got, dy, x, w, pre, act, g, b)


@pytest.mark.parametrize("B,H,N,d", [(1, 2, 300, 64), (2, 12, 150, 128), (3, 5, 7, 40), (40, 4, 1, 64), (2, 4, 1030, 64), (1, 9, 20, 17)])
def test_gradients_of_heads(ops, B, H, N, d):
    x, w, g = randn(B, H, N, d, seed=N), weights(72, H * d), randn(B, 72, seed=3)
    dy, pre, b = randn(B * N, 72, seed=4), randn(B * N, 72, seed=5), randn(72, seed=6)
    got = ops.linear_backward(dy, x, w, bias=b)
    assert got.x.shape == x.shape
    R.check_linear_backward(got, dy, x, w, bias=b)
    R.check_linear_backward(ops.linear_backward(dy, x, w, pre=pre, activation="silu", gate=g, bias=b), dy, x, w, pre, "silu", g, b)
    # results in heads: their gradient comes so as well
    xr, w2, dh = randn(B * N, 64, seed=7), weights(H * d, 64), randn(B, H, N, d, seed=8)
    R.check_linear_backward(ops.linear_backward(dh, xr, w2, bias=None), dh, xr, w2)
    w3 = weights(H * d, H * d)
    R.check_linear_backward(ops.linear_backward(dh, x, w3), dh, x, w3)
    other = randn(1, H, B * N, d, seed=9)                     # entries that differ from x's
    R.check_linear_backward(ops.linear_backward(other, x, w3), other, x, w3)


@pytest.mark.parametrize("m,k,n", [(4096, 512, 512), (3000, 1536, 1536), (2600, 264, 2048), (128, 256, 4096)])
def test_gradients_of_larger_products(ops, m, k, n):
    x, w, dy, pre, b = randn(m, k, seed=1), weights(n, k), randn(m, n, seed=2), randn(m, n, seed=3), randn(n, seed=4)
    got = ops.linear_backward(dy, x, w, pre=pre, activation="gelu", bias=b)
    R.check_linear_backward(got, dy, x, w, pre, "gelu", None, b)
    again = ops.linear_backward(dy, x, w, pre=pre, activation="gelu", bias=b)
    assert all(torch.equal(a, c) for a, c in zip(got[:3], again[:3]))


def test_gradients_that_are_asked_for(ops):
    m, n, k = 40, 24, 16
    x, w, dy, g = randn(m, k), weights(n, k), randn(m, n, seed=1), randn(n, seed=2)
    got = ops.linear_backward(dy, x, w, gate=g, gate_grad=False, w_grad=False)
    assert got.w is None and got.gate is None and got.bias is None
    R.check_linear_backward(got, dy, x, w, gate=g)
    assert ops.linear_backward(dy, x, w, x_grad=False).x is None


@pytest.mark.parametrize("stride", [200, 193])
def test_gradients_of_strided_operands(ops, stride):
    m, n, k = 150, 120, 184
    x, w, dy = (randn(r, stride, seed=r)[:, 1:1 + c] if stride == 193 else randn(r, stride, seed=r)[:, :c] for r, c in ((m, k), (n, k), (m, n)))
    R.check_linear_backward(ops.linear_backward(dy, x, w, bias=randn(n)), dy, x, w, bias=randn(n))
    pre = randn(m, stride, seed=7)[:, 3:3 + n]
    R.check_linear_backward(ops.linear_backward(dy, x, w, pre=pre, activation="relu"), dy, x, w, pre, "relu")


def test_gradients_against_differences(ops):
    """The forward call's results along a direction of the bias, whose steps are exact in fp32, against the gradient along it."""
    m, n, k = 6, 16, 32
    x, w, dy = randn(m, k, seed=1), weights(n, k), randn(m, n, dtype=F32, seed=2)
    h = 2.0 ** -7
    for act in ("silu", "gelu", "gelu_tanh"):
        b, u = randn(n, seed=3).float(), randn(n, seed=4).float()
        r = torch.zeros(m, n, dtype=F32, device="cuda")
        y = [(ops.linear(x, w, bias=b + s * h * u, activation=act, residual=r).to(R.F64) * dy.to(R.F64)).sum() for s in (1, -1)]
        _, pre = ops.linear(x, w, bias=b, activation=act, residual=r, keep_pre=True)
        got = ops.linear_backward(dy, x, w, pre=pre, activation=act, bias=b)
        along = float((got.bias.to(R.F64) * u.to(R.F64)).sum())
        # pre is 2^-8 off where it is kept: slopes change by up to 1.2 of that and |z| is below 8; third derivatives below 2 over 96 terms of size 4
        size = float((dy.abs() * u.abs()).sum())
        assert abs(float((y[0] - y[1]) / (2 * h)) - along) <= size * (1.2 * 8 * 2.0 ** -8 + 20 * h * h), act


# ------------------------------------------------------------------------------------------------ calls
def test_nothing_to_do(ops):
    x, w, b = randn(0, 64), weights(32, 64), randn(32)
    assert ops.linear(x, w).shape == (0, 32) and ops.linear(randn(5, 64), randn(0, 64)).shape == (5, 0)
    got = ops.linear_backward(randn(0, 32), x, w, bias=b)
    assert got.x.shape == (0, 64) and not bool(got.w.any()) and not bool(got.bias.any())


def test_offsets_past_32_bits(ops):
    """Results, their gradients and weights of 2^32 elements and more: the rows at the end, of which gradients are the only ones that are not 0."""
    m, n, k = (1 << 22) + 130, 1032, 72
    last = slice(m - 130, m)
    x, w, b = randn(m, k), weights(n, k), randn(n, seed=3)
    y, z = ops.linear(x, w, bias=b, activation="silu", keep_pre=True)
    R.check_linear(y[last], x[last], w, b, "silu", pre=z[last])
    del z
    dy = y.zero_()
    dy[last] = randn(130, n, seed=4)
    pre = torch.zeros(m, n, dtype=BF16, device="cuda")
    pre[last] = randn(130, n, seed=5)
    got = ops.linear_backward(dy, x, w, pre=pre, activation="silu", bias=b)
    assert not bool(got.x[:-130].any())
    R.check_linear_backward(ops.LinearGradients(got.x[last], got.w, got.bias, None), dy[last], x[last], w, pre[last], "silu", None, b)
    del x, y, dy, pre, got
    n, k = 1 << 20, 4104
    w = torch.zeros(n, k, dtype=BF16, device="cuda")
    w[-40:] = weights(40, k)
    for rows in (2, 300):
        x = randn(rows, k, seed=rows)
        y = ops.linear(x, w)
        assert not bool(y[:, :-40].any())
        R.check_linear(y[:, -40:], x, w[-40:])


def test_streams_and_graphs(ops):
    """Calls with workspaces on two streams and in two graphs, replayed one after the other."""
    x, w, dy, pre = randn(300, 4096, seed=1), weights(128, 4096), randn(300, 128, seed=2), randn(300, 128, seed=3)
    odd_x, odd_w = randn(100, 77, seed=4), weights(50, 77)
    want, back, odd = ops.linear(x, w, activation="silu"), ops.linear_backward(dy, x, w, pre=pre, activation="silu"), ops.linear(odd_x, odd_w)
    sides = [torch.cuda.Stream() for _ in range(2)]
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    got = [[ops.linear(x, w, activation="silu", stream=s) for s in sides] for _ in range(4)]
    for s in sides:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(y, want) for pair in got for y in pair)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = (ops.linear(x, w, activation="silu"), ops.linear(odd_x, odd_w), *ops.linear_backward(dy, x, w, pre=pre, activation="silu")[:2])
        graphs.append((g, out))
    for _ in range(2):
        for g, _ in graphs:
            g.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, (want, odd, back.x, back.w)))


def test_refusals(ops):
    x, w, b, g, r = randn(6, 64), weights(32, 64), randn(32), randn(2, 32), randn(6, 32)
    dy, pre = randn(6, 32), randn(6, 32)
    bad = [lambda: ops.linear(x.float(), w), lambda: ops.linear(x, w.float()), lambda: ops.linear(x, w[:, :32]), lambda: ops.linear(x.cpu(), w), lambda: ops.linear(x[0], w), lambda: ops.linear(x.t(), w),
           lambda: ops.linear(x, w.reshape(1, 2, 16, 64)), lambda: ops.linear(x, w, bias=b[:31]), lambda: ops.linear(x, w, bias=b.half()), lambda: ops.linear(x, w, gate=randn(4, 32)), lambda: ops.linear(x, w, gate=g[:, :16]),
           lambda: ops.linear(x, w, activation="tanh"), lambda: ops.linear(x, w, residual=r[:5]), lambda: ops.linear(x, w, residual=r.half()), lambda: ops.linear(x, w, out=r[:, :31]), lambda: ops.linear(x, w, out=r.double()),
           lambda: ops.linear(x, w, keep_pre=r.float()), lambda: ops.linear(x, w, keep_pre=r[:5]), lambda: ops.linear(x.requires_grad_(), w), lambda: ops.linear(randn(6, 0), randn(32, 0)),
           lambda: ops.linear_backward(dy[:5], x.detach(), w), lambda: ops.linear_backward(dy, x.detach(), w, activation="silu"), lambda: ops.linear_backward(dy, x.detach(), w, gate=b),
           lambda: ops.linear_backward(dy, x.detach(), w, pre=pre.float()), lambda: ops.linear_backward(dy, x.detach(), w, pre=pre[:, :16]), lambda: ops.linear_backward(dy, x.detach(), w, bias=b[:3])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)
    x = x.detach()
    for f in (lambda: ops.linear(x, w, out=r[:1].expand(6, 32)), lambda: ops.linear(x, w, out=randn(8, 32).as_strided((6, 32), (16, 1)))):
        with pytest.raises(ops.AsError):
            f()
    version = r._version
    ops.linear(x, w, out=r)
    assert r._version > version


def test_refuses_results_over_other_tensors(ops):
    """A result at an input's address, but for the residual's own."""
    x, w, r = randn(32, 32), weights(32, 32), randn(32, 32)
    r4 = randn(2, 4, 4, 32)
    for f in (lambda: ops.linear(x, w, out=x), lambda: ops.linear(x, w, out=w), lambda: ops.linear(x, w, out=r, keep_pre=r), lambda: ops.linear(x, w, keep_pre=x), lambda: ops.linear(x, w, residual=r, keep_pre=r),
              lambda: ops.linear(x, w, residual=r, out=r.view(1, 4, 32, 8)),
              lambda: ops.linear(randn(8, 32), weights(128, 32), residual=r4, out=r4.view(8, 128))):
        with pytest.raises(ops.AsError):
            f()
    want = ops.linear(x, w, residual=r)
    ops.linear(x, w, residual=r, out=r)
    assert torch.equal(r, want)


# what is computed, summed elements, rows of results, columns of results
@pytest.mark.parametrize("what,k,m,n", [("w", 1 << 23, 128, 128), ("w", 1 << 19, 2560, 2048), ("x", 1 << 19, 2560, 2048), ("y", 1 << 19, 2560, 2048)])
def test_long_sums_in_bf16_lean_to_no_side(ops, what, k, m, n):
    """Sums of 8192 steps (and of 16 times as many in 16 parts), all products of one sign.  The matrix instructions truncate what they add up, 2^-23 of it at most, in runs of at most 4 * 342 (256 steps and a
    third more in a first run), and the runs are added up rounded to nearest; a result's rounding to bf16 is at most 2^-8, independent from one to the next, so that the mean of 128 x 128 of them is off by
    less than four times 2^-8 / 3 ** 0.5 / 128.  In one run the sums were off by 3.5e-3 in the mean, always towards 0."""
    if what == "w":                                              # [m, n] = dy [k, m]^T x [k, n]
        dy, x = (randn(k, c, seed=c).abs_() for c in (m, n))
        got = ops.linear_backward(dy, x, weights(m, n), x_grad=k > 1 << 20).w
        a, b = dy[:, :128].T, x[:, :128].T
    elif what == "x":                                            # [m, n] = dy [m, k] w [k, n]
        dy, w = randn(m, k, seed=1).abs_(), randn(k, n, seed=2).abs_()
        got = ops.linear_backward(dy, randn(m, n), w, w_grad=False).x
        a, b = dy[:128], w[:, :128].T
    else:
        x, w = randn(m, k, seed=1).abs_(), randn(n, k, seed=2).abs_()
        got = ops.linear(x, w)
        a, b = x[:128], w[:128]
    ref = sum(a[:, i:i + (1 << 17)].to(R.F64) @ b[:, i:i + (1 << 17)].to(R.F64).T for i in range(0, k, 1 << 17))
    off = float(((got[:128, :128].to(R.F64) - ref) / ref).mean())
    assert abs(off) <= 4 * 342 * 2.0 ** -23 + 4 * 2.0 ** -8 / 3 ** 0.5 / 128, off


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N", [48, 80, 104])
def test_residuals_in_heads_that_tiles_cross(ops, N, dtype):
    """Entries of tokens that 32 does not divide: a warp's rows come and go by copies where they are of one entry, by its own loads and stores where they are of two, from tile to tile by turns."""
    B, H, d, k = 9600 // N, 12, 128, 64
    x, w, r = randn(B * N, k, seed=1), weights(H * d, k), randn(B, H, N, d, dtype=dtype, seed=2)
    want = r.clone()
    y = ops.linear(x, w, residual=r)
    R.check_linear(y, x, w, None, None, None, r)
    for _ in range(5):
        r.copy_(want)
        assert torch.equal(ops.linear(x, w, residual=r, out=r), y)
