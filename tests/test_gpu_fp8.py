"""The 8-bit projections on a GPU against their formulas in 64 bits: rows, widths and tiles where they can go wrong, layouts, strides and alignments, values that are no
numbers, streams, graphs, and the layer that runs them together."""
import pytest
import torch

from tests import _fp8 as R
from tests._util import Guarded

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# t * w and its product with the row's scale are rounded to fp32 each, the sum of squares in some order: cols <= 16384 positive values, each rounding 2^-24
SLACK = 2.0 ** -17


@pytest.fixture(scope="module", autouse=True)
def ops():
    import paper_2509_24899_b200 as pkg
    yield pkg
    torch.cuda.synchronize()
    assert pkg.fp8_last_status() == 0


def randn(*shape, dtype=BF16, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * gain).to(dtype)


def close_bf16(y, ref, slack=SLACK):
    """Half a spacing of bf16 and the slack."""
    off = (y.to(R.F64) - ref).abs()
    assert bool((off <= ref.abs() * (2.0 ** -8 + slack) + 1e-38).all()), float((off / ref.abs().clamp(min=1e-30)).max())


# ------------------------------------------------------------------------------------------------ norm
WIDTHS = [1, 2, 8, 15, 16, 24, 64, 127, 128, 129, 136, 256, 264, 511, 512, 520, 1000, 1024, 1160, 1536, 1544, 2048, 2049, 3080, 4104, 6144, 8200, 12288, 12296, 16384]


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("x,residual", [(BF16, None), (BF16, BF16), (BF16, F32), (F32, None), (F32, F32)])
def test_norm_widths(ops, cols, x, residual):
    for rows, fp8, wd in ((1, True, BF16), (9, False, F32), (37, True, F32), (5, False, BF16), (3, True, None)):
        xv, w = randn(rows, cols, dtype=x, seed=cols), None if wd is None else (1 + 0.3 * randn(cols, dtype=F32, seed=3)).to(wd)
        r = None if residual is None else randn(rows, cols, dtype=residual, seed=7, gain=3.0)
        got = ops.rms_norm(xv, w, residual=r, eps=1e-5, fp8=fp8)
        y, t = R.norm64(xv, w, r, 1e-5)
        if r is not None:
            got, total = got
            # the sum in fp32, rounded once
            assert torch.equal(total, (xv.float() + r.float()).to(residual))
        if fp8:
            R.check_form(got, y, slack=SLACK)
        else:
            assert got.shape == xv.shape and got.dtype == BF16
            close_bf16(got, y)


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 295, 296, 297, 2368, 2369, 5000])
@pytest.mark.parametrize("cols", [64, 200, 256, 1536, 1537])
def test_norm_rows(ops, rows, cols):
    """CTAs that go on from row to row: one row, all of a turn's, one more, several turns."""
    x, w = randn(rows, cols, seed=rows), randn(cols, seed=1)
    y, _ = R.norm64(x, w)
    R.check_form(ops.rms_norm(x, w, fp8=True), y, slack=SLACK)
    close_bf16(ops.rms_norm(x, w), y)


@pytest.mark.parametrize("B,H,N,d", [(1, 2, 33, 64), (2, 12, 50, 128), (3, 5, 7, 40), (2, 3, 31, 8), (1, 9, 20, 4), (2, 4, 9, 17)])
def test_norm_between_layouts(ops, B, H, N, d):
    """Rows to heads, heads to rows, heads to 8 bits, with rows that lie in a wider matrix."""
    wide = randn(B * N, 3 * H * d, seed=2)
    w = randn(H * d, seed=5)
    for part in range(3):
        x = wide[:, part * H * d:(part + 1) * H * d]
        y, _ = R.norm64(x, w)
        out = torch.full((B, H, N, d), 7.0, dtype=BF16, device="cuda")
        assert ops.rms_norm(x, w, out=out) is out
        close_bf16(R.rows_of(out), y)
        back = torch.empty(B * N, H * d, dtype=BF16, device="cuda")
        y2, _ = R.norm64(out, w)
        ops.rms_norm(out, w, out=back)
        close_bf16(back, y2)
        R.check_form(ops.rms_norm(out, w, fp8=True), y2, slack=SLACK)
        R.check_form(ops.quantize_fp8(out), R.rows_of(out).to(R.F64))
    # heads that lie in rows: [B, N, H, d] seen as [B, H, N, d]
    seen = wide[:, :H * d].reshape(B, N, H, d).permute(0, 2, 1, 3)
    R.check_form(ops.rms_norm(seen, w, fp8=True), R.norm64(seen, w)[0], slack=SLACK)


@pytest.mark.parametrize("shift", [0, 1, 2, 4, 8, 16])
@pytest.mark.parametrize("stride", [1536, 1537, 1544, 1552, 0])
def test_norm_alignment_and_strides(ops, shift, stride):
    """Addresses and strides that allow 32, 16 and 2 bytes an access; all rows the same one."""
    rows, cols = 12, 1536
    flat = randn(40000, seed=11)
    x = flat[shift:].as_strided((rows, cols), (stride, 1), flat.storage_offset() + shift)
    w = randn(cols + 32, seed=4)[shift:shift + cols]
    y, _ = R.norm64(x, w)
    R.check_form(ops.rms_norm(x, w, fp8=True), y, slack=SLACK)
    close_bf16(ops.rms_norm(x, w), y)
    R.check_form(ops.quantize_fp8(x), x.to(R.F64))
    R.check_form(ops.quantize_fp8(x, block_rows=128), x.to(R.F64), block_rows=128)


def test_residual_in_place_and_given_outputs(ops):
    x, r, w = randn(20, 1536, seed=1), randn(20, 1536, dtype=F32, seed=2), randn(1536, seed=3)
    y, _ = R.norm64(x, w, r)
    want = x.float() + r
    out = ops.empty_fp8(20, 1536)
    got, total = ops.rms_norm(x, w, residual=r, fp8=True, out=out, residual_out=r)
    assert got is out and total is r and torch.equal(r, want)
    R.check_form(out, y, slack=SLACK)


def test_norm_of_special_rows(ops):
    """Rows of zeros, of one value, of huge and tiny ones; with infinity and NaN, whose rows alone are no numbers."""
    cols = 400
    x = randn(9, cols, seed=8)
    x[1] = 0
    x[2] = 1e-20
    x[3] = 3e18
    x[4, 5] = float("inf")
    x[5, 390] = float("nan")
    x[6, :128] = 0
    ok = [0, 1, 2, 3, 6, 7, 8]
    for fp8 in (False, True):
        got = ops.rms_norm(x, None, eps=1e-6, fp8=fp8)
        y, _ = R.norm64(x[ok], None)
        if fp8:
            R.check_form((got.data[ok], got.scales[:, ok].contiguous()), y, slack=SLACK)
            v = R.value64(got)
        else:
            close_bf16(got[ok], y)
            v = got.to(R.F64)
        assert bool(v[5].isnan().all()) and bool(v[4, 5].isnan())
    q = ops.quantize_fp8(x)
    e, _ = R.table(q.scales, cols)
    assert e[4].tolist()[0] == 255 and e[5].tolist()[3] == 255 and bool((e[4, 1:] < 255).all()) and bool((e[5, :3] < 255).all())
    assert e[1].tolist() == [0] * 4 and e[6, 0] == 0 and bool((q.data[1].float() == 0).all())
    # eps 0: a row of zeros is 0 / 0, as in the formula
    assert bool(ops.rms_norm(x[1:2], None, eps=0.0)[0].isnan().all())


@pytest.mark.parametrize("cols", [100, 200, 1536, 2049, 5000])
@pytest.mark.parametrize("x,residual", [(BF16, None), (BF16, BF16), (BF16, F32), (F32, None)])
def test_norm_of_rows_whose_squares_fp32_does_not_hold(ops, cols, x, residual):
    """Beside ordinary rows.  With a residual in bf16 the mean is that of t as it was rounded: 2^-8 more."""
    xv, w = randn(11, cols, dtype=x, seed=1), randn(cols, seed=2)
    r = None if residual is None else randn(11, cols, dtype=residual, seed=3)
    for i, gain in ((2, 1e19), (3, 1e25), (9, 1e35)):
        xv[i] *= gain
    y, _ = R.norm64(xv, w, r)
    slack = SLACK + (2.0 ** -8 if residual is BF16 else 0.0)
    got = ops.rms_norm(xv, w, residual=r)
    close_bf16(got if r is None else got[0], y, slack)
    got = ops.rms_norm(xv, w, residual=r, fp8=True)
    R.check_form(got if r is None else got[0], y, slack=slack)


def test_scales_at_their_bounds(ops):
    """Blocks whose largest value is 448 * 2^e, the next number above, and the smallest and largest that bf16 has."""
    x = torch.zeros(8, 256, dtype=BF16, device="cuda")
    for i, v in enumerate((448.0, 450.0, 1.75 * 2.0 ** -30, 1.765625 * 2.0 ** -30, 2.0 ** -126, 3.3895e38, 2.0 ** -118, 1.0)):
        x[i, 3], x[i, 200] = v, -v
    for block_rows in (1, 128):
        R.check_form(ops.quantize_fp8(x, block_rows=block_rows), x.to(R.F64), block_rows=block_rows)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (127, 129), (128, 512), (129, 513), (300, 1160), (257, 1544), (1000, 72)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weights_to_8_bits(ops, rows, cols, dtype):
    x = randn(rows, cols, dtype=dtype, seed=rows, gain=0.03)
    R.check_form(ops.quantize_fp8(x, block_rows=128), x.to(R.F64), block_rows=128)
    R.check_form(ops.quantize_fp8(x), x.to(R.F64))


# ------------------------------------------------------------------------------------------------ product
def operands(M, N, K, seed=0):
    a = R.pair_of(randn(M, K, dtype=R.F64, seed=seed))
    return a, R.pair_of(randn(N, K, dtype=R.F64, seed=seed + 1, gain=0.05), 128), randn(N, seed=seed + 2)


SHAPES = [(1, 1, 1), (1, 16, 16), (1, 15, 128), (2, 9216, 129), (3, 17, 1001), (7, 40, 2048), (8, 1000, 1536), (8, 33, 6145), (5, 5000, 15), (4, 31, 127),
          (9, 16, 128), (9, 1, 1), (31, 77, 130), (33, 1536, 512), (127, 224, 640), (128, 225, 513), (129, 192, 1024), (255, 193, 17), (256, 256, 256), (257, 31, 999),
          (500, 1000, 1160), (1000, 64, 4096), (1001, 4608, 128), (2047, 1536, 384), (2300, 1337, 700), (4096, 160, 256), (7800, 1536, 512), (20011, 448, 257),
          (300, 20000, 192), (12345, 96, 64), (640, 640, 16384),
          (16, 5000, 1536), (17, 1000, 2000), (24, 15, 6145), (40, 512, 1280), (64, 130, 2392), (100, 17, 130), (256, 128, 2392), (256, 64, 100), (15, 3000, 4100),
          (128, 1536, 6144), (300, 512, 4096), (512, 1536, 6144), (129, 321, 6145), (77, 3000, 8200), (200, 1, 16384), (1000, 200, 5121), (640, 40, 3585)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_matmul_shapes(ops, M, N, K):
    a, w, bias = operands(M, N, K)
    R.check_matmul(ops.matmul_fp8(a, w), a, w)
    R.check_matmul(ops.matmul_fp8(a, w, bias=bias), a, w, bias)


@pytest.mark.parametrize("M,K", [(2, 300), (40, 300), (700, 300), (260, 4200)])
@pytest.mark.parametrize("B,H,d", [(2, 3, 64), (2, 4, 128), (1, 5, 32), (2, 6, 16), (2, 3, 40), (1, 7, 9), (2, 2, 8)])
def test_matmul_into_heads(ops, M, K, B, H, d):
    """Strips that TMA takes, that cross into the next batch entry, that warps store 16 bytes or an element at a time; nothing else is written."""
    a, w, bias = operands(M, H * d, K, seed=M)
    box = Guarded(M * H * d * 2)
    out = box.view(BF16, (B, H, M // B, d))
    assert ops.matmul_fp8(a, w, bias=bias, out=out) is out
    R.check_matmul(out, a, w, bias)
    box.check("heads")
    # heads that lie in rows, with other columns between the rows
    wide = torch.full((M, H * d + 24), 3.0, dtype=BF16, device="cuda")
    seen = wide.as_strided((B, H, M // B, d), (M // B * (H * d + 24), d, H * d + 24, 1), 16)
    ops.matmul_fp8(a, w, bias=bias, out=seen)
    R.check_matmul(seen, a, w, bias)
    assert bool((wide[:, :16] == 3).all()) and bool((wide[:, 16 + H * d:] == 3).all())


@pytest.mark.parametrize("M,N", [(3, 40), (64, 100), (300, 1000), (513, 512)])
@pytest.mark.parametrize("shift,extra", [(0, 0), (0, 8), (8, 8), (1, 3), (0, 1), (4, 4)])
def test_matmul_row_strides(ops, M, N, shift, extra):
    a, w, _ = operands(M, N, 200, seed=N)
    wide = torch.full((M, shift + N + extra), 5.0, dtype=BF16, device="cuda")
    out = wide[:, shift:shift + N]
    ops.matmul_fp8(a, w, out=out)
    R.check_matmul(out, a, w)
    assert bool((wide[:, :shift] == 5).all()) and bool((wide[:, shift + N:] == 5).all())


@pytest.mark.parametrize("M", [4, 200])
def test_matmul_of_parts_of_matrices(ops, M):
    """Rows out of the middle of larger pairs, and a pitch wider than the columns, whose bytes are not looked at."""
    a, w, _ = operands(M + 40, 300, 270)
    for pair in (a, w):
        base = pair[0].as_strided((pair[0].shape[0], pair[0].stride(0)), (pair[0].stride(0), 1))
        base[:, pair[0].shape[1]:] = float("nan")
    a1 = (a[0][16:16 + M], a[1][:, 16:16 + M])
    w1 = (w[0][128:300], w[1][:, 128:300])
    R.check_matmul(ops.matmul_fp8(a1, w1), a1, w1)


@pytest.mark.parametrize("M", [3, 150])
def test_matmul_of_scales_at_their_bounds(ops, M):
    """Scales far apart from block to block and row to row; one that is NaN takes its row or column with it and nothing else."""
    K, N = 1100, 140
    a, w, _ = operands(M, N, K, seed=5)
    g = torch.Generator(device="cuda").manual_seed(9)
    for pair in (a, w):
        e = torch.randint(100, 155, pair[1].shape, generator=g, device="cuda")
        pair[1].copy_(e.to(torch.uint8))
    R.check_matmul(ops.matmul_fp8(a, w), a, w)
    a[1][1, 2, 3] = 255
    w[1][2, 77, 0] = 255
    out = ops.matmul_fp8(a, w)
    nan = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    nan[2], nan[:, 77] = True, True
    assert torch.equal(out.isnan(), nan)
    a[1][1, 2, 3], w[1][2, 77, 0] = 0, 0                                       # 2^-127: as good as nothing
    R.check_matmul(ops.matmul_fp8(a, w), a, w)


@pytest.mark.parametrize("M", [3, 150])
def test_matmul_of_values_that_are_no_numbers(ops, M):
    a, w, _ = operands(M, 50, 300)
    a[0][1, 299] = float("nan")
    out = ops.matmul_fp8(a, w)
    assert bool(out[1].isnan().all()) and not bool(out[[0, 2]].isnan().any())


def test_offsets_past_31_bits(ops):
    """Rows that lie 2^30 elements apart."""
    apart = 1 << 30
    flat = torch.empty(2 * apart + 4096, dtype=BF16, device="cuda")
    x = flat.as_strided((3, 512), (apart, 1))
    x.copy_(randn(3, 512, seed=1))
    y, _ = R.norm64(x, None)
    R.check_form(ops.rms_norm(x, fp8=True), y, slack=SLACK)
    a, w, _ = operands(3, 512, 512)
    out = flat.as_strided((3, 512), (apart, 1), 1024)
    ops.matmul_fp8(a, w, out=out)
    R.check_matmul(out, a, w)
    a, w, _ = operands(200, 512, 512)
    out = flat.as_strided((100, 512), (apart // 64, 1)).as_strided((100, 512), (apart // 64, 1), 2048)
    ops.matmul_fp8((a[0][:100], a[1][:, :100]), w, out=out)
    R.check_matmul(out, (a[0][:100], a[1][:, :100]), w)
    ops.rms_norm(out, out=out)
    del flat


def test_no_rows(ops):
    a = ops.empty_fp8(0, 256)
    w = ops.quantize_fp8(randn(64, 256), block_rows=128)
    assert ops.matmul_fp8(a, w).shape == (0, 64)
    assert ops.rms_norm(torch.empty(0, 256, dtype=BF16, device="cuda"), fp8=True).data.shape == (0, 256)
    assert ops.quantize_fp8(torch.empty(1, 2, 0, 64, dtype=BF16, device="cuda")).data.shape == (0, 128)


# ------------------------------------------------------------------------------------------------ calls
def test_same_bits_every_time(ops):
    for M, N, K in ((2, 1000, 1536), (40, 200, 1000), (300, 512, 4096), (700, 1000, 1536), (5000, 1536, 512)):
        a, w, bias = operands(M, N, K)
        first = ops.matmul_fp8(a, w, bias=bias)
        for _ in range(3):
            assert torch.equal(first, ops.matmul_fp8(a, w, bias=bias))


def test_streams_and_graphs(ops):
    """A chain of dependent calls on another stream, then captured and replayed on new inputs."""
    x, w8 = randn(300, 1536, seed=1), ops.quantize_fp8(randn(256, 1536, seed=2, gain=0.05), block_rows=128)
    y = torch.empty(300, 256, dtype=BF16, device="cuda")
    x8, z8 = ops.empty_fp8(300, 1536), ops.empty_fp8(300, 256)

    def chain():
        ops.rms_norm(x, fp8=True, out=x8)
        ops.matmul_fp8(x8, w8, out=y)
        ops.quantize_fp8(y, out=z8)

    def check():
        R.check_form(x8, R.norm64(x)[0], slack=SLACK)
        R.check_matmul(y, x8, w8)
        R.check_form(z8, y.to(R.F64))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(5):
            chain()
    side.synchronize()
    check()
    ops.rms_norm(x, fp8=True, out=x8, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for seed in (3, 4):
        x.copy_(randn(300, 1536, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        check()


def test_python_refusals(ops):
    x, w = randn(4, 256), ops.quantize_fp8(randn(64, 256), block_rows=128)
    a = ops.quantize_fp8(x)
    bad = [lambda: ops.rms_norm(x.cpu()), lambda: ops.rms_norm(x.half()), lambda: ops.rms_norm(x[:, ::2]), lambda: ops.rms_norm(x[0]),
           lambda: ops.rms_norm(x, weight=randn(255)), lambda: ops.rms_norm(x, residual=randn(4, 255)), lambda: ops.rms_norm(x, residual_out=x),
           lambda: ops.rms_norm(x, out=randn(4, 255)), lambda: ops.rms_norm(x, fp8=True, out=ops.empty_fp8(4, 255)), lambda: ops.quantize_fp8(x, out=ops.empty_fp8(5, 256)),
           lambda: ops.matmul_fp8(a, ops.quantize_fp8(randn(64, 255))), lambda: ops.matmul_fp8(a, w, bias=randn(63)), lambda: ops.matmul_fp8(a, w, bias=randn(64, dtype=F32)),
           lambda: ops.matmul_fp8(a, w, out=randn(4, 64, dtype=F32)), lambda: ops.matmul_fp8(a, w, out=randn(4, 63)),
           lambda: ops.matmul_fp8((a[0], a[1][:, :3]), w), lambda: ops.matmul_fp8((x, a[1]), w), lambda: ops.matmul_fp8((a[0], a[1].to(torch.int32)), w)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ops.quantize_fp8(x, block_rows=3), lambda: ops.matmul_fp8(a, w, out=torch.empty(64, dtype=BF16, device="cuda").expand(4, 64)),
              lambda: ops.rms_norm(x, eps=-1.0), lambda: ops.rms_norm(randn(1, 16385)), lambda: ops.rms_norm(randn(4, 256, dtype=F32), residual=x)):
        with pytest.raises(ops.AsError):
            f()


def test_layer(ops):
    """The attention half of a layer: norm, three products into heads, hybrid attention, 8-bit form, output projection, against the oracle in 64 bits on the weights as they
    were given.  Each 8-bit operand is up to 2^-4 off (2.6 % in the root mean square of its values); q, k and o see two of them, so 2 x 2.6 % x sqrt(2) = 7.4 %
    of the output's root mean square bounds the relative error of a layer whose attention does not amplify them; with the hybrid attention's own 0.5 % the test asks for 10 %."""
    from oracle import hybrid_attention as O
    from paper_2509_24899_b200 import HybridAttention, workloads as W
    from paper_2509_24899_b200.fp8_layer import Fp8AttentionLayer
    wl = W.CONFIGS["tiny"]
    B, H, N, d = wl.B, wl.H, wl.N, wl.d
    D = H * d
    data = W.generate(wl, wq_gain=2e-3)
    phi = {n: torch.from_numpy(data[n].view("int16")).cuda().view(BF16) for n in ("wq", "wk")}
    weights = {n: randn(D, D, seed=i, gain=D ** -0.5) for i, n in enumerate("qkvo")}
    weights |= {"bias_" + n: randn(D, seed=10 + i, gain=0.1) for i, n in enumerate("qkvo")}
    weights |= {n: (1 + 0.1 * randn(D, dtype=F32, seed=20)).to(BF16) for n in ("norm", "norm_q", "norm_k")}
    hidden, residual = randn(B * N, D, seed=30), randn(B * N, D, dtype=F32, seed=31)
    layer = Fp8AttentionLayer(HybridAttention.from_workload(wl), weights, phi)
    y, total = layer.forward(hidden, residual)
    assert torch.equal(total, hidden.float() + residual)

    w64 = {n: w.to(R.F64) for n, w in weights.items()}
    x = R.norm64(hidden, weights["norm"], residual)[0]
    q, k, v = (x @ w64[n].T + w64["bias_" + n] for n in "qkv")
    q, k = (t / torch.sqrt(t.square().mean(1, keepdim=True) + 1e-6) * w64[n] for t, n in ((q, "norm_q"), (k, "norm_k")))
    o, _ = O.hybrid_attention(*(R.heads_of(t, B, d).contiguous().cpu().numpy() for t in (q, k, v)), *(p.double().cpu().numpy() for p in phi.values()),
                              O.softmax_token_mask(wl.grid, wl.block, wl.rate))
    ref = R.rows_of(torch.from_numpy(o).cuda()) @ w64["o"].T + w64["bias_o"]
    rel = float((y.to(R.F64) - ref).norm() / ref.norm())
    assert rel <= 0.10, rel
    with pytest.raises(ValueError):
        Fp8AttentionLayer(layer.attention, dict(weights, q=weights["q"][:, :-8]), phi)
