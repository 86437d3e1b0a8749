"""The 8-bit projections at the ends of fp32's range, against their formulas in 64 bits."""
import pytest
import torch

from tests import _fp8 as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# The sum of squares: at most 64 values a lane one after another, 5 steps between lanes, 8 warps, each a rounding of 2^-24 of the sum, so half of 77 of them for its root; two
# ulp (2^-22) for rsqrt; three products of 2^-24; a factor below fp32's normal numbers has 22 bits (2^-22).  In all below 2^-18; twice that.
SLACK = 2.0 ** -17
KINDS = [(BF16, None), (BF16, BF16), (BF16, F32), (F32, None), (F32, F32)]
WIDTHS = [100, 128, 200, 256, 1536, 1537, 2049, 5000, 16384]


@pytest.fixture(scope="module", autouse=True)
def ops():
    import paper_2509_24899_b200 as pkg
    yield pkg
    torch.cuda.synchronize()
    assert pkg.fp8_last_status() == 0


def randn(*shape, dtype=BF16, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * gain).to(dtype)


def close_bf16(y, ref):
    """Half a spacing of bf16 (2^-8 relative; 2^-134 below its normal numbers) and the slack, which is as much of fp32's smallest normal number."""
    off = (y.to(R.F64) - ref).abs()
    assert bool((off <= ref.abs() * (2.0 ** -8 + SLACK) + 2.0 ** -134).all()), float((off / ref.abs().clamp(min=1e-38)).max())


def check_norm(ops, x, w, r, eps=1e-6):
    """Both forms of the output, and the residual."""
    y, t = R.norm64(x, w, r, eps)
    assert bool(t.isfinite().all()) and bool(y.isfinite().all())
    got = ops.rms_norm(x, w, residual=r, eps=eps)
    close_bf16(R.rows_of(got if r is None else got[0]), y)
    if r is not None:
        assert torch.equal(got[1], (x.float() + r.float()).to(r.dtype))
    got = ops.rms_norm(x, w, residual=r, eps=eps, fp8=True)
    R.check_form(got if r is None else got[0], y, slack=SLACK)


def rows_with(cols, x, residual, gains, rows=13):
    """x (and a residual): ordinary rows, and from row 2 on every second one times one of the gains."""
    xv = randn(rows, cols, dtype=F32, seed=cols).clamp(-4, 4)
    rv = None if residual is None else randn(rows, cols, dtype=F32, seed=cols + 1).clamp(-4, 4)
    for i, gain in enumerate(gains):
        xv[2 + 2 * i] *= gain
        if rv is not None:
            rv[2 + 2 * i] *= gain
    return xv.to(x), rv if rv is None else rv.to(residual)


# ------------------------------------------------------------------------------------------------ large values
@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("x,residual", KINDS)
def test_norm_of_rows_up_to_the_largest_numbers(ops, cols, x, residual):
    """Rows whose largest values are near fp32's largest (4 + 4 times 4e37 of 3.4e38), without weights and with ones up to 1."""
    xv, r = rows_with(cols, x, residual, (1e19, 1e30, 1e36, 1e37, 4e37))
    check_norm(ops, xv, None, r)
    check_norm(ops, xv, torch.linspace(-1, 1, cols, device="cuda").to(BF16), r)
    # every value the same, the largest that the type has
    top = torch.full((3, cols), torch.finfo(x).max, dtype=x, device="cuda")
    check_norm(ops, top, None, None)


@pytest.mark.parametrize("cols", [100, 200, 1536, 1537, 5000])
@pytest.mark.parametrize("x,residual", KINDS)
def test_norm_goes_by_the_sum_as_it_was_added(ops, cols, x, residual):
    """Rows whose squares fp32 does not hold: their mean is that of the unrounded sum for every type of the residual, as in ordinary rows."""
    xv, r = rows_with(cols, x, residual, (1e19, 3e19, 1e25, 1e30, 1e35))
    check_norm(ops, xv, randn(cols, seed=2).clamp(-1, 1), r)


# ------------------------------------------------------------------------------------------------ weights
@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("x,residual", KINDS)
@pytest.mark.parametrize("wd", [BF16, F32])
def test_norm_with_large_and_small_weights(ops, cols, x, residual, wd):
    """Values times weights that lie beyond fp32's range on either side, and normed values times weights that do not."""
    xv, r = rows_with(cols, x, residual, (1e10, 1e19, 1e30, 1e36, 4e37))
    w = torch.exp(torch.linspace(-30, 30, cols, device="cuda")).to(wd)
    check_norm(ops, xv, w, r)
    check_norm(ops, xv, w.flip(0) * 1e20, r)
    xv, r = rows_with(cols, x, residual, (1e-4, 1e-6, 1e-8, 1e-10, 1e-12))
    check_norm(ops, xv, w * 1e-24, r, eps=1e-12)


# ------------------------------------------------------------------------------------------------ small values
@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("x,residual", KINDS)
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-30, 1e-20])
def test_norm_of_rows_whose_squares_are_too_small(ops, cols, x, residual, eps):
    """Rows whose squares vanish in fp32 with an eps that does as well, or nearly."""
    xv, r = rows_with(cols, x, residual, (1e-12, 1e-16, 1e-20, 1e-26, 1e-33))
    check_norm(ops, xv, None, r, eps=eps)
    check_norm(ops, xv, randn(cols, seed=2), r, eps=eps)
    # every value the same, the smallest that the type has
    check_norm(ops, torch.full((3, cols), torch.finfo(x).smallest_normal * torch.finfo(x).eps, dtype=x, device="cuda"), None, None, eps=eps)


# ------------------------------------------------------------------------------------------------ scales of a product
@pytest.mark.parametrize("M", [3, 11, 150, 700])
@pytest.mark.parametrize("ea,ew", [((0, 40), (214, 254)), ((214, 254), (0, 40)), ((0, 3), (252, 254)), ((127, 254), (0, 127)), ((230, 250), (4, 24)), ((0, 10), (120, 254)),
                                   ((67, 127), (67, 127))])
def test_matmul_of_opposed_scales(ops, M, ea, ew):
    """Scales each of which takes a block's sum beyond fp32's range, on either side, while both together do not."""
    K, N = 1100, 140
    a, w = R.pair_of(randn(M, K, dtype=R.F64, seed=5)), R.pair_of(randn(N, K, dtype=R.F64, seed=6), 128)
    g = torch.Generator(device="cuda").manual_seed(9)
    for pair, (lo, hi) in ((a, ea), (w, ew)):
        pair[1].copy_(torch.randint(lo, hi + 1, pair[1].shape, generator=g, device="cuda").to(torch.uint8))
    # no sum may pass bf16's largest number: block by block, e_a + e_w of at most 254 + 100
    e = torch.minimum(a[1].amax(1, keepdim=True).to(torch.int64) + w[1].amax(1, keepdim=True).to(torch.int64), torch.full((), 354, device="cuda"))
    for pair, other in ((a, w), (w, a)):
        pair[1].copy_(torch.minimum(pair[1].to(torch.int64), e - other[1].amax(1, keepdim=True).to(torch.int64)).to(torch.uint8))
    av, wv = R.value64(a), R.value64(w)
    ref, size = av @ wv.T, av.abs() @ wv.abs().T
    # as check_matmul, and half a spacing of bf16 and of fp32 for each block below their normal numbers
    tol = ref.abs() * 2.0 ** -8 + size * 2.0 ** -23 * 2 * (K / 32 + 2) + 2.0 ** -134 + 9 * 2.0 ** -149
    assert float(size.max()) < 3e38
    off = (ops.matmul_fp8(a, w).to(R.F64) - ref).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
