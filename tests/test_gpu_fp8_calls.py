"""What the calls of the 8-bit projections take and keep: pairs, gradients, status and errors."""
import pytest
import torch

from tests import _fp8 as R

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def ops():
    import paper_2509_24899_b200 as pkg
    yield pkg
    torch.cuda.synchronize()
    assert pkg.fp8_last_status() == 0


def randn(*shape, dtype=BF16, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * gain).to(dtype)


# ------------------------------------------------------------------------------------------------ pairs
@pytest.mark.parametrize("M", [3, 300])
def test_pairs_whose_tensors_nothing_else_holds(ops, M):
    """The call holds a pair's tensors until its work is on the stream, also where the pair is an iterator that has let go of them and the output could take their place."""
    a, w = ops.quantize_fp8(randn(M, 512, seed=1)), ops.quantize_fp8(randn(M, 512, seed=2))
    want = ops.matmul_fp8(a, w)
    for made in (lambda p: (t.clone(memory_format=torch.preserve_format) for t in p), lambda p: map(torch.Tensor.view_as, p, p), lambda p: [t.clone() for t in p], iter):
        for _ in range(8):
            assert torch.equal(ops.matmul_fp8(made(a), made(w)), want)


def test_what_is_no_pair_is_refused(ops):
    a = ops.quantize_fp8(randn(2, 512))
    for bad in (a[0], a[1], (a[0],), (*a, a[0]), (t[:, :4] for t in a), {a[0]: a[1]}, (a[0], None)):
        with pytest.raises(ValueError):
            ops.matmul_fp8(bad, a)
    for bad in (None, 3):
        with pytest.raises(TypeError):
            ops.matmul_fp8(bad, a)
