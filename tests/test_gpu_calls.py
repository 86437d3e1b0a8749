"""What the calls that take PyTorch tensors refuse of every tensor, whichever call it is given to."""
import pytest
import torch
import torch.autograd.forward_ad as fwad

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ops():
    import paper_2509_24899_b200 as pkg
    return pkg


def randn(*shape, dtype=BF16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def calls(ops):
    """(name, a call of one tensor, that tensor)"""
    x, w, q = randn(6, 64), randn(32, 64, seed=1), randn(1, 2, 5, 64, seed=2)
    table = ops.rotary_table((5,), (32,))
    w8 = ops.quantize_fp8(w, block_rows=128)
    return [("x", lambda t: ops.linear(t, w), x), ("w", lambda t: ops.linear(x, t), w), ("bias", lambda t: ops.linear(x, w, bias=t), randn(32)), ("gate", lambda t: ops.linear(x, w, gate=t), randn(32, dtype=F32)),
            ("residual", lambda t: ops.linear(x, w, residual=t), randn(6, 32)), ("dy", lambda t: ops.linear_backward(t, x, w), randn(6, 32)),
            ("rotated", lambda t: ops.rotary(t, table), q), ("factors", lambda t: ops.rotary(q, (t, (5,), (32,))), table.factors), ("normed", lambda t: ops.qk_norm_rotary(t, None, table=table), q),
            ("norm's weight", lambda t: ops.qk_norm_rotary(q, None, t, None, table), randn(64)), ("dq", lambda t: ops.qk_norm_rotary_backward(t, None, q, None, table=table), q),
            ("rms_norm", lambda t: ops.rms_norm(t), x), ("quantize_fp8", lambda t: ops.quantize_fp8(t), x), ("matmul_fp8", lambda t: ops.matmul_fp8(ops.quantize_fp8(x), w8, bias=t), randn(32))]


def test_tensors_with_a_forward_mode_tangent_are_refused(ops):
    """Their results would carry none; a program that wants the value alone takes the primal, or turns forward mode off."""
    with fwad.dual_level():
        for name, call, t in calls(ops):
            dual = fwad.make_dual(t, torch.ones_like(t))
            with pytest.raises(ValueError, match="tangent"):
                call(dual)
                print("not refused:", name)
            call(fwad.unpack_dual(dual).primal)
            with fwad._set_fwd_grad_enabled(False):
                call(dual)
        x, w, out = randn(6, 64), randn(32, 64), fwad.make_dual(randn(6, 32), randn(6, 32))
        with pytest.raises(ValueError, match="tangent"):
            ops.linear(x, w, out=out)


def test_views_whose_values_count_negated_are_refused(ops):
    """(The imaginary part of a conjugate is one: what lies in memory has the other sign.)"""
    column = torch.complex(randn(5, 1, dtype=F32), randn(5, 1, dtype=F32)).conj().imag
    assert column.is_neg()
    with pytest.raises(ValueError, match="negated"):
        ops.rms_norm(column)
    for name, call, t in calls(ops):
        with pytest.raises(ValueError, match="negated"):
            call(torch._neg_view(t))
            print("not refused:", name)
        call(torch._neg_view(t).resolve_neg())
