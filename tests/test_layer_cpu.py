"""The bf16 steps around the attention without a GPU: the plain forms against values worked by hand, and the refusals of the C entries, which come before any CUDA call."""
import ctypes as C
import math
import os
import re

import pytest
import torch

from paper_2509_24899_b200 import binding, build
from tests import _layer as R

INVALID, UNSUPPORTED = binding.AS_ERR_INVALID_ARG, binding.AS_ERR_UNSUPPORTED
P = 1 << 20                                                     # an address that nothing is read from


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


# ------------------------------------------------------------------------------------------------ plain forms
def test_rotation_by_hand():
    # two positions of one axis, two pairs of angles 1 and 1/100 a position
    table = R.table64((3,), (2,))
    assert torch.allclose(table[2, :, 0], torch.tensor([math.cos(2.0), math.cos(0.02)], dtype=R.F64)) and torch.allclose(table[1, :, 1], torch.tensor([math.sin(1.0), math.sin(0.01)], dtype=R.F64))
    x = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0], dtype=R.F64).reshape(1, 1, 1, 5)
    cs = (torch.tensor([0.0, 1.0], dtype=R.F64).reshape(1, 1, 1, 2), torch.tensor([1.0, 0.0], dtype=R.F64).reshape(1, 1, 1, 2))       # a quarter turn, and none
    assert R.turn64(x, cs, "interleaved").flatten().tolist() == [-2.0, 1.0, 3.0, 4.0, 5.0]
    assert R.turn64(x, cs, "half").flatten().tolist() == [-3.0, 2.0, 1.0, 4.0, 5.0]
    assert R.turn64(R.turn64(x, cs, "half"), cs, "half", inverse=True).equal(x)


def test_scaled_frequencies_by_hand():
    f, a = R.frequencies64(4, base=16.0)
    assert f == [1.0, 0.5, 0.25, 0.125] and a == 1.0
    assert R.frequencies64(4, base=16.0, scaling="linear", factor=2.0)[0] == [0.5, 0.25, 0.125, 0.0625]
    assert R.frequencies64(2, base=16.0, scaling="ntk", factor=4.0)[0] == [1.0, 256.0 ** -0.5]
    # turns over 64 pi positions: 32, 16, 8 and 4
    f, a = R.frequencies64(4, base=16.0, scaling="yarn", factor=2.0, original=64 * math.pi)
    assert f == pytest.approx([1.0, 0.5 * (15 / 31) + 0.25 * (16 / 31), 0.25 * (7 / 31) + 0.125 * (24 / 31), 0.125 * (3 / 31) + 0.0625 * (28 / 31)]) and a == pytest.approx(0.1 * math.log(2) + 1)


def test_positions_of_a_grid_by_hand():
    table = (torch.arange(9, dtype=R.F64).reshape(9, 1, 1).expand(9, 3, 2).clone(), (2, 3, 4), (1, 1, 1))
    c, _ = R.factors64(table, 1, 24)
    # token 17 of 2 x 3 x 4 is (1, 1, 1): rows 1, 2 + 1 and 2 + 3 + 1
    assert c[0, 0, 17].tolist() == [1.0, 3.0, 6.0] and R.factors64(table, 1, 2, first=16)[0][0, 0, 1].tolist() == [1.0, 3.0, 6.0]
    c, _ = R.factors64(table, 1, 2, torch.tensor([[0, 2, 3], [2, 0, -1]]))
    assert c[0, 0, 0].tolist() == [0.0, 4.0, 8.0] and c[0, 0, 1].isnan().tolist() == [True, False, True]


def test_gradients_of_the_plain_forms():
    torch.manual_seed(0)
    for norm in ("head", "row"):
        x, w = torch.randn(2, 3, 4, 6, dtype=R.F64, requires_grad=True), torch.randn(18 if norm == "row" else 6, dtype=R.F64, requires_grad=True)
        cs = R.factors64((R.table64((4,), (2,)), (4,), (2,)), 2, 4)
        for layout in ("interleaved", "half"):
            def f(x, w):
                n, _, s = R.normed64(x, w, norm, 1e-3)
                return R.turn64(n * s, cs, layout)
            y = f(x, w)
            dy = torch.randn_like(y)
            dx, dw = torch.autograd.grad(y, (x, w), dy)
            n, r, s = R.normed64(x.detach(), w.detach(), norm, 1e-3)
            d = R.turn64(dy, cs, layout, inverse=True)
            dims = (3,) if norm == "head" else (1, 3)
            assert torch.allclose(dx, r * (d * s - n * (d * s * n).mean(dims, keepdim=True)))
            assert torch.allclose(dw, (d * n).sum((0, 1, 2)) if norm == "head" else (d * n).sum((0, 2)).reshape(-1))
    for act in (None, "relu", "silu", "gelu", "gelu_tanh"):
        z = torch.linspace(-9, 9, 401, dtype=R.F64, requires_grad=True)
        u, slope = R.act64(z, act)
        assert torch.allclose(torch.autograd.grad(u.sum(), z)[0], slope.detach())
        lib = {None: lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}
        assert torch.allclose(u, lib[act](z), atol=1e-12)


def test_the_checks_see_a_wrong_value():
    torch.manual_seed(1)
    x, w = torch.randn(5, 16).to(torch.bfloat16), torch.randn(8, 16).to(torch.bfloat16)
    z = x.to(R.F64) @ w.to(R.F64).T
    R.check_linear(z.to(torch.bfloat16), x, w)
    for spoil in (1.01, 0.98):
        y = z.clone()
        y[2, 3] *= spoil
        with pytest.raises(AssertionError):
            R.check_linear(y.to(torch.bfloat16), x, w)
    q = torch.randn(1, 2, 3, 8).to(torch.bfloat16)
    n, _, s = R.normed64(q, None, "head", 1e-6)
    R.check_forward(n.to(torch.bfloat16), q, None, None, "head", 1e-6, None)
    with pytest.raises(AssertionError):
        R.check_forward((n * 1.01).to(torch.bfloat16), q, None, None, "head", 1e-6, None)


# ------------------------------------------------------------------------------------------------ refusals of the C entries
def _rows(rows, cols, data=P, dtype=binding.AS_DTYPE_BF16, head_dim=None, tokens=None, strides=None):
    sb, sh, st = strides or (0, 0, cols)
    return binding.as_rows_t(data, dtype, cols if head_dim is None else head_dim, rows if tokens is None else tokens, sb, sh, st)


def _heads(B=2, H=3, N=5, d=16, data=P, dtype=binding.AS_DTYPE_BF16):
    return binding.as_rows_t(data, dtype, d, N, H * N * d, N * d, d)


def _axis(**kw):
    a = binding.as_rotary_axis_t(size=4, pairs=3, base=10000.0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(size=0), INVALID), (dict(pairs=0), INVALID), (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID), (dict(reserved=1), INVALID), (dict(base=0.0), INVALID), (dict(base=float("inf")), INVALID),
    (dict(base=float("nan")), INVALID), (dict(scaling=1, factor=0.5), INVALID), (dict(scaling=2, factor=float("nan")), INVALID), (dict(scaling=3, factor=2.0), INVALID), (dict(pairs=8193), UNSUPPORTED)])
def test_table_refuses(lib, kw, status):
    axes = (binding.as_rotary_axis_t * 1)(_axis(**kw))
    assert lib.as_rotary_table(axes, 1, P, None) == status


def test_table_refuses_its_arguments(lib):
    axes = (binding.as_rotary_axis_t * 5)(*[_axis() for _ in range(5)])
    for args in ((None, 1, P), (axes, 0, P), (axes, 5, P), (axes, 1, None), (axes, 1, P + 8)):
        assert lib.as_rotary_table(args[0], args[1], args[2], None) == INVALID


def _turn(rotation=None, **kw):
    a = binding.as_qk_norm_rotary_t(struct_size=C.sizeof(binding.as_qk_norm_rotary_t), norm=1, rows=10, head_dim=16, q_heads=3, k_heads=3, eps=1e-6, q=_heads(), k=_heads(), q_out=_heads(), k_out=_heads())
    r = a.rotation
    r.table, r.n_axes, r.size[0], r.pairs[0] = P, 1, 5, 8
    for k, v in kw.items():
        setattr(a, k, v)
    for k, v in (rotation or {}).items():
        if k in ("size", "pairs"):
            for i, x in enumerate(v):
                getattr(r, k)[i] = x
        else:
            setattr(r, k, v)
    return a


TURNS = [dict(struct_size=8), dict(norm=3), dict(norm=-1), dict(rows=-1), dict(rows=1 << 31), dict(rows=9), dict(head_dim=0), dict(head_dim=8), dict(head_dim=1025), dict(q_heads=0), dict(k_heads=0), dict(q_heads=4),
         dict(eps=-1.0), dict(eps=float("nan")), dict(q=_heads(data=0)), dict(q=_heads(data=P + 1)), dict(q=_heads(dtype=binding.AS_DTYPE_F32)), dict(k=_heads(dtype=binding.AS_DTYPE_F32)), dict(k=_heads(N=10, B=1)),
         dict(weight_dtype=9), dict(q_weight=P + 1), dict(weight_dtype=1, k_weight=P + 2), dict(reserved=1)]
TURNS_R = [dict(table=P + 4), dict(n_axes=0), dict(n_axes=5), dict(layout=2), dict(inverse=2), dict(size=(0,)), dict(pairs=(0,)), dict(pairs=(9,)), dict(n_axes=2, size=(5, 5), pairs=(8, 1)), dict(first=1), dict(first=-1),
           dict(size=(4,)), dict(positions=P, position_bytes=2), dict(positions=P + 4, position_bytes=8), dict(positions=P, position_bytes=4, positions_stride=-1)]


@pytest.mark.parametrize("kw", TURNS)
def test_turns_refuse(lib, kw):
    assert lib.as_qk_norm_rotary(C.addressof(_turn(**kw)), None) == INVALID
    if "struct_size" not in kw:
        b = _back(_turn(**kw))
        assert lib.as_qk_norm_rotary_backward(C.addressof(b), None) == INVALID


@pytest.mark.parametrize("kw", TURNS_R)
def test_rotations_refuse(lib, kw):
    assert lib.as_qk_norm_rotary(C.addressof(_turn(rotation=kw)), None) == INVALID


def test_turns_refuse_outputs(lib):
    for kw in (dict(q_out=_heads(data=0)), dict(k_out=binding.as_rows_t()), dict(k=binding.as_rows_t()), dict(q_out=_rows(10, 48)), dict(q_out=binding.as_rows_t(P, 0, 16, 5, 240, 80, 15)), dict(q_out=_heads(dtype=1))):
        assert lib.as_qk_norm_rotary(C.addressof(_turn(**kw)), None) == INVALID
    wide = binding.as_rows_t(P, 0, 16, 5, 0, 16, 16 * 1025)
    assert lib.as_qk_norm_rotary(C.addressof(_turn(norm=2, rows=5, q_heads=1025, k=binding.as_rows_t(), k_out=binding.as_rows_t(), q=wide, q_out=wide)), None) == UNSUPPORTED


def _back(fwd, **kw):
    b = binding.as_qk_norm_rotary_backward_t(struct_size=C.sizeof(binding.as_qk_norm_rotary_backward_t), fwd=C.pointer(fwd), dq=_heads(), dk=_heads(), dq_out=_heads(), dk_out=_heads())
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def test_turns_backward_refuse(lib):
    n = C.c_uint64()
    fwd = _turn(q_weight=P, k_weight=P)
    for kw in (dict(struct_size=8), dict(reserved=1), dict(dq=_heads(data=0)), dict(dk=binding.as_rows_t()), dict(dq_out=_heads(dtype=1)), dict(dk_out=binding.as_rows_t()), dict(dq_weight=P + 1)):
        b = _back(fwd, **kw)
        assert lib.as_qk_norm_rotary_backward(C.addressof(b), None) == INVALID
        assert lib.as_qk_norm_rotary_backward_workspace_bytes(C.addressof(b), C.byref(n)) == INVALID
    b = _back(_turn(norm=0))
    assert lib.as_qk_norm_rotary_backward(C.addressof(b), None) == INVALID
    b = _back(_turn(), dq_weight=P)                              # a gradient of no weight
    assert lib.as_qk_norm_rotary_backward(C.addressof(b), None) == INVALID
    assert lib.as_qk_norm_rotary_backward_workspace_bytes(C.addressof(_back(fwd)), None) == INVALID and lib.as_qk_norm_rotary_backward(None, None) == INVALID


def test_no_rows_need_no_device(lib):
    none = _turn(rows=0)
    assert lib.as_qk_norm_rotary(C.addressof(none), None) == binding.AS_OK


def test_linear_without_a_context(lib):
    a = binding.as_linear_t(struct_size=C.sizeof(binding.as_linear_t))
    b = binding.as_linear_backward_t(struct_size=C.sizeof(binding.as_linear_backward_t))
    n = C.c_uint64()
    assert lib.as_linear(None, C.addressof(a), None) == INVALID and lib.as_linear_backward(None, C.addressof(b), None) == INVALID
    assert lib.as_linear_workspace_bytes(None, C.addressof(a), C.byref(n)) == INVALID and lib.as_linear_backward_workspace_bytes(None, C.addressof(b), C.byref(n)) == INVALID


def test_calls_without_a_device_fail_loudly(lib):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    from paper_2509_24899_b200 import linear, linear_backward, qk_norm_rotary, qk_norm_rotary_backward, rotary, rotary_table
    x, q = torch.zeros(2, 4, dtype=torch.bfloat16), torch.zeros(1, 1, 2, 4, dtype=torch.bfloat16)
    table = (torch.zeros(2, 2, 2), (2,), (2,))
    for f in (lambda: linear(x, x), lambda: linear_backward(x, x, x), lambda: rotary(q, table), lambda: qk_norm_rotary(q, q), lambda: qk_norm_rotary_backward(q, q, q, q), lambda: rotary_table((2,), (2,))):
        with pytest.raises((ValueError, RuntimeError)):
            f()


def test_struct_sizes():
    assert [C.sizeof(s) for s in (binding.as_rotary_axis_t, binding.as_rotation_t, binding.as_qk_norm_rotary_t, binding.as_qk_norm_rotary_backward_t, binding.as_linear_t, binding.as_linear_backward_t)] == [40, 80, 328, 240, 328, 384]


def test_no_failed_cuda_call_leaves_its_error_behind():
    """Calls that give up because one of CUDA's has failed say so through `failed`, which takes the pending error away; and no call sets a kernel's limits for itself alone."""
    for name in ("rotary.cu", "linear.cu"):
        with open(os.path.join(build.CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        assert "failed()" in text and "AS_ERR_CUDA" not in text, name
        assert text.count("cudaFuncSetAttribute") == (1 if name == "rotary.cu" else 0), name
