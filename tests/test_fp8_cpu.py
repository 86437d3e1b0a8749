"""The 8-bit projections without a GPU: the plain forms against values worked by hand, the structs that the binding packs, and the refusals of the C entries, which
come before any CUDA call."""
import ctypes as C

import pytest
import torch

from paper_2509_24899_b200 import binding, build
from tests import _fp8 as R


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_exponents_by_hand():
    top = torch.tensor([[448.0], [449.0], [1.0], [1.75], [1.7500001], [0.0], [3.5 * 2.0 ** -20]], dtype=R.F64)
    # 1.75 = 448 * 2^-8; 1 needs 2^-8 as well (448 * 2^-9 = 0.875); 3.5 * 2^-20 = 448 * 2^-27
    assert R.exponents64(top).flatten().tolist() == [0, 1, -8, -8, -7, -127, -27]


def test_values_by_hand():
    data, scales = R.pair_of(torch.tensor([[1.0, -448.0] + [0.0] * 126 + [2.0]], dtype=R.F64))
    assert scales.flatten().tolist() == [127, 127 - 7, 0, 0]                   # 2 / 448 needs 2^-7 (448 * 2^-8 = 1.75)
    assert data[0, :2].float().tolist() == [1.0, -448.0] and float(data[0, 128]) == 256.0
    assert R.value64((data, scales))[0, [0, 1, 128]].tolist() == [1.0, -448.0, 2.0]


def test_the_checks_see_a_wrong_scale_and_a_wrong_value():
    torch.manual_seed(0)
    y = torch.randn(5, 300, dtype=R.F64)
    R.check_form(R.pair_of(y), y)
    for spoil in ("scale", "value", "behind"):
        data, scales = R.pair_of(y)
        if spoil == "scale":
            scales[0, 2, 1] += 1
        elif spoil == "value":
            data[3, 200] = 3 * float(data[3, 200]) + 8
        else:
            scales[0, 1, 3] = 1
        with pytest.raises(AssertionError):
            R.check_form((data, scales), y)


def _rows(rows, cols, data=1 << 20, dtype=binding.AS_DTYPE_BF16, head_dim=None, tokens=None, strides=None):
    sb, sh, st = strides or (0, 0, cols)
    return binding.as_rows_t(data, dtype, cols if head_dim is None else head_dim, rows if tokens is None else tokens, sb, sh, st)


def _matrix(rows, cols, data=1 << 20, scales=1 << 20, pitch=None, scale_rows=None):
    return binding.as_fp8_matrix_t(data, (cols + 15) // 16 * 16 if pitch is None else pitch, scales, rows if scale_rows is None else scale_rows)


def _norm(rows=4, cols=256, **kw):
    a = binding.as_rms_norm_t(struct_size=C.sizeof(binding.as_rms_norm_t), rows=rows, cols=cols, x=_rows(rows, cols), out=_rows(rows, cols), eps=1e-6)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


INVALID, UNSUPPORTED = binding.AS_ERR_INVALID_ARG, binding.AS_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), INVALID), (dict(rows=-1), INVALID), (dict(rows=1 << 31), INVALID), (dict(cols=0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(eps=-1.0), INVALID), (dict(x=_rows(4, 256, data=0)), INVALID), (dict(x=_rows(4, 256, data=(1 << 20) + 1)), INVALID),
    (dict(x=_rows(4, 256, dtype=7)), INVALID), (dict(x=_rows(4, 256, head_dim=100)), INVALID), (dict(x=_rows(4, 256, tokens=3)), INVALID),
    (dict(x=_rows(4, 256, strides=(0, 0, -256))), INVALID), (dict(out=_rows(4, 256, dtype=binding.AS_DTYPE_F32)), INVALID),
    (dict(out=_rows(4, 256, strides=(0, 0, 255))), INVALID),                                    # rows that overlap
    (dict(out=_rows(4, 256, head_dim=64, tokens=2, strides=(64, 512, 64))), INVALID),            # the batch's second entry on the first one's second token
    (dict(out8=_matrix(4, 256)), INVALID),                                                      # both forms of the output
    (dict(out=binding.as_rows_t()), INVALID),                                                   # neither
    (dict(out=binding.as_rows_t(), out8=_matrix(4, 256, pitch=248)), INVALID), (dict(out=binding.as_rows_t(), out8=_matrix(4, 256, pitch=240)), INVALID),
    (dict(out=binding.as_rows_t(), out8=_matrix(4, 256, data=(1 << 20) + 8)), INVALID), (dict(out=binding.as_rows_t(), out8=_matrix(4, 256, scales=(1 << 20) + 2)), INVALID),
    (dict(out=binding.as_rows_t(), out8=_matrix(4, 256, scale_rows=3)), INVALID),
    (dict(residual=_rows(4, 256)), INVALID), (dict(residual_out=_rows(4, 256)), INVALID),       # one without the other
    (dict(residual=_rows(4, 256), residual_out=_rows(4, 256, dtype=binding.AS_DTYPE_F32)), INVALID),
    (dict(weight=1 << 20, weight_dtype=9), INVALID), (dict(weight=(1 << 20) + 1), INVALID),
    (dict(x=_rows(4, 256, dtype=binding.AS_DTYPE_F32), residual=_rows(4, 256), residual_out=_rows(4, 256)), UNSUPPORTED),
    (dict(cols=16385, x=_rows(4, 16385), out=_rows(4, 16385)), UNSUPPORTED)])
def test_norm_refuses(lib, kw, status):
    assert lib.as_rms_norm(C.addressof(_norm(**kw)), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=8), INVALID), (dict(block_rows=2), INVALID), (dict(reserved=1), INVALID), (dict(rows=-1), INVALID), (dict(cols=0), INVALID),
    (dict(out=_matrix(4, 256, data=0)), INVALID), (dict(x=_rows(4, 256, tokens=0)), INVALID), (dict(cols=16640, x=_rows(4, 16640), out=_matrix(4, 16640)), UNSUPPORTED)])
def test_quantize_refuses(lib, kw, status):
    a = binding.as_quantize_fp8_t(struct_size=C.sizeof(binding.as_quantize_fp8_t), rows=4, cols=256, x=_rows(4, 256), out=_matrix(4, 256), block_rows=1)
    for k, v in kw.items():
        setattr(a, k, v)
    assert lib.as_quantize_fp8(C.addressof(a), None) == status


def test_null_arguments_and_empty_calls(lib):
    for f in (lib.as_rms_norm, lib.as_quantize_fp8):
        assert f(None, None) == INVALID
    assert lib.as_matmul_fp8(None, None, None) == INVALID and lib.as_fp8_create(None) == INVALID and lib.as_fp8_last_status(None, None) == INVALID
    assert lib.as_fp8_destroy(None) == binding.AS_OK
    # no rows: nothing to launch, and no device needed
    assert lib.as_rms_norm(C.addressof(_norm(rows=0, x=_rows(0, 256), out=_rows(0, 256))), None) == binding.AS_OK


def test_struct_sizes(lib):
    """The binding's structs have the sizes that the C entries ask for: they get past that check."""
    for f, struct in ((lib.as_rms_norm, binding.as_rms_norm_t), (lib.as_quantize_fp8, binding.as_quantize_fp8_t)):
        a = struct(struct_size=C.sizeof(struct), rows=0, cols=8, x=_rows(0, 8), out=_rows(0, 8) if struct is binding.as_rms_norm_t else _matrix(0, 8))
        if struct is binding.as_quantize_fp8_t:
            a.block_rows = 1
        assert f(C.addressof(a), None) == binding.AS_OK
    assert C.sizeof(binding.as_rows_t) == 48 and C.sizeof(binding.as_fp8_matrix_t) == 32 and C.sizeof(binding.as_matmul_fp8_t) == 144


def test_calls_without_a_device_fail_loudly(lib):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    from paper_2509_24899_b200 import matmul_fp8, quantize_fp8, rms_norm
    x = torch.zeros(2, 4, dtype=torch.bfloat16)
    for f in (lambda: rms_norm(x), lambda: quantize_fp8(x), lambda: matmul_fp8((x, x), (x, x))):
        with pytest.raises((ValueError, RuntimeError)):
            f()
    with pytest.raises(binding.AsError):
        binding.as_fp8_create()
