"""CPU-only: the 4-bit format's pitch and argument checks through the C ABI (no kernel is launched), and
the tests' own statement of the format against hand-worked blocks."""
import numpy as np
import pytest

import mx_util as M
from paper_2602_21140_b200 import binding as B
from paper_2602_21140_b200 import build as build_mod


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build_library()


def test_scale_pitch():
    for cols in (32, 64, 512, 544, 1024, 4096, 7168):
        assert B.moe_mx_scale_pitch(cols) == M.pitch(cols) == B._mx_pitch(cols)
    for cols in (0, -32, 16, 33, 48):
        assert B.moe_mx_scale_pitch(cols) == 0


P = 1 << 20      # any 16-byte aligned non-null value: refused calls never look at it


@pytest.mark.parametrize("args,status", [
    ((P, 3, 1, 32, 32, P, P), B.MOE_ERR_INVALID_ARG), ((P, -1, 1, 32, 32, P, P), B.MOE_ERR_INVALID_ARG),
    ((P, 0, -1, 32, 32, P, P), B.MOE_ERR_INVALID_ARG), ((P, 0, 1, 0, 32, P, P), B.MOE_ERR_INVALID_ARG),
    ((P, 0, 1, 40, 40, P, P), B.MOE_ERR_INVALID_ARG), ((P, 0, 2, 64, 32, P, P), B.MOE_ERR_INVALID_ARG),
    ((P, 0, 2, 32, 36, P, P), B.MOE_ERR_INVALID_ARG), ((P + 2, 0, 1, 32, 32, P, P), B.MOE_ERR_INVALID_ARG),
    ((P, 0, 1, 32, 32, P + 8, P), B.MOE_ERR_INVALID_ARG), ((P, 0, 1, 32, 32, P, P + 1), B.MOE_ERR_INVALID_ARG),
    ((0, 0, 1, 32, 32, P, P), B.MOE_ERR_INVALID_ARG), ((P, 0, 1, 32, 32, 0, P), B.MOE_ERR_INVALID_ARG),
    ((P, 0, 1, 32, 32, P, 0), B.MOE_ERR_INVALID_ARG), ((P, 0, 1 << 40, 32, 32, P, P), B.MOE_ERR_CAPACITY),
    ((0, 0, 0, 32, 32, 0, 0), B.MOE_OK)])
def test_quantize_arguments(args, status):
    x, dtype, rows, cols, stride, codes, scales = args
    assert B.moe_mx_quantize(x, dtype, rows, cols, stride, codes, scales) == status
    assert B.moe_mx_dequantize(codes, scales, rows, cols, x, dtype, stride) == status


def test_context_calls_without_a_context():
    assert B.moe_mx_expert_product(None, P, P, 1, P, P, P, P, 8, 32, P) == B.MOE_ERR_INVALID_ARG
    assert B.moe_mx_expert_gated(None, P, P, 1, P, P, P, P, 32, 32, P, P) == B.MOE_ERR_INVALID_ARG
    assert B.moe_mx_dispatch(None, P, P, 1, B.moe_dispatch_out(), P, P) == B.MOE_ERR_INVALID_ARG
    assert B.moe_combine_backward(None, P, P, 1, P, P) == B.MOE_ERR_INVALID_ARG
    assert B.moe_dispatch_backward(None, P, P, P, 1, P, P) == B.MOE_ERR_INVALID_ARG


def test_cpu_tensors_are_refused():
    import torch
    with pytest.raises(B.MoeError):
        B.mx_quantize(torch.zeros(2, 32))
    with pytest.raises(B.MoeError):
        B.mx_dequantize(B.MxRows(torch.zeros(2, 16, dtype=torch.uint8), torch.zeros(2, 16, dtype=torch.uint8)))


def test_the_tests_own_format():
    """Hand-worked: largest magnitude 7.9 -> scale 2^0, saturating; ties go to the even code."""
    x = np.zeros((1, 32))
    x[0, :9] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9, -0.26]
    codes, scales = M.quantize(x)
    assert scales.shape == (1, 16) and scales[0, 0] == 127 and (scales[0, 1:] == 0).all()
    want = [0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -0.5]
    assert M.values(codes, scales)[0, :9].tolist() == want
    assert codes[0, 0] == (0 | (2 << 4)) and codes[0, 4] == 0x9       # low half: the even element
    x[0] = 0
    assert M.quantize(x)[1][0, 0] == 0
    x[0, 5] = 2.0 ** -149
    assert M.quantize(x)[1][0, 0] == 0
    x[0, 5] = np.inf
    assert M.quantize(x)[1][0, 0] == 255 and np.isnan(M.values(*M.quantize(x))).all()
    x[0, 5] = 3.0
    assert M.quantize(x)[1][0, 0] == 126        # floor(log2 3) - 2 = -1
