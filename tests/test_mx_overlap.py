"""CPU-only: quantising or dequantising onto its own input is refused.  (Without a GPU a call that passes the checks
ends at its launch with MOE_ERR_CUDA, so nothing is ever read or written here.)"""
import numpy as np
import pytest
import torch

from paper_2602_21140_b200 import binding as B
from paper_2602_21140_b200 import build as build_mod

A = 1 << 30                 # some 16-byte aligned address


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build_library()
    if torch.cuda.is_available():
        pytest.skip("calls that pass the checks would be launched")


def _both(x, dtype, rows, cols, stride, codes, scales):
    st = B.moe_mx_quantize(x, dtype, rows, cols, stride, codes, scales)
    assert B.moe_mx_dequantize(codes, scales, rows, cols, x, dtype, stride) == st
    return st


def test_apart_and_adjacent_buffers_pass():
    # 4 rows of 64 bf16: 512 bytes; codes 128 bytes, scales 64 bytes
    for codes, scales in ((A + 512, A + 640), (A - 128, A - 192), (A + 512, A - 64)):
        assert _both(A, 0, 4, 64, 64, codes, scales) == B.MOE_ERR_CUDA


@pytest.mark.parametrize("codes,scales", [(A, A + 4096), (A + 496, A + 4096), (A - 112, A + 4096), (A + 4096, A), (A + 4096, A + 496),
                                          (A + 4096, A - 48), (A + 4096, A + 4096 + 112), (A + 4096, A + 4096 - 48), (A + 64, A + 96)])
def test_shared_bytes_are_refused(codes, scales):
    assert _both(A, 0, 4, 64, 64, codes, scales) == B.MOE_ERR_INVALID_ARG


def test_between_strided_rows():
    """Codes in the gap between two rows share nothing with them."""
    # 2 rows of 64 fp32 (256 bytes), 1024 bytes apart; codes 64 bytes, scales 32
    assert _both(A, 2, 2, 64, 256, A + 256, A + 992) == B.MOE_ERR_CUDA
    assert _both(A, 2, 2, 64, 256, A + 240, A + 512) == B.MOE_ERR_INVALID_ARG
    assert _both(A, 2, 2, 64, 256, A + 256, A + 1008) == B.MOE_ERR_INVALID_ARG
    assert _both(A, 2, 2, 64, 256, A + 1280, A + 512) == B.MOE_ERR_CUDA


def test_against_sets_of_bytes():
    rng = np.random.default_rng(1)
    seen = set()
    for _ in range(400):
        rows, cols, dtype = int(rng.integers(1, 5)), 32 * int(rng.integers(1, 4)), int(rng.integers(0, 3))
        size = 4 if dtype == 2 else 2
        stride = cols + 16 // size * int(rng.integers(0, 20))
        x = {A + r * stride * size + b for r in range(rows) for b in range(cols * size)}
        codes, scales = (A + 16 * int(v) for v in rng.integers(-20, 120, 2))
        c = set(range(codes, codes + rows * cols // 2))
        s = set(range(scales, scales + rows * B.moe_mx_scale_pitch(cols)))
        want = B.MOE_ERR_INVALID_ARG if (x & c or x & s or c & s) else B.MOE_ERR_CUDA
        assert _both(A, dtype, rows, cols, stride, codes, scales) == want
        seen.add(want)
    assert len(seen) == 2
