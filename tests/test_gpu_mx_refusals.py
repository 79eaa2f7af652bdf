"""Calls of the 4-bit operators that the host has to refuse before anything is launched."""
import pytest
import torch

from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


def _router(P):
    return B.MoeRouter(B.make_config(P, 1, 64, 16, P, 1, 1), range(P), None, [1.0] * P)


def test_features_that_an_int_cannot_round_up():
    """test_mx_limits shows on the CPU that product_fits refuses these sizes."""
    r = _router(2)
    rows, w = B.mx_quantize(torch.zeros(4, 64, device="cuda")), B.mx_quantize(torch.zeros(2, 128, 64, device="cuda"))
    counts = torch.tensor([2, 2], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    y = torch.full((4, 128), -7.0, dtype=torch.bfloat16, device="cuda")
    for n_out in (2 ** 31 - 8, 2 ** 31 - 128, 2 ** 30 + 8):
        assert B.moe_mx_expert_product(r._ctx, rows.codes.data_ptr(), rows.scales.data_ptr(), 4, counts.data_ptr(), offsets.data_ptr(),
                                       w.codes.data_ptr(), w.scales.data_ptr(), n_out, 64, y.data_ptr()) == B.MOE_ERR_CAPACITY
    torch.cuda.synchronize()
    assert (y == -7).all() and r.device_status() == 0
    r.close()
