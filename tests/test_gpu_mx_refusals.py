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


def test_buffers_of_a_smaller_dispatch():
    """test_mx_binding shows on the CPU that such a call does not reach the library."""
    r = _router(4)
    logits, x = torch.randn(9, 4, device="cuda"), torch.randn(9, 64, device="cuda").bfloat16()
    whole = torch.full((64,), -7, dtype=torch.int32, device="cuda")
    out = r.alloc_outputs(8, send_buf=False)
    out.dst_row = whole[:8]
    with pytest.raises(B.MoeError):
        r.mx_dispatch(logits, x, out)
    gate_up, down = (B.mx_quantize(torch.randn(4, 64, cols, device="cuda")) for cols in (64, 32))
    with pytest.raises(B.MoeError):
        r.mx_step(logits, x, gate_up, down, out)
    torch.cuda.synchronize()
    assert (whole == -7).all()
    large = r.alloc_outputs(12, send_buf=False)              # room for more tokens is fine
    r.mx_dispatch(logits, x, large)
    want, _ = r.mx_dispatch(logits, x)
    torch.cuda.synchronize()
    for f in ("topk_ids", "topk_slot", "dst_row", "src_index"):
        a = getattr(want, f).flatten()
        assert torch.equal(getattr(large, f).flatten()[:a.numel()], a), f
    r.close()


def test_a_step_into_a_shorter_y():
    """test_mx_binding shows on the CPU that nothing is launched."""
    r = _router(4)
    logits, x = torch.randn(9, 4, device="cuda"), torch.randn(9, 64, device="cuda").bfloat16()
    gate_up, down = (B.mx_quantize(torch.randn(4, 64, cols, device="cuda")) for cols in (64, 32))
    whole = torch.full((9, 64), -7.0, dtype=torch.bfloat16, device="cuda")
    for y in (whole[:8], whole[:, :32], whole.float(), whole.cpu()):
        with pytest.raises(B.MoeError):
            r.mx_step(logits, x, gate_up, down, y=y)
    torch.cuda.synchronize()
    assert (whole == -7).all()
    want = r.mx_step(logits, x, gate_up, down)
    assert torch.equal(r.mx_step(logits, x, gate_up, down, y=whole), want)
    r.close()
