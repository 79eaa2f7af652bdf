"""Calls of the 16-bit experts that the host has to refuse before anything is launched: sizes, alignment, missing buffers, and
outputs over inputs or over one another."""
import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu

BAD, CAP, OK = B.MOE_ERR_INVALID_ARG, B.MOE_ERR_CAPACITY, B.MOE_OK


@pytest.fixture
def room():
    """A megabyte to place buffers in, which no refused call may change."""
    r = U.make_router(2)
    big = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    base = big.data_ptr()
    big[8192:8200].view(torch.int32).copy_(torch.tensor([2, 4])); big[8448:8456].view(torch.int32).copy_(torch.tensor([0, 2]))
    before = big.clone()
    yield r, base
    torch.cuda.synchronize()
    assert torch.equal(big, before) and r.device_status() == 0
    r.close()


n, H, I = 6, 64, 32
A, C, O, W, Y, Z, S, D = 0, 8192, 8448, 1 << 16, 1 << 17, 1 << 18, 1 << 19, 3 << 18


def test_sizes_and_alignment(room):
    r, base = room
    at = lambda o: base + o                                    # noqa: E731
    c = r._ctx
    for n_out, n_in, want in ((12, 64, BAD), (64, 12, BAD), (0, 64, BAD), (64, 0, BAD), ((1 << 30) + 8, 64, CAP), (64, (1 << 30) + 8, CAP), (-8, 64, BAD)):
        assert B.moe_expert_product(c, at(A), n, at(C), at(O), at(W), n_out, n_in, at(Y)) == want
        assert B.moe_expert_rows_backward(c, at(A), n, at(C), at(O), at(W), n_out, n_in, at(Y)) == want
        assert B.moe_expert_weight_backward(c, at(A), at(Z), n, at(C), at(O), n_out, n_in, at(Y), 0, 0) == want
    for hidden in (0, 8, 24, -16, (1 << 29) + 16):
        assert B.moe_expert_gated(c, at(A), n, at(C), at(O), at(W), hidden, H, at(Y)) == BAD
        assert B.moe_expert_gated_backward(c, at(A), n, at(C), at(O), at(W), H, hidden, at(Z), 0, at(Y), at(D)) == BAD
    assert B.moe_expert_product(c, at(A), -1, at(C), at(O), at(W), H, H, at(Y)) == BAD
    assert B.moe_expert_product(c, at(A), (1 << 30) + 1, at(C), at(O), at(W), H, H, at(Y)) == CAP
    for i in (0, 2, 3, 4, 7):                                  # each pointer missing, and each but the int ones askew
        args = [at(A), n, at(C), at(O), at(W), H, H, at(Y)]
        for bad in (0, args[i] + 8):
            if bad and i in (2, 3):
                continue
            call = args[:i] + [bad] + args[i + 1:]
            assert B.moe_expert_product(c, *call) == BAD and B.moe_expert_rows_backward(c, *call) == BAD, (i, bad)
    assert B.moe_expert_gated(c, at(A), n, at(C), at(O), at(W), I, H, at(Y), 0, at(S)) == BAD        # scales without codes
    assert B.moe_expert_gated(c, at(A), n, at(C), at(O), at(W), I, H, at(Y), at(Z) + 8, 0) == BAD
    assert B.moe_expert_gated_backward(c, at(A), n, at(C), at(O), at(W), H, I, 0, 0, at(Y), at(D)) == BAD
    for dtype, add in ((1, 0), (3, 0), (0, 1)):
        assert B.moe_expert_weight_backward(c, at(A), at(Z), n, at(C), at(O), H, I, at(Y), dtype, add) == BAD
    assert B.moe_expert_weight_backward(c, 0, 0, 0, 0, 0, H, I, 0, 0, 0) == BAD                      # even without rows it is written
    assert B.moe_redispatch(c, at(A), at(S), 4, at(Y)) == BAD                                        # nothing was dispatched


def test_outputs_over_inputs(room):
    r, base = room
    c, at = r._ctx, lambda o: base + o                         # noqa: E731
    rows = n * H * 2
    for y in (A, A + rows - 16, W, W + 2 * H * H * 2 - 16, C - 16, O):
        assert B.moe_expert_product(c, at(A), n, at(C), at(O), at(W), H, H, at(y)) == BAD
        assert B.moe_expert_rows_backward(c, at(A), n, at(C), at(O), at(W), H, H, at(y)) == BAD
    for h, z, s in ((A, Z, S), (Y, A, S), (Y, Z, A), (Y, Y, S), (Y, Z, Y + 16), (Y, Z, Z + 64), (W, Z, None), (Y, W, None), (Y, Y + 16, None)):
        assert B.moe_expert_gated(c, at(A), n, at(C), at(O), at(W), I, H, at(h), at(z), 0 if s is None else at(s)) == BAD
    for dz, h, s in ((A, Y, S), (Y, A, S), (Y, Y + 16, S), (Z, Y, S), (Y, Z, S), (S, Y, S), (Y, W, S), (Z + 16, Y, None)):
        assert B.moe_expert_gated_backward(c, at(A), n, at(C), at(O), at(W), H, I, at(Z), 0 if s is None else at(s), at(dz), at(h)) == BAD
    for dw in (A, Z, C - 64, Z + n * I * 2 - 16):
        assert B.moe_expert_weight_backward(c, at(A), at(Z), n, at(C), at(O), H, I, at(dw), 2, 1) == BAD


def test_redispatch_over_inputs_and_after_other_routing():
    r = B.MoeRouter(B.make_config(4, 2, 64, 16, 1, 4, 1), range(4), None, [1.0] * 4)
    logits, x = torch.randn(8, 4, device="cuda"), U.bf16(8, 64, seed=1)
    out = r.dispatch(logits, x)
    big = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = big.data_ptr()
    for codes, scales, send in ((0, 8192, 0), (0, 8192, 496), (8192, 0, 0), (0, 8192, 8192 + 112)):
        assert B.moe_redispatch(r._ctx, p + codes, p + scales, 8, p + send) == BAD
    assert B.moe_redispatch(r._ctx, p, p + 8192, 8, out.dst_row.data_ptr() // 16 * 16) == BAD
    assert B.moe_redispatch(r._ctx, p, p + 8192, 7, p + 16384) == BAD
    assert B.moe_redispatch(r._ctx, p, p + 8, 8, p + 16384) == BAD
    torch.cuda.synchronize()
    assert not big.any() and r.device_status() == 0
    assert B.moe_redispatch(r._ctx, p, p + 8192, 8, p + 16384) == OK
    r.ep_attach(1, 0, [big.data_ptr()], 16)
    r.ep_route(logits, out)
    assert B.moe_redispatch(r._ctx, p, p + 8192, 8, p + 16384) == BAD
    torch.cuda.synchronize()
    r.close()
