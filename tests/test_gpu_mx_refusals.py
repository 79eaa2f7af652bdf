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


def test_outputs_over_inputs():
    """Other CTAs read the rows and the weights while a tile is written."""
    r = _router(2)
    n, K, N = 6, 256, 512                                      # gated: 256 features, rows as large as those that come in
    big = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")

    def at(start, *shape, dtype=torch.uint8):
        count = torch.Size(shape).numel()
        return big[start:start + count * torch.empty(0, dtype=dtype).element_size()].view(dtype).view(shape)

    rows, w = B.MxRows(at(0, n, K // 2), at(4096, n, 16)), B.MxRows(at(1 << 18, 2, N, K // 2), at(1 << 17, 2, N, 16))
    counts, offsets = at(8192, 2, dtype=torch.int32), at(8448, 3, dtype=torch.int32)
    counts.copy_(torch.tensor([2, 4])); offsets.copy_(torch.tensor([0, 2, 6]))
    apart = B.MxRows(at(12288, n, K // 2), at(16384, n, 16))
    before = big.clone()
    for bad in (B.MxRows(rows.codes, apart.scales), B.MxRows(apart.codes, rows.scales), rows, B.MxRows(at((n - 1) * K // 2, n, K // 2), apart.scales),
                B.MxRows(at(4096 - 64, n, K // 2), apart.scales), B.MxRows(w.codes[1, :n], apart.scales), B.MxRows(apart.codes, w.scales[0, :n]),
                B.MxRows(at(8192 - 128, n, K // 2), apart.scales), B.MxRows(apart.codes, at(8448 - 16, n, 16)),
                B.MxRows(apart.codes, at(12288 + 64, n, 16))):
        with pytest.raises(B.MoeError):
            r.mx_expert_gated(rows, counts, offsets, w, bad)
    for start in (0, 4096 - 64, 8192 - 1024, (1 << 18) - 16, (1 << 17) + 16 * N * 2 - 16):
        with pytest.raises(B.MoeError):
            r.mx_expert_product(rows, counts, offsets, w, at(start, n, N, dtype=torch.bfloat16))
    with pytest.raises(B.MoeError):                            # the hidden rows of a whole network over the rows that come in
        r.mx_expert_ffn(rows, counts, offsets, w, B.MxRows(at(1 << 19, 2, 64, K // 2), at(20480, 2, 64, 16)), hidden=rows)
    x, logits = at(32768, 8, 64, dtype=torch.bfloat16), torch.zeros(8, 2, device="cuda")
    for codes, scales in ((32768, 65536), (65536, 32768), (65536, 65536 + 128), (32768 + 1008, 65536), (32768 - 240, 65536)):
        with pytest.raises(B.MoeError):
            r.mx_dispatch(logits, x, rows=B.MxRows(at(codes, 8, 32), at(scales, 8, 16)))
    torch.cuda.synchronize()
    assert torch.equal(big, before) and r.device_status() == 0
    # side by side is fine
    r.mx_expert_gated(rows, counts, offsets, w, apart)
    r.mx_expert_product(rows, counts, offsets, w, at(49152, n, N, dtype=torch.bfloat16))
    r.mx_dispatch(logits, x, rows=B.MxRows(at(32768 + 1024, 8, 32), at(32768 + 1024 + 256, 8, 16)))
    torch.cuda.synchronize()
    assert r.device_status() == 0
    r.close()
