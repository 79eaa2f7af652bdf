"""Gradients written over what they are computed from: rows are read ahead of the ones that are written, tokens are
taken by whichever CTA is free, so every shared byte is refused before anything is launched."""
import pytest
import torch

from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [1, 2])
def test_shared_bytes_are_refused(k):
    T, H, E = 8, 64, 8
    r = B.MoeRouter(B.make_config(E, k, H, T, E, 1, 1), range(E), None, [1.0] * E)
    g = torch.Generator(device="cuda").manual_seed(k)
    logits = torch.randn(T, E, device="cuda", generator=g)
    out = r.dispatch(logits, torch.randn(T, H, device="cuda", generator=g).bfloat16())
    big = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    n, bf, f32 = T * k, torch.bfloat16, torch.float32

    def at(start, *shape, dtype=bf):
        size = torch.Size(shape).numel() * torch.empty(0, dtype=dtype).element_size()
        return big[start:start + size].view(dtype).view(shape)

    rows_bytes, x_bytes = n * H * 2, T * H * 2
    buf, dy, d_buf, d_w = at(0, n, H), at(8192, T, H), at(16384, n, H), at(24576, T, k, dtype=f32)
    big.copy_(torch.arange(1 << 16, device="cuda") % 64)      # small bf16 and fp32 numbers
    before, bad = big.clone(), []
    for s in (0, 128, rows_bytes - 16, 8192, 8192 + x_bytes - 16, 8192 - rows_bytes + 16, 24576 - rows_bytes + 16):
        bad.append(lambda s=s: r.combine_backward(buf, dy, at(s, n, H), d_w))
    for s in (0, rows_bytes - 4, 8192, 8192 + x_bytes - 4, 16384, 16384 + rows_bytes - 4):
        bad.append(lambda s=s: r.combine_backward(buf, dy, d_buf, at(s, T, k, dtype=f32)))
    d_send, lg, dx, d_l = buf, at(28672, T, E, dtype=f32), at(32768, T, H), at(40960, T, E, dtype=f32)
    for s in (0, rows_bytes - 16, 24576, 28672, 40960, 40960 - x_bytes + 16):
        bad.append(lambda s=s: r.dispatch_backward(lg, d_send, d_w, at(s, T, H), d_l))
    for s in (0, rows_bytes - 16, 24576, 28672, 28672 + 4 * E, 32768, 32768 + x_bytes - 16):
        bad.append(lambda s=s: r.dispatch_backward(lg, d_send, d_w, dx, at(s, T, E, dtype=f32)))
    bad.append(lambda: r.dispatch_backward(None, d_send, None, at(0, T, H)))
    for i, call in enumerate(bad):
        with pytest.raises(B.MoeError):
            call()
            pytest.fail(f"call {i} was accepted")
    torch.cuda.synchronize()
    assert torch.equal(big, before) and r.device_status() == 0
    # side by side: the same bits as in tensors of their own
    near = r.combine_backward(buf, dy, at(16384, n, H), at(16384 + rows_bytes, T, k, dtype=f32))
    own = r.combine_backward(buf.clone(), dy.clone())
    assert all(torch.equal(a, b) for a, b in zip(near, own))
    lg.copy_(logits)
    near = r.dispatch_backward(lg, d_send, d_w, at(rows_bytes, T, H), at(rows_bytes + x_bytes, T, E, dtype=f32))
    own = r.dispatch_backward(logits, d_send.clone(), d_w.clone())
    assert all(torch.equal(a, b) for a, b in zip(near, own))
    del out
    r.close()
