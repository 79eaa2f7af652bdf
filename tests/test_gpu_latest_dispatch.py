"""combine and the gradients read the buffers of the latest dispatch through the context.  A caller who lets go of
them (mx_step returns y alone) still gets that dispatch's results, whatever is allocated afterwards."""
import pytest
import torch

from gpu_util import make_router, to_dev
from paper_2602_21140_b200 import binding as B
from paper_2602_21140_b200 import workloads as W

pytestmark = pytest.mark.gpu


def _weights(P, N, K, g):
    return B.mx_quantize(torch.randn(P, N, K, device="cuda", generator=g, dtype=torch.bfloat16) * K ** -0.5)


def _reuse(router, T):
    """Tensors of the sizes that a dispatch's buffers have, so that the allocator hands freed ones on."""
    spare = []
    for _ in range(4):
        out = router.alloc_outputs(T, send_buf=False)
        for f in out.__dataclass_fields__:
            t = getattr(out, f)
            if t is not None:
                t.zero_()
        spare.append(out)
    return spare


@pytest.mark.parametrize("how", ["mx_step", "mx_dispatch", "dispatch"])
def test_buffers_outlive_the_caller(how):
    wl = W.WORKLOADS["tiny"]
    T, H, I = 64, 256, 64
    inp = W.make_inputs(wl, T=T, H=H)
    router = make_router(wl, inp, max_tokens=T, hidden=H)
    g = torch.Generator(device="cuda").manual_seed(7)
    gate_up, down = _weights(wl.P, 2 * I, H, g), _weights(wl.P, H, I, g)
    logits, x = to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16)
    dy = torch.randn(T, H, device="cuda", generator=g).bfloat16()
    buf = torch.randn(T * wl.k, H, device="cuda", generator=g).bfloat16()

    def backward():
        d_buf, d_w = router.combine_backward(buf, dy)
        return (router.combine(buf, T), d_buf, d_w, *router.dispatch_backward(logits, d_buf, d_w))

    def forward(out):
        if how == "mx_step":
            router.mx_step(logits, x, gate_up, down, out)
        else:
            getattr(router, how)(logits, x, out)

    held = router.alloc_outputs(T)
    forward(held)
    want = backward()
    forward(None)
    spare = _reuse(router, T)
    got = backward()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert router.device_status() == 0
    # a refused call changes nothing: the dispatch before it is still the latest
    with pytest.raises(B.MoeError):
        router.mx_dispatch(torch.zeros(T + 1, wl.E, device="cuda"), torch.zeros(T + 1, H, device="cuda", dtype=torch.bfloat16))
    spare += _reuse(router, T)
    for a, b in zip(backward(), want):
        assert torch.equal(a, b)
    router.close()
