"""A norm's output object used again with and without a residual: the rows that callers gave stay as they were."""
import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_earlier_calls_stay(dtype):
    x, x2, res = (U.bf16(37, 256, seed=s).to(dtype) for s in range(3))
    was = [t.clone() for t in (x, x2, res)]
    w = torch.ones(256, device="cuda")
    want = [B.rms_norm(a, w, r, keep=True) for a, r in ((x, None), (x2, res), (x2, None), (x, res))]
    out = B.rms_norm(x, w, keep=True)
    got = [(out.y.clone(), out.h.clone())]
    for a, r in ((x2, res), (x2, None), (x, res)):
        assert B.rms_norm(a, w, r, keep=True, out=out) is out
        got.append((out.y.clone(), out.h.clone()))
    torch.cuda.synchronize()
    for t, before in zip((x, x2, res), was):
        assert torch.equal(t, before)
    for (y, h), o in zip(got, want):
        assert torch.equal(y, o.y) and torch.equal(h, o.h)


def test_h_in_the_residuals_place():
    """As the caller says, also where the residual was the x of the call before."""
    stream, branch, w = U.bf16(37, 256, seed=1), U.bf16(37, 256, seed=2), torch.ones(256, device="cuda")
    want = (stream.float() + branch.float()).bfloat16()
    out = B.rms_norm(stream, w)
    out.h = stream
    B.rms_norm(branch, w, stream, out=out)
    torch.cuda.synchronize()
    assert out.h is stream and torch.equal(stream, want)
