"""Weights' gradients of segments of every length within a stage, with rows of NaN and infinity behind each: the lines between a
segment's end and a whole K = 16 count as zeros in both CTAs of a pair, in both operands, whatever the tile."""
import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stages", [0, 1, 7])
def test_every_end_of_a_segment(stages):
    counts = [64 * stages + 1 + i for i in range(64)]
    r = U.make_router(len(counts))
    n_, off, n = U.layout(counts, gap=2)
    dy, a = U.bf16(n, 264, seed=1), U.bf16(n, 328, seed=2)     # both CTAs of a pair have features and columns, in two chunks
    inside = torch.zeros(n, dtype=torch.bool, device="cuda")
    for o, c in zip(off.tolist(), counts):
        inside[o:o + c] = True
    dy[~inside] = float("nan")
    a[~inside] = float("inf")
    f32 = r.expert_weight_backward(dy, a, n_, off, dtype=torch.float32)
    b16 = r.expert_weight_backward(dy, a, n_, off)
    before = torch.ones_like(f32)
    added = r.expert_weight_backward(dy, a, n_, off, before.clone(), add=True)
    torch.cuda.synchronize()
    assert r.device_status() == 0 and torch.equal(added, f32 + before)
    for p, (o, c) in enumerate(zip(off.tolist(), counts)):
        left, right = dy[o:o + c].double(), a[o:o + c].double()
        want, bound = left.T @ right, U.sum_bound(c, left.abs().T @ right.abs())
        for got in (f32[p], b16[p]):
            half = U.HALF[got.dtype]
            U.within(got, want, (1 + half) * bound + half * want.abs())
    r.close()


def test_the_last_segment_ends_the_buffer():
    """Zeros are loaded from beyond the rows, here from behind a buffer that a segment's last line ends."""
    r = U.make_router(3)
    n_, off, n = U.layout([64, 0, 45])
    dy, a = U.bf16(n, 520, seed=1), U.bf16(n, 136, seed=2)
    got = r.expert_weight_backward(dy, a, n_, off, dtype=torch.float32)
    torch.cuda.synchronize()
    for p, o, c in ((0, 0, 64), (2, 64, 45)):
        left, right = dy[o:o + c].double(), a[o:o + c].double()
        U.within(got[p], left.T @ right, U.sum_bound(c, left.abs().T @ right.abs()) + 2.0 ** -24 * (left.T @ right).abs())
    assert not got[1].any() and r.device_status() == 0
    r.close()
