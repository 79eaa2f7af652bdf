"""Waits of the experts' products that run out: with no polls allowed each role gives up at the first look at a barrier that has not
completed.  The kernels return on their own, the status says so, nothing beyond the outputs is touched, and the next calls are
right again."""
import time

import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("polls", [0, 3, 40])
@pytest.mark.parametrize("counts", [[5, 0, 33, 64], [700, 300, 17, 1030]], ids=["short", "long"])
def test_the_products_give_up_report_and_recover(counts, polls):
    P, H, I = len(counts), 1032, 528
    r = U.make_router(P)
    n_, off, n = U.layout(counts)
    guard = 64
    a, dy = U.bf16(n, H, seed=1), U.bf16(n, H, seed=2)
    gate_up, down = U.bf16(P, 2 * I, H, seed=3, scale=H ** -0.5), U.bf16(P, H, I, seed=4, scale=I ** -0.5)

    def rows(cols):
        return torch.full((n + 2 * guard, cols), -7.0, dtype=torch.bfloat16, device="cuda")

    def step(z16, z8, outs):
        y, h, dz, h2, da = (o[guard:guard + n] for o in outs)
        r.expert_ffn(a, n_, off, gate_up, down, y, h, z8)
        r.expert_ffn(a, n_, off, gate_up, down, y, h, z16)
        r.expert_gated_backward(dy, n_, off, down, z16, dz, h2)
        r.expert_rows_backward(dz, n_, off, gate_up, da)
        return [r.expert_weight_backward(x, w, n_, off, dtype=t) for x, w in ((dz, a), (dy, h2)) for t in (torch.bfloat16, torch.float32)]

    def run():
        z16, z8, outs = rows(2 * I)[guard:guard + n], B.mx8_empty(n, 2 * I), [rows(c) for c in (H, I, 2 * I, I, H)]
        grads = step(z16, z8, outs)
        torch.cuda.synchronize()
        return z16, outs, grads

    want = run()
    assert r.device_status() == 0
    assert B.moe_set_tuning(r._ctx, B.MOE_TUNE_SPIN_LIMIT, polls) == B.MOE_OK
    t0 = time.perf_counter()
    for _ in range(3):
        _, outs, _ = run()
        assert all((o[:guard] == -7).all() and (o[-guard:] == -7).all() for o in outs)
        status = r.device_status()
        assert status in (0, B.MOE_ERR_DEVICE_TIMEOUT)
        if polls == 0:
            assert status == B.MOE_ERR_DEVICE_TIMEOUT and r.device_status() == 0
    assert time.perf_counter() - t0 < 10.0
    assert B.moe_set_tuning(r._ctx, B.MOE_TUNE_SPIN_LIMIT, -1) == B.MOE_OK
    got = run()
    assert r.device_status() == 0
    assert torch.equal(got[0], want[0])
    for g, w in zip(got[1] + got[2], want[1] + want[2]):
        assert torch.equal(g, w)
    r.close()


def test_a_wait_through_other_tiles_is_no_reason_to_give_up():
    """Segments that end with a whole K = 16 and one at the end that does not, with polls for single tiles: the second CTA of every pair
    waits through all of its tiles."""
    P, M, N = 48, 1024, 2304
    counts = [2048] * (P - 1) + [2041]
    r = U.make_router(P)
    assert B.moe_set_tuning(r._ctx, B.MOE_TUNE_SPIN_LIMIT, 4000) == B.MOE_OK
    n_, off, n = U.layout(counts)
    dy, a = U.bf16(n, M, seed=1), U.bf16(n, N, seed=2)
    got = [r.expert_weight_backward(dy, a, n_, off, dtype=t) for t in (torch.float32, torch.bfloat16)]
    torch.cuda.synchronize()
    assert r.device_status() == 0
    for p in (0, P - 2, P - 1):
        s = slice(2048 * p, 2048 * p + counts[p])
        left, right = dy[s].double(), a[s].double()
        want, bound = left.T @ right, U.sum_bound(counts[p], left.abs().T @ right.abs())
        for g in got:
            U.within(g[p], want, (1 + U.HALF[g.dtype]) * bound + U.HALF[g.dtype] * want.abs())
    r.close()
