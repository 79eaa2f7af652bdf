"""Waits of the experts' products that run out: with no polls allowed a role gives up at the first poll that ends without its barrier
being complete.  The kernels return on their own, the status says so, nothing beyond the outputs is touched, and the next calls are
right again."""
import time

import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("polls", [0, 1, 3])
@pytest.mark.parametrize("counts", [[5, 0, 33, 64], [2000, 1300, 17, 2030]], ids=["short", "long"])
def test_the_products_give_up_report_and_recover(counts, polls):
    """A poll lasts up to 7800 clocks.  The gated product and the gate's gradient of long segments with a K of 64 wait for their epilogues for
    longer than that (11000 and 19000 a tile), tile after tile; of the others some may."""
    P, H, I = len(counts), 64, 4096
    r = U.make_router(P)
    n_, off, n = U.layout(counts)
    guard = 64
    a, dy = U.bf16(n, H, seed=1), U.bf16(n, H, seed=2)
    gate_up, down = U.bf16(P, 2 * I, H, seed=3, scale=H ** -0.5), U.bf16(P, H, I, seed=4, scale=I ** -0.5)
    z16 = U.bf16(n, 2 * I, seed=5)

    def rows(cols):
        return torch.full((n + 2 * guard, cols), -7.0, dtype=torch.bfloat16, device="cuda")

    def run():
        """Results, and the status behind each operator."""
        outs = h, y, dz, h2, da = [rows(c) for c in (I, H, 2 * I, I, H)]
        h, y, dz, h2, da = (o[guard:guard + n] for o in outs)
        z8, grads, status = B.mx8_empty(n, 2 * I), [], []
        calls = [lambda: r.expert_gated(a, n_, off, gate_up, h, z8), lambda: r.expert_gated_backward(dy, n_, off, down, z16, dz, h2),
                 lambda: r.expert_product(h, n_, off, down, y), lambda: r.expert_rows_backward(dz, n_, off, gate_up, da)]
        for left, right in ((dz, a), (dy, h2)):
            calls.append(lambda left=left, right=right: grads.append(r.expert_weight_backward(left, right, n_, off)))
            calls.append(lambda left=left, right=right: grads.append(r.expert_weight_backward(
                left, right, n_, off, torch.ones(P, left.shape[1], right.shape[1], device="cuda"), add=True)))
        for call in calls:
            call()
            torch.cuda.synchronize()
            status.append(r.device_status())
        return outs, grads, status

    want, want_grads, status = run()
    assert not any(status)
    assert B.moe_set_tuning(r._ctx, B.MOE_TUNE_SPIN_LIMIT, polls) == B.MOE_OK
    t0 = time.perf_counter()
    for _ in range(3):
        outs, _, status = run()
        assert all((o[:guard] == -7).all() and (o[-guard:] == -7).all() for o in outs)
        assert set(status) <= {0, B.MOE_ERR_DEVICE_TIMEOUT}
        if polls == 0 and n > 1000:
            assert status[:2] == [B.MOE_ERR_DEVICE_TIMEOUT] * 2
    assert time.perf_counter() - t0 < 10.0
    assert B.moe_set_tuning(r._ctx, B.MOE_TUNE_SPIN_LIMIT, -1) == B.MOE_OK
    got, got_grads, status = run()
    assert not any(status)
    for g, w in zip(got + got_grads, want + want_grads):
        assert torch.equal(g, w)
    r.close()


def test_a_wait_through_other_tiles_is_no_reason_to_give_up():
    """Segments that end with a whole K = 16 and one at the end that does not, with polls for single tiles (sixteen of up to 7800 clocks): the
    second CTA of a pair waits through all 23 of its tiles, of 16384 clocks each."""
    P, M, N = 48, 1024, 2304
    counts = [2048] * (P - 1) + [2041]
    r = U.make_router(P)
    assert B.moe_set_tuning(r._ctx, B.MOE_TUNE_SPIN_LIMIT, 16) == B.MOE_OK
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


@pytest.mark.parametrize("slots,rows", [(32, 40), (4, 2000)], ids=["single CTAs", "pairs"])
def test_the_products_on_4_bit_rows_give_up_and_recover(slots, rows):
    """The gated product's epilogue outlasts a poll at a K of 64; whether a wait runs out is the hardware's to say."""
    H, I = 64, 4096
    r = U.make_router(slots)
    n_, off, n = U.layout([rows] * slots)
    a = B.mx_quantize(U.bf16(n, H, seed=1))
    gate_up, down = B.mx_quantize(U.bf16(slots, 2 * I, H, seed=2, scale=H ** -0.5)), B.mx_quantize(U.bf16(slots, H, I, seed=3, scale=I ** -0.5))

    def run():
        y = torch.full((n + 128, H), -7.0, dtype=torch.bfloat16, device="cuda")
        h = r.mx_expert_gated(a, n_, off, gate_up)
        r.mx_expert_product(h, n_, off, down, y[64:64 + n])
        torch.cuda.synchronize()
        return h.codes, h.scales[:, :I // 32].clone(), y

    want = run()
    assert r.device_status() == 0
    assert B.moe_set_tuning(r._ctx, B.MOE_TUNE_SPIN_LIMIT, 0) == B.MOE_OK
    for _ in range(3):
        y = run()[2]
        assert (y[:64] == -7).all() and (y[-64:] == -7).all()
        assert r.device_status() in (0, B.MOE_ERR_DEVICE_TIMEOUT)
    assert B.moe_set_tuning(r._ctx, B.MOE_TUNE_SPIN_LIMIT, -1) == B.MOE_OK
    got = run()
    assert r.device_status() == 0 and all(torch.equal(g, w) for g, w in zip(got, want))
    r.close()
