"""The two variants of the products, single CTAs with narrow tiles and pairs of CTAs with wide ones, give the same
bits: a sum's order over K does not depend on the tile.  Which one runs goes by rows per slot, so the same segments
run as either one, with more empty slots or with a longer buffer."""
import numpy as np
import pytest
import torch

import mx_util as M
import test_gpu_mx_product as plain
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(12))
def test_same_bits(seed):
    rng = np.random.default_rng(seed)
    P = int(rng.integers(1, 9))
    counts = np.where(rng.random(P) < 0.5, rng.integers(1, 700, P), rng.integers(0, 40, P)).astype(np.int32)
    I, K = 32 * int(rng.integers(1, 20)), 32 * int(rng.integers(1, 80))
    N, n = 2 * I, int(counts.sum())
    if n == 0:
        counts[0] = n = 1
    narrow_P = max(P, -(-n // 64))                            # rows <= 64 * slots
    wide_rows = 64 * P + n + 1                                # rows > 64 * slots
    x = M.random_rows(wide_rows, K, seed, 2.0)
    w = plain._weights(P, N, K, seed + 9)
    results = []
    for slots, rows in ((narrow_P, n), (P, wide_rows)):
        r = plain._router(slots)
        a = plain._mx(x[:rows])
        c = np.zeros(slots, np.int32)
        c[:P] = counts
        c, o = M.segments(c)
        ww = B.MxRows(*(torch.cat([t, t[:1].expand(slots - P, *t.shape[1:])]) for t in (w.codes, w.scales)))
        for _ in range(3):
            y = r.mx_expert_product(a, plain._dev(c), plain._dev(o), ww)
            h = r.mx_expert_gated(a, plain._dev(c), plain._dev(o), ww)
            results.append((y[:n].clone(), h.codes[:n].clone(), h.scales[:n, :I // 32].clone()))
        torch.cuda.synchronize()
        assert r.device_status() == 0
        r.close()
    for got in results[1:]:
        for a, b in zip(got, results[0]):
            assert torch.equal(a, b)
