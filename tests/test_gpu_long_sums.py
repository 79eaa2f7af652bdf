"""Long sums of one sign, whose errors add up: what the accumulators of a limited length are for.

A tensor core adds the 16 products of a step to the accumulator and cuts the sum off to 24 bits: less than one unit in the last place, at most
2^-23 of what the sum has reached.  (Products 2^10 and more below the sum lose bits of their own besides; pieces of up to 1024 products
end where that sets in.)  A piece of n steps of like size is off by at most (n + 1) / 2 * 2^-23 of itself then, and adding up q pieces in fp32
adds at most (q + 1) / 2 * 2^-24."""
import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


def _off(steps, pieces):
    return (steps + 1) / 2 * 2.0 ** -23 + ((pieces + 1) / 2 * 2.0 ** -24 if pieces > 1 else 0.0)


def _of_one_sign(rows, cols, seed):
    """Positive, of rows whose sizes differ by up to four times."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, device="cuda", generator=g).abs()
    return (x * torch.exp2(2 * torch.rand(rows, 1, device="cuda", generator=g))).bfloat16()


@pytest.mark.parametrize("rows", [900, 20000, 65000])
def test_fp32_gradients(rows):
    """Pieces of 960 rows at most.  (In one accumulator 20000 rows are off by 1e-4.)"""
    r = U.make_router(1)
    n_, off, n = U.layout([rows])
    dy, a = U.bf16(n, 264, seed=1).abs(), U.bf16(n, 328, seed=2).abs()
    got = r.expert_weight_backward(dy, a, n_, off, dtype=torch.float32)[0].double()
    want = dy.double().T @ a.double()
    assert r.device_status() == 0
    assert float(((got - want).abs() / want).max()) <= _off(60, -(-rows // 960))
    r.close()


@pytest.mark.parametrize("K", [1024, 7168, 16384])
def test_codes_of_kept_sums(K):
    """Pieces of 1024.  A code falls the other way where its sum, off by d of itself, crosses a boundary: these are 2^-3 of a binade apart, so at
    most 16 d of the codes do.  (In one accumulator the scales of K = 7168 are already off by more than such a d.)"""
    m, cols = 2048, 2048
    r = U.make_router(1)
    n_, off, n = U.layout([m])
    a, w = _of_one_sign(m, K, 3), (_of_one_sign(cols, K, 4).float() * K ** -0.5).bfloat16()
    z = B.mx8_empty(n, cols)
    r.expert_gated(a, n_, off, w[None].contiguous(), z=z)
    v = (a.double() @ w.double().T).unflatten(-1, (-1, 32))
    assert r.device_status() == 0
    d = _off(64, -(-K // 1024))
    scale = torch.exp2(z.scales[:, :cols // 32].double() - 127)[..., None]
    q = v / scale
    assert (q <= 448 * (1 + d)).all() and (q.amax(-1) > 224 * (1 - d)).all()
    step = torch.exp2(torch.floor(torch.log2(q.clamp(min=2.0 ** -6))) - 3)
    want = (torch.round(q / step) * step * scale).flatten(-2)
    off_codes = int((U.values8(z) != want).sum())
    most = 16 * d * v.numel()
    assert off_codes <= most + 6 * most ** 0.5, off_codes
    r.close()
