"""The experts' products on 4-bit rows against 64-bit products of the values that the rows stand for.

Bound of an accumulated sum: products of two 4-bit values with power-of-two scales are exact in fp32.
The tensor core adds 64 of them at a time to an fp32 accumulator; each of those K/64 additions, and the
at most 64 alignments inside one, loses at most one unit in the last place of fp32 (2^-23, truncation
allowed for) of the sum of magnitudes S = sum |a w|:  |error| <= (K/64 + 64) * 2^-23 * S.
A bf16 output adds half a step, 2^-8 of its value (2^-8 is a whole half-step bound for bf16's 8 bits)."""
import numpy as np
import pytest
import torch

import mx_util as M
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu


def _router(P, k=1):
    E = P
    cfg = B.make_config(min(E, 512), k, 64, 16, 1 if P <= 512 else P // 512, P if P <= 512 else 512, 8)
    return B.MoeRouter(cfg, [p % cfg.num_experts for p in range(P)], None, [1.0] * P)


def _mx(x64):
    c, s = M.quantize(x64)
    s = s.copy()
    s[..., x64.shape[-1] // 32:] = 0xEE              # the padding is never interpreted
    return B.MxRows(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda())


def _weights(P, N, K, seed):
    return _mx(M.random_rows(P * N, K, seed, 1.0).reshape(P, N, K) * K ** -0.5)


def _vals(m):
    return torch.from_numpy(M.values(m.codes.cpu().numpy(), m.scales.cpu().numpy())).cuda()


def _sums(a, w, counts, offsets, rows):
    """(sum a w, sum |a| |w|) of every row with its slot's matrix, f64; NaN where no slot owns the row."""
    out = torch.full((rows, w.shape[1]), float("nan"), dtype=torch.float64, device="cuda")
    mag = out.clone()
    for p, c in enumerate(counts):
        r = slice(int(offsets[p]), int(offsets[p]) + int(c))
        out[r] = a[r] @ w[p].T
        mag[r] = a[r].abs() @ w[p].abs().T
    return out, mag


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


CASES = [
    # counts, N, K
    ([1], 128, 256), ([1], 8, 32), ([5], 128, 256), ([16], 256, 512), ([33], 136, 288), ([0, 7, 0, 1], 128, 64),
    ([64], 128, 1024), ([65, 63], 264, 320), ([129], 128, 256), ([200, 0, 31], 128, 768), ([300, 17], 384, 1056),
    ([450, 1, 230], 512, 2048), ([1] * 40, 256, 7168), ([2, 0] * 30, 512, 544), ([700], 1000, 4096),
]


@pytest.mark.parametrize("counts,N,K", CASES)
def test_product(counts, N, K):
    P, n = len(counts), sum(counts)
    r = _router(P)
    a = _mx(M.random_rows(n, K, n + K, 2.0))
    w = _weights(P, N, K, N + K)
    c, o = M.segments(counts)
    y = r.mx_expert_product(a, _dev(c), _dev(o), w)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    want, mag = _sums(_vals(a), _vals(w), c, o, n)
    err = (y.double() - want).abs()
    tol = (K / 64 + 64) * 2.0 ** -23 * mag + 2.0 ** -8 * want.abs()
    assert (err <= tol).all(), f"{(err > tol).sum()} of {err.numel()} outside, worst {(err / tol).max()}"
    r.close()


@pytest.mark.parametrize("counts,I,K", [([1], 32, 32), ([3, 0, 9], 64, 256), ([31], 96, 288), ([130, 2], 160, 1024),
                                        ([0, 257, 30], 256, 512), ([1] * 33, 128, 2048), ([225], 64, 7168)])
def test_gated(counts, I, K):
    P, n = len(counts), sum(counts)
    r = _router(P)
    a = _mx(M.random_rows(n, K, n + K, 1.0))
    w = _weights(P, 2 * I, K, I + K)
    c, o = M.segments(counts)
    h = r.mx_expert_gated(a, _dev(c), _dev(o), w)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    s, mag = (t.cpu().numpy() for t in _sums(_vals(a), _vals(w), c, o, n))
    g, u = s[:, 0::2], s[:, 1::2]
    e = (K / 64 + 64) * 2.0 ** -23 * mag
    silu = g / (1 + np.exp(-g))
    want = silu * u
    # |silu'| <= 1.1; exp, the division and the product in fp32 add (8 + |g|) units of 2^-23 of the value
    tol = 1.1 * e[:, 0::2] * (np.abs(u) + e[:, 1::2]) + np.abs(silu) * e[:, 1::2] + (8 + np.abs(g)) * 2.0 ** -23 * np.abs(want)
    got = M.values(h.codes.cpu().numpy(), h.scales.cpu().numpy())
    sb = h.scales.cpu().numpy()[:, :I // 32].astype(np.int64)
    # rounding is monotonic: under the scale that was chosen, the value lies between those of want -+ tol,
    # and the scale between those of the largest magnitude -+ tol
    lo = M.values(*_pack(M.round_codes(want - tol, sb), sb))
    hi = M.values(*_pack(M.round_codes(want + tol, sb), sb))
    assert ((got >= lo) & (got <= hi)).all()
    amax = np.abs(want).reshape(n, -1, 32)
    t = tol.reshape(n, -1, 32)
    s_lo = M.scale_bytes(np.maximum(amax - t, 0).reshape(n, I))
    s_hi = M.scale_bytes((amax + t).reshape(n, I))
    assert ((sb >= s_lo) & (sb <= s_hi)).all()
    r.close()


def _pack(codes, sb):
    packed = (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)
    s = np.zeros((*codes.shape[:-1], M.pitch(codes.shape[-1])), np.uint8)
    s[..., :sb.shape[-1]] = sb
    return packed, s


def test_rows_outside_segments_stay():
    """Gaps between segments, slots in another order, and rows behind the last segment."""
    P, N, K, rows = 4, 136, 256, 200
    r = _router(P)
    a, w = _mx(M.random_rows(rows, K, 1)), _weights(P, N, K, 2)
    counts, offsets = _dev([40, 0, 3, 70]), _dev([120, 0, 5, 17])
    y = torch.full((rows, N), -7.0, dtype=torch.bfloat16, device="cuda")
    r.mx_expert_product(a, counts, offsets, w, y)
    want, mag = _sums(_vals(a), _vals(w), [40, 0, 3, 70], [120, 0, 5, 17], rows)
    own = ~torch.isnan(want[:, 0])
    assert own.sum() == 113 and (y[~own] == -7).all()
    tol = (K / 64 + 64) * 2.0 ** -23 * mag + 2.0 ** -8 * want.abs()
    assert ((y.double() - want).abs() <= tol)[own].all()
    r.close()


def test_segments_that_leave_the_buffer_are_cut():
    P, N, K, rows = 6, 128, 64, 50
    r = _router(P)
    a, w = _mx(M.random_rows(rows, K, 3)), _weights(P, N, K, 4)
    guard = torch.full((rows + 64, N), -7.0, dtype=torch.bfloat16, device="cuda")
    y = guard[32:32 + rows]
    counts, offsets = _dev([10, -5, 100, 7, 3, 2 ** 31 - 1]), _dev([0, 3, 20, -4, 2 ** 31 - 1, 50])
    r.mx_expert_product(a, counts, offsets, w, y)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    assert (guard[:32] == -7).all() and (guard[32 + rows:] == -7).all() and (y[10:20] == -7).all()
    want, mag = _sums(_vals(a), _vals(w), [10, 0, 30], [0, 0, 20], rows)
    own = ~torch.isnan(want[:, 0])
    tol = (K / 64 + 64) * 2.0 ** -23 * mag + 2.0 ** -8 * want.abs()
    assert ((y.double() - want).abs() <= tol)[own].all()
    r.close()


def test_nan_scales_stay_in_their_row():
    """A row with a NaN block gives NaN; its neighbours in the same tile do not notice."""
    P, N, K, n = 1, 128, 512, 20
    r = _router(P)
    x = M.random_rows(n, K, 5)
    x[7, 300] = np.inf
    a, w = _mx(x), _weights(P, N, K, 6)
    c, o = M.segments([n])
    y = r.mx_expert_product(a, _dev(c), _dev(o), w)
    assert torch.isnan(y[7]).all()
    y[7] = 0
    assert torch.isfinite(y).all()
    r.close()


def test_no_rows_and_empty_slots():
    r = _router(3)
    w = _weights(3, 128, 64, 1)
    z = _dev([0, 0, 0])
    assert r.mx_expert_product(B.mx_empty(0, 64), z, z, w).shape == (0, 128)
    y = torch.full((5, 128), -7.0, dtype=torch.bfloat16, device="cuda")
    r.mx_expert_product(_mx(M.random_rows(5, 64, 1)), z, z, w, y)
    torch.cuda.synchronize()
    assert (y == -7).all() and r.device_status() == 0
    r.close()
