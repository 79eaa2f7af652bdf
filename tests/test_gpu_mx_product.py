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
    cfg = B.make_config(min(E, 512), k, 64, 16, P, 1, 8)          # P ranks of one slot
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


@pytest.mark.parametrize("P", [1024, 1025, 1536])
def test_many_slots(P):
    """Around the number of slots up to which the kernel keeps its full tables, most of them empty."""
    counts = np.zeros(P, np.int32)
    rng = np.random.default_rng(P)
    counts[rng.choice(P, 40, replace=False)] = rng.integers(1, 9, 40)
    counts[P - 1], counts[0], counts[P // 2] = 70, 0, 230
    N, K = 136, 96
    r = _router(P)
    n = int(counts.sum())
    a, w = _mx(M.random_rows(n, K, 1)), _weights(P, N, K, 2)
    c, o = M.segments(counts)
    y = r.mx_expert_product(a, _dev(c), _dev(o), w)
    want, mag = _sums(_vals(a), _vals(w), c, o, n)
    assert ((y.double() - want).abs() <= (K / 64 + 64) * 2.0 ** -23 * mag + 2.0 ** -8 * want.abs()).all()
    # the same rows in few slots' worth of the wide kernel: many rows a slot on average
    big = np.zeros(P, np.int32)
    big[[3, P - 2]] = [32 * P, 33 * P + 7]
    c, o = M.segments(big)
    n = int(big.sum())
    a = _mx(M.random_rows(n, K, 3))
    y = r.mx_expert_product(a, _dev(c), _dev(o), w)
    want, mag = _sums(_vals(a), _vals(w), c, o, n)
    assert ((y.double() - want).abs() <= (K / 64 + 64) * 2.0 ** -23 * mag + 2.0 ** -8 * want.abs()).all()
    assert r.device_status() == 0
    r.close()


@pytest.mark.parametrize("seed", range(6))
def test_skewed_slots_in_any_order(seed):
    """A few slots with many row tiles among slots with one or none, laid out in a random order with gaps."""
    rng = np.random.default_rng(seed)
    P = int(rng.integers(2, 14))
    counts = np.where(rng.random(P) < 0.3, rng.integers(225, 1500, P), rng.integers(0, 200, P)).astype(np.int32)
    N, K = int(rng.integers(1, 60)) * 8, int(rng.integers(1, 40)) * 32
    order = rng.permutation(P)
    offsets, at = np.zeros(P + 1, np.int32), 0
    for p in order:
        at += int(rng.integers(0, 40))
        offsets[p] = at
        at += counts[p]
    n = at + int(rng.integers(0, 50))
    r = _router(P)
    a, w = _mx(M.random_rows(n, K, seed, 1.0)), _weights(P, N, K, seed + 50)
    y = torch.full((n, N), -7.0, dtype=torch.bfloat16, device="cuda")
    r.mx_expert_product(a, _dev(counts), _dev(offsets), w, y)
    want, mag = _sums(_vals(a), _vals(w), counts, offsets, n)
    own = ~torch.isnan(want[:, 0])
    assert (y[~own] == -7).all()
    tol = (K / 64 + 64) * 2.0 ** -23 * mag + 2.0 ** -8 * want.abs()
    assert ((y.double() - want).abs() <= tol)[own].all()
    assert r.device_status() == 0
    r.close()


def test_refusals():
    r = _router(2)
    a, w, z = _mx(M.random_rows(4, 64, 1)), _weights(2, 128, 64, 1), _dev([2, 2])
    o = _dev([0, 2, 4])
    ok = lambda **k: r.mx_expert_product(**{**dict(rows=a, slot_counts=z, slot_offsets=o, weight=w), **k})   # noqa: E731
    ok()
    for bad in (dict(weight=_weights(3, 128, 64, 1)), dict(weight=_weights(2, 128, 32, 1)), dict(weight=_weights(2, 132, 64, 1)),
                dict(slot_counts=z.long()), dict(slot_counts=_dev([1, 1, 2])), dict(slot_offsets=o[:1]), dict(slot_counts=z.cpu()),
                dict(rows=B.MxRows(a.codes[:, :16], a.scales)), dict(rows=B.MxRows(a.codes, a.scales[:3])),
                dict(rows=B.MxRows(a.codes.float(), a.scales)), dict(y=torch.empty(4, 120, dtype=torch.bfloat16, device="cuda")),
                dict(y=torch.empty(4, 128, device="cuda"))):
        with pytest.raises(B.MoeError):
            ok(**bad)
    with pytest.raises(B.MoeError):                                   # gate and up rows come in pairs of 32 features
        r.mx_expert_gated(a, z, o, _weights(2, 96, 64, 1))
    p = a.codes.data_ptr()
    args = [r._ctx, p, a.scales.data_ptr(), 4, z.data_ptr(), o.data_ptr(), w.codes.data_ptr(), w.scales.data_ptr(), 128, 64, p]
    for i, v in ((1, p + 8), (2, 0), (3, -1), (4, 0), (5, 0), (6, p + 1), (7, 0), (8, 0), (8, 12), (9, 16), (10, p + 4), (10, 0)):
        bad = list(args)
        bad[i] = v
        assert B.moe_mx_expert_product(*bad) == B.MOE_ERR_INVALID_ARG, i
    args[3] = (1 << 30) + 1                                           # more rows than the call takes
    assert B.moe_mx_expert_product(*args) == B.MOE_ERR_CAPACITY
    torch.cuda.synchronize()
    r.close()


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


def test_segments_that_overlap_stay_inside():
    """Not a dispatch's output, but it must not reach outside of y: every slot claims every row."""
    P, N, K, rows = 40, 128, 64, 300
    r = _router(P)
    a, w = _mx(M.random_rows(rows, K, 3)), _weights(P, N, K, 4)
    guard = torch.full((rows + 64, N), -7.0, dtype=torch.bfloat16, device="cuda")
    r.mx_expert_product(a, _dev([2 ** 31 - 1] * P), _dev([0] * P), w, guard[32:32 + rows])
    torch.cuda.synchronize()
    assert r.device_status() == 0
    assert (guard[:32] == -7).all() and (guard[32 + rows:] == -7).all()
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
