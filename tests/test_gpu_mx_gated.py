"""The gated product's stores: rows outside every segment, segments that leave the buffer, guard zones, NaN and
overflow.  Its epilogue shares nothing with the plain product's.  Values are bracketed as in test_gpu_mx_product."""
import numpy as np
import pytest
import torch

import mx_util as M
import test_gpu_mx_product as plain
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu
FILL = 0xAB


def _out(rows, I):
    """h inside larger buffers: (MxRows, the two whole buffers)."""
    c = torch.full((rows * I // 2 + 64,), FILL, dtype=torch.uint8, device="cuda")
    s = torch.full((rows * M.pitch(I) + 64,), FILL, dtype=torch.uint8, device="cuda")
    return B.MxRows(c[32:-32].view(rows, I // 2), s[32:-32].view(rows, M.pitch(I))), (c, s)


def _check(h, whole, a, w, counts, offsets, I):
    """Values of the rows that a slot owns; everything else as it was, the padding of the scales too."""
    rows, K = a.codes.shape[0], a.cols
    want, mag = (t.cpu().numpy() for t in plain._sums(plain._vals(a), plain._vals(w), counts, offsets, rows))
    own = ~np.isnan(want[:, 0])
    codes, scales = h.codes.cpu().numpy(), h.scales.cpu().numpy()
    assert (codes[~own] == FILL).all() and (scales[~own] == FILL).all() and (scales[:, I // 32:] == FILL).all()
    for t in whole:
        assert (t[:32] == FILL).all() and (t[-32:] == FILL).all()
    g, u = want[own, 0::2], want[own, 1::2]
    e = ((K / 64 + 64) * 2.0 ** -23 * mag)[own]
    silu = g / (1 + np.exp(-g))
    v = silu * u
    # as in test_gpu_mx_product.test_gated
    tol = 1.1 * e[:, 0::2] * (np.abs(u) + e[:, 1::2]) + np.abs(silu) * e[:, 1::2] + (8 + np.abs(g)) * 2.0 ** -23 * np.abs(v)
    sb = scales[own][:, :I // 32].astype(np.int64)
    got = M.values(codes[own], scales[own])
    assert (got >= M.values(*plain._pack(M.round_codes(v - tol, sb), sb))).all()
    assert (got <= M.values(*plain._pack(M.round_codes(v + tol, sb), sb))).all()
    amax, t = np.abs(v).reshape(len(v), -1, 32), tol.reshape(len(v), -1, 32)
    assert (sb >= M.scale_bytes(np.maximum(amax - t, 0).reshape(len(v), I))).all()
    assert (sb <= M.scale_bytes((amax + t).reshape(len(v), I))).all()
    return own


@pytest.mark.parametrize("seed", range(8))
def test_any_order_with_gaps(seed):
    rng = np.random.default_rng(seed)
    P = int(rng.integers(2, 12))
    long = seed % 2 == 0                                      # the wide variant, or the narrow one
    counts = np.where(rng.random(P) < 0.3, rng.integers(225, 700, P) if long else rng.integers(0, 60, P), rng.integers(0, 150 if long else 30, P))
    counts = counts.astype(np.int32)
    I, K = 32 * int(rng.integers(1, 12)), 32 * int(rng.integers(1, 24))
    offsets, at = np.zeros(P + 1, np.int32), 0
    for p in rng.permutation(P):
        at += int(rng.integers(0, 40))
        offsets[p] = at
        at += counts[p]
    n = at + int(rng.integers(1, 50))
    r = plain._router(P)
    a, w = plain._mx(M.random_rows(n, K, seed, 1.0)), plain._weights(P, 2 * I, K, seed + 50)
    h, whole = _out(n, I)
    r.mx_expert_gated(a, plain._dev(counts), plain._dev(offsets), w, h)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    own = _check(h, whole, a, w, counts, offsets, I)
    assert own.sum() == counts.sum()
    r.close()


@pytest.mark.parametrize("scale", [1, 9])
def test_segments_that_leave_the_buffer_are_cut(scale):
    P, I, K, rows = 6, 96, 64, 50 * scale
    r = plain._router(P)
    a, w = plain._mx(M.random_rows(rows, K, 3)), plain._weights(P, 2 * I, K, 4)
    h, whole = _out(rows, I)
    counts, offsets = [10, -5, 2 ** 31 - 1, 7, 3, 2 ** 31 - 1], [0, 3, 20, -4, 2 ** 31 - 1, rows]
    r.mx_expert_gated(a, plain._dev(counts), plain._dev(offsets), w, h)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    own = _check(h, whole, a, w, [10, 0, rows - 20], [0, 0, 20], I)
    assert own.sum() == rows - 10
    r.close()


def test_segments_that_overlap_stay_inside():
    P, I, K, rows = 40, 64, 64, 300
    r = plain._router(P)
    a, w = plain._mx(M.random_rows(rows, K, 3)), plain._weights(P, 2 * I, K, 4)
    h, whole = _out(rows, I)
    r.mx_expert_gated(a, plain._dev([2 ** 31 - 1] * P), plain._dev([0] * P), w, h)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    for t in whole:
        assert (t[:32] == FILL).all() and (t[-32:] == FILL).all()
    r.close()


@pytest.mark.parametrize("n", [20, 64, 230, 700])
def test_nan_stays_in_its_row_and_in_its_feature(n):
    """A NaN block of a row, of a gate and of an up-projection, among other rows and features of the same tiles (of one
    CTA up to 64 rows a slot, of a pair beyond).  Everything else keeps its bits."""
    I, K = 160, 544
    r = plain._router(1)
    c, o = M.segments([n])
    x, wx = M.random_rows(n, K, n), M.random_rows(2 * I, K, 7).reshape(1, 2 * I, K) * K ** -0.5

    def run(x, wx):
        a, w = plain._mx(x), plain._mx(wx)
        h = r.mx_expert_gated(a, plain._dev(c), plain._dev(o), w)
        y = r.mx_expert_product(a, plain._dev(c), plain._dev(o), w)
        torch.cuda.synchronize()
        assert r.device_status() == 0
        return h.codes.clone(), h.scales[:, :I // 32].clone(), y

    codes, scales, y = run(x, wx)
    assert (scales != 255).all() and torch.isfinite(y).all()
    bad_rows = sorted({0, n // 2, n - 1})
    bx = x.copy()
    for i, t in enumerate(bad_rows):
        bx[t, (40, 300, K - 1)[i % 3]] = (np.nan, np.inf, -np.inf)[i % 3]
    got_c, got_s, got_y = run(bx, wx)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[bad_rows] = False
    assert (got_s[~keep] == 255).all() and (got_c[~keep] == 0).all() and torch.isnan(got_y[~keep]).all()
    assert torch.equal(got_s[keep], scales[keep]) and torch.equal(got_c[keep], codes[keep]) and torch.equal(got_y[keep], y[keep])
    bw = wx.copy()
    bw[0, 2 * 37, 33] = np.inf                                # gate of feature 37 (block 1)
    bw[0, 2 * 130 + 1, K - 2] = np.nan                        # up-projection of feature 130 (block 4)
    got_c, got_s, got_y = run(x, bw)
    blocks = torch.tensor([b not in (1, 4) for b in range(I // 32)], device="cuda")
    assert (got_s[:, ~blocks] == 255).all() and torch.equal(got_s[:, blocks], scales[:, blocks])
    per_block = lambda t: t.view(n, I // 32, 16)              # noqa: E731
    assert (per_block(got_c)[:, ~blocks] == 0).all() and torch.equal(per_block(got_c)[:, blocks], per_block(codes)[:, blocks])
    nan = torch.isnan(got_y)
    assert nan[:, [74, 261]].all() and nan.sum() == 2 * n
    assert torch.equal(got_y[~nan], y[~nan])
    r.close()


@pytest.mark.parametrize("n", [3, 200])
def test_overflow_and_saturated_gates(n):
    """Gates and up-projections at the ends of fp32: an infinite product makes its block NaN, a far negative gate gives
    zeros, a far positive one the product itself."""
    K, I = 32, 64
    r = plain._router(1)
    c, o = M.segments([n])
    codes = torch.full((n, K // 2), 0x11 * 2, dtype=torch.uint8, device="cuda")            # ones
    scales = torch.full((n, 16), 127, dtype=torch.uint8, device="cuda")
    w_codes = np.zeros((1, 2 * I, K), np.float64)
    w_codes[0, 0::2, 0], w_codes[0, 1::2, 0] = 1.0, 1.0                                  # one term each: sums are exact
    big = 2.0 ** 70
    w_codes[0, 0, 0], w_codes[0, 1, 0] = big, big                                        # feature 0: 2^140 overflows
    w_codes[0, 2 * 32:, 0] = 2.0 ** 60                                                   # block 1: 2^120 everywhere ...
    w_codes[0, 2 * 40, 0] = -2.0 ** 60                                                   # ... but a gate far below zero
    w_codes[0, 2 * 41, 0] = 0.0                                                          # ... and one at zero
    h = r.mx_expert_gated(B.MxRows(codes, scales), plain._dev(c), plain._dev(o), plain._mx(w_codes))
    torch.cuda.synchronize()
    v = M.values(h.codes.cpu().numpy(), h.scales.cpu().numpy())
    assert np.isnan(v[:, :32]).all() and (h.scales[:, 0] == 255).all()
    want = np.full(32, 2.0 ** 120)
    want[[8, 9]] = 0.0
    assert (v[:, 32:] == want).all()
    assert r.device_status() == 0
    r.close()
