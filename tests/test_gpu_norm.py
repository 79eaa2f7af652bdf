"""The norm with the residual's addition, its 8-bit output and its gradient against the formulas in 64 bits."""
import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu

# rows x columns: a lane, a warp with one, two and four units, a CTA from 64 threads to 512, one row and more than a wave
SIZES = [(1, 8), (3, 32), (9, 264), (17, 520), (300, 1024), (5, 1032), (1, 7168), (700, 2080), (37, 4096), (3, 8200), (2, 16384), (2500, 96)]
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _rows(rows, cols, dtype, seed, stride=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols if stride is None else stride, device="cuda", generator=g)
    x *= torch.exp2(torch.randint(-6, 7, (rows, 1), device="cuda", generator=g).float())
    return x.to(dtype)[:, :cols]


def _weight(cols, dtype, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (1 + 0.3 * torch.randn(cols, device="cuda", generator=g)).to(dtype)


# Sums: a thread adds at most 4 units of 8 in turn, then trees of 5 and of at most 4 levels, then the division and a root or a
# product: 48 roundings of 2^-24 are more than any of them takes.
SUM = 48 * 2.0 ** -24


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype):
    half = U.HALF[dtype]
    for residual, wtype, strided in ((True, dtype, False), (False, torch.float32, True), (True, torch.bfloat16, True), (False, torch.float16, False)):
        stride = cols + 24 if strided else None
        x = _rows(rows, cols, dtype, 1, stride)
        res = _rows(rows, cols, dtype, 2, stride) if residual else None
        w, keep = _weight(cols, wtype), cols % 32 == 0
        out = B.rms_norm(x, w, res, 1e-5, keep=keep)
        torch.cuda.synchronize()
        if residual:
            assert torch.equal(out.h, (x.float() + res.float()).to(dtype))      # one rounding
        else:
            assert out.h is x
        h = out.h.double()
        rstd = 1 / torch.sqrt(h.square().mean(1) + 1e-5)
        U.within(out.rstd, rstd, SUM * rstd)
        y = h * rstd[:, None] * w.double()
        off = (SUM + 2.0 ** -22) * y.abs()
        tiny = 2.0 ** -25 if dtype is torch.float16 else 2.0 ** -134            # half a subnormal step
        U.within(out.y, y, half * y.abs() + (1 + half) * off + tiny)
        if keep:
            U.check8(out.y8, y, off)
            assert (out.y8.scales[:, cols // 32:] == 0).all()
            again = B.rms_norm(x, w, res, 1e-5, keep=True, out=out)             # into the same buffers
            assert again is out
        if rows > 1:                                                           # rows do not depend on their number
            one = B.rms_norm(x[1:2], w, None if res is None else res[1:2], 1e-5)
            assert torch.equal(one.y[0], out.y[1])


def test_eight_bit_values():
    """Every code under many scales, in all types, against its bits."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(4, 1).contiguous()
    scales = torch.zeros(4, 16, dtype=torch.uint8, device="cuda")
    scales[:, :8] = torch.tensor([[0, 1, 100, 127, 128, 140, 200, 255], [120, 121, 122, 123, 124, 125, 126, 127],
                                  [110, 112, 118, 119, 130, 133, 134, 135], [126, 127, 128, 60, 50, 40, 30, 246]], dtype=torch.uint8)
    m = B.Mx8Rows(codes, scales)
    want = U.values8(m)
    for dtype in (torch.float32, torch.bfloat16):
        # exact where the type has the number: scales 0 and 1 leave multiples of 2^-136, and a bf16 is one of 2^-133
        got = B.mx8_dequantize(m, dtype)
        steps = want * 2.0 ** (149 if dtype is torch.float32 else 133)
        fine = torch.isfinite(want) & (steps == steps.round())
        assert fine.float().mean() > 0.9
        assert torch.equal(got.double()[fine], want[fine]) and torch.isnan(got[torch.isnan(want)]).all()
    got = B.mx8_dequantize(m, torch.float16).double()
    fine = want.abs() <= 65504
    assert ((got - want).abs()[fine] <= (2.0 ** -11 * want.abs() + 2.0 ** -25)[fine]).all()
    wide = torch.full((4, 320), -7.0, device="cuda")
    B.mx8_dequantize(m, torch.float32, wide[:, 8:264])
    assert torch.equal(wide[:, 8:264][torch.isfinite(want)], B.mx8_dequantize(m, torch.float32)[torch.isfinite(want)])
    assert (wide[:, :8] == -7).all() and (wide[:, 264:] == -7).all()


def test_rows_that_are_not_numbers():
    """Zeros, an infinity and a NaN stay in their rows; eps = 0 of a row of zeros is 0 * inf, as the formula has it."""
    x = torch.randn(6, 64, device="cuda").bfloat16()
    x[1] = 0
    x[2, 5], x[3, 40] = float("inf"), float("nan")
    w = torch.ones(64, device="cuda").bfloat16()
    out = B.rms_norm(x, w, keep=True)
    torch.cuda.synchronize()
    assert (out.y[1] == 0).all() and (out.y8.codes[1] == 0).all() and (out.y8.scales[1] == 0).all()
    assert torch.isnan(out.y[3]).all() and (out.y8.scales[3, :2] == 255).all()
    # 1 / sqrt(inf) = 0: zeros, and 0 * inf where the infinity stands
    assert torch.isnan(out.y[2, 5]) and (out.y[2, :5] == 0).all() and out.y8.scales[2, 0] == 255 and out.y8.scales[2, 1] == 0
    assert torch.isfinite(out.y[[0, 4, 5]]).all() and torch.isfinite(B.mx8_dequantize(out.y8)[[0, 4, 5]]).all()
    assert torch.isnan(B.rms_norm(x, w, eps=0.0).y[1]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(rows, cols, dtype):
    half = U.HALF[dtype]
    h, w = _rows(rows, cols, dtype, 1), _weight(cols, TYPES[rows % 3])
    h = h.contiguous()
    rstd = torch.rsqrt(h.double().square().mean(1) + 1e-5).float()
    dy, dh = (torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(s)).to(dtype) for s in (5, 6))
    n, r = h.double() * rstd.double()[:, None], rstd.double()[:, None]
    g = dy.double() * w.double()
    mean = (g * n).mean(1, keepdim=True)
    for past in (dh, None):
        dx, dw = B.rms_norm_backward(dy, h, rstd, w, past)
        torch.cuda.synchronize()
        want = r * (g - n * mean) + (0 if past is None else past.double())
        # the mean's sum, and six roundings of the terms
        bound = r * (n.abs() * (g * n).abs().mean(1, keepdim=True) * SUM + 6 * 2.0 ** -24 * (g.abs() + (n * mean).abs()))
        U.within(dx, want, (1 + half) * (bound + 2.0 ** -24 * want.abs()) + half * want.abs() + (2.0 ** -25 if dtype is torch.float16 else 0))
        # a CTA adds its rows (at most rows / 148 + 1, or eight times as many in warps), then trees of up to 8 + 28 + 32
        terms = dy.double() * n
        U.within(dw, terms.sum(0), (rows / 148 + 72) * 2.0 ** -24 * terms.abs().sum(0))
        again = B.rms_norm_backward(dy, h, rstd, w, past)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
        for t in (dy, h) + (() if past is None else (past,)):                   # in the place of an input
            bufs = {id(t): t.clone()}
            at = lambda v: bufs.get(id(v), v)                                  # noqa: E731
            got = B.rms_norm_backward(at(dy), at(h), rstd, w, None if past is None else at(past), dx=bufs[id(t)])
            assert torch.equal(got[0], dx) and torch.equal(got[1], dw)


def test_gradient_against_differences():
    """The forward formula in 64 bits, differentiated numerically along random directions."""
    rows, cols = 6, 1056
    h, w = _rows(rows, cols, torch.float32, 1).contiguous(), _weight(cols, torch.float32)
    dy, dh = torch.randn(rows, cols, device="cuda"), torch.randn(rows, cols, device="cuda")
    out = B.rms_norm(h, w)
    dx, dw = B.rms_norm_backward(dy, h, out.rstd, w, dh)

    def loss(h_, w_):
        return (h_ / torch.sqrt(h_.square().mean(1, keepdim=True) + 1e-6) * w_ * dy.double()).sum() + (h_ * dh.double()).sum()

    h64, w64, e = h.double(), w.double(), 2.0 ** -20
    for s in range(4):
        g = torch.Generator(device="cuda").manual_seed(s)
        u, v = (torch.randn(t.shape, device="cuda", generator=g, dtype=torch.float64) for t in (h, w))
        u *= h64.abs().mean(1, keepdim=True)
        for got, diff, size in (((u * dx).sum(), (loss(h64 + e * u, w64) - loss(h64 - e * u, w64)) / (2 * e), (u * dx).abs().sum()),
                                ((v * dw).sum(), (loss(h64, w64 + e * v) - loss(h64, w64 - e * v)) / (2 * e), (v * dw).abs().sum())):
            assert abs(got - diff) <= 1e-5 * size                               # 2^-24 times some tens, and e^2


def test_the_sum_in_the_place_of_the_residual():
    x, res, w = _rows(40, 512, torch.bfloat16, 1), _rows(40, 512, torch.bfloat16, 2), _weight(512, torch.bfloat16)
    x, res = x.contiguous(), res.contiguous()
    want = B.rms_norm(x, w, res)
    for place in (res.clone(), x.clone()):
        a, b = (place, res) if torch.equal(place, x) else (x, place)
        out = B.RmsNormOut(torch.empty_like(x), place, torch.empty(40, device="cuda"))
        B.rms_norm(a, w, b, out=out)
        assert torch.equal(out.h, want.h) and torch.equal(out.y, want.y) and out.h is place


def test_no_rows_and_graphs():
    w = _weight(256, torch.bfloat16)
    empty = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    out = B.rms_norm(empty, w, empty, keep=True)
    dx, dw = B.rms_norm_backward(empty, out.h, out.rstd, w)
    assert out.y.shape == dx.shape == (0, 256) and (dw == 0).all() and dw.shape == (256,)
    x, dy = _rows(300, 2048, torch.bfloat16, 1), _rows(300, 2048, torch.bfloat16, 2)
    w = _weight(2048, torch.float32)
    both = lambda: (lambda o: (o.y, o.rstd, *B.rms_norm_backward(dy, o.h, o.rstd, w)))(B.rms_norm(x, w, dy, keep=True))   # noqa: E731
    want = both()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = both()
    x.mul_(0.5)
    graph.replay()
    want2 = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want2)) and not torch.equal(want[0], want2[0])
    del graph
    lead = B.rms_norm(x.view(3, 100, 2048), w, keep=True)                      # any leading dimensions
    flat = B.rms_norm(x, w, keep=True)
    assert torch.equal(lead.y.view(300, 2048), flat.y) and lead.rstd.shape == (3, 100) and lead.y8.codes.shape == (3, 100, 2048)


def test_offsets_past_32_bits():
    rows, cols = 300_000, 8192                                                  # 2.5e9 elements
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[:4], x[-4:] = _rows(4, cols, torch.bfloat16, 1), _rows(4, cols, torch.bfloat16, 2)
    x[4:-4] = 1.0
    w = _weight(cols, torch.bfloat16)
    out = B.rms_norm(x, w, keep=True)
    tail = B.rms_norm(x[-4:], w, keep=True)
    assert torch.equal(out.y[-4:], tail.y) and torch.equal(out.y8.codes[-4:], tail.y8.codes) and torch.equal(out.y8.scales[-4:], tail.y8.scales)
    dx, _ = B.rms_norm_backward(x, out.h, out.rstd, w, dx=out.y)
    want, _ = B.rms_norm_backward(x[-4:].contiguous(), tail.h.contiguous(), tail.rstd, w)
    assert torch.equal(dx[-4:], want)
    del x, out, dx
    torch.cuda.empty_cache()
