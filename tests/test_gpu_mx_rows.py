"""moe_mx_quantize / moe_mx_dequantize against the format written out in 64 bits (mx_util), bit for bit."""
import numpy as np
import pytest
import torch

import mx_util as M
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _check(x: torch.Tensor, m: B.MxRows):
    codes, scales = M.quantize(x.double().cpu().numpy())
    assert np.array_equal(m.scales.cpu().numpy(), scales)
    assert np.array_equal(m.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", [(1, 32), (3, 64), (5, 96), (1, 7168), (17, 1000 // 32 * 32), (33, 4096), (1000, 544), (129, 2048)])
def test_rows_match_the_definition(dtype, rows, K):
    x = torch.from_numpy(M.random_rows(rows, K, rows + K, 4.0)).to(TYPES[dtype]).cuda()
    m = B.mx_quantize(x)
    _check(x, m)
    want = M.values(*M.quantize(x.double().cpu().numpy()))
    for out in TYPES.values():
        got = B.mx_dequantize(m, out)
        assert got.shape == x.shape and got.dtype == out
        # exact in fp32 and bf16; fp16 rounds (or overflows) once, as the cast of the value does.  Blocks in
        # which the fp16 input itself overflowed are NaN on both sides.
        torch.testing.assert_close(got.cpu(), torch.from_numpy(want).to(out), rtol=0, atol=0, equal_nan=True)


def test_many_units_take_the_wide_launch():
    x = torch.from_numpy(M.random_rows(700, 7168, 9)).to(torch.bfloat16).cuda()
    _check(x, B.mx_quantize(x))


def test_special_values():
    rng = np.random.default_rng(0)
    rows = []
    base = rng.standard_normal(32).astype(np.float32)
    for special in (np.nan, -np.nan, np.inf, -np.inf):
        r = base.copy(); r[rng.integers(32)] = special; rows.append(r)
    rows.append(np.zeros(32, np.float32))
    rows.append(-np.zeros(32, np.float32))
    tiny = np.zeros(32, np.float32); tiny[3] = np.float32(2.0 ** -149); rows.append(tiny)     # smallest subnormal
    sub = (base * np.float32(2.0 ** -128)).astype(np.float32); rows.append(sub)
    big = np.full(32, np.finfo(np.float32).max, np.float32); big[::2] *= -1; rows.append(big)
    # every midpoint and every neighbour of a midpoint, at a block maximum of 7.9 (saturates to 6)
    for eps in (0.0, 2.0 ** -20, -2.0 ** -20):
        r = np.zeros(32, np.float32)
        r[:8] = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], np.float32) + np.float32(eps)
        r[8:16] = -r[:8]
        r[31] = 7.9
        rows.append(r)
    x = torch.from_numpy(np.stack(rows)).cuda()
    m = B.mx_quantize(x)
    _check(x, m)
    y = B.mx_dequantize(m, torch.float32)
    assert torch.isnan(y[:4]).all() and (y[4:6] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_16_bit_pattern(dtype):
    """All 65536 bit patterns, NaN, infinities and subnormals among them: one to a block of ordinary numbers, and
    as blocks of neighbours."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    alone = torch.from_numpy(M.random_rows(65536, 32, 1)).to(dtype)
    alone[torch.arange(65536), torch.arange(65536) % 32] = bits.view(dtype)
    for x in (alone, bits.view(dtype).view(2048, 32), bits.view(dtype).view(32, 2048).t().contiguous()):
        x = x.cuda()
        _check(x, B.mx_quantize(x))


def test_leading_dimensions_and_strided_rows():
    x = torch.randn(3, 5, 64, device="cuda", dtype=torch.float16)
    m = B.mx_quantize(x)
    assert m.codes.shape == (3, 5, 32) and m.scales.shape == (3, 5, 16)
    _check(x, m)
    wide = torch.randn(7, 200, device="cuda", dtype=torch.bfloat16)
    part = wide[:, 8:8 + 96]                         # rows 400 bytes apart, first row 16 bytes in
    m = B.mx_quantize(part)
    _check(part.contiguous(), m)
    back = torch.full_like(wide, -3.0)
    B.mx_dequantize(m, torch.bfloat16, out=back[:, 16:16 + 96])
    assert torch.equal(back[:, 16:112], B.mx_dequantize(m))
    assert (back[:, :16] == -3).all() and (back[:, 112:] == -3).all()


def test_no_rows():
    m = B.mx_quantize(torch.empty(0, 64, device="cuda"))
    assert m.codes.shape == (0, 32) and B.mx_dequantize(m).shape == (0, 64)


def test_other_stream_and_graph():
    x = torch.randn(40, 512, device="cuda", dtype=torch.bfloat16)
    out = B.mx_empty(40, 512)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        m = B.mx_quantize(x)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.mx_quantize(x, out)
    s.synchronize()
    _check(x, m)
    x.copy_(torch.randn_like(x))
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    _check(x, out)


def test_guard_zones():
    rows, K = 37, 1056                               # 33 blocks a row: ragged warps and a padded row of scales
    c = torch.full((rows * K // 2 + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.full((rows * M.pitch(K) + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    m = B.MxRows(c[32:-32].view(rows, K // 2), s[32:-32].view(rows, M.pitch(K)))
    x = torch.randn(rows, K, device="cuda")
    B.mx_quantize(x, m)
    _check(x, m)
    for t in (c, s):
        assert (t[:32] == 0xAB).all() and (t[-32:] == 0xAB).all()
