"""Experts in 16 bits and the 8-bit rows once more for the tests, in 64 bits, with the bounds that their sums allow."""
import torch

from paper_2602_21140_b200 import binding as B

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # half a step, relative


def make_router(P, H=64, T=16):
    return B.MoeRouter(B.make_config(P, 1, H, T, P, 1, 1), range(P), None, [1.0] * P)


def bf16(*shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, device="cuda", generator=g) * scale).bfloat16()


def layout(counts, gap=0, order=None):
    """(counts, offsets) of segments laid out in `order`, `gap` rows before each and behind the last; rows in all."""
    off, at = [0] * len(counts), 0
    for p in (range(len(counts)) if order is None else order):
        at += gap
        off[p] = at
        at += counts[p]
    i32 = dict(dtype=torch.int32, device="cuda")
    return torch.tensor(counts, **i32), torch.tensor(off, **i32), at + gap


def sum_bound(K, magnitude):
    """A sum of K products, `magnitude` in absolute terms, on the tensor cores: sixteen at a time are added to the accumulator
    and what does not fit 24 bits beside the largest term is cut off, 17 terms a step, each by at most 2^-24 of `magnitude`
    twice over (its own bits and the accumulator's)."""
    return (K / 16 + 1) * 2.0 ** -22 * magnitude


def values8(m: B.Mx8Rows) -> torch.Tensor:
    """The f64 values of 8-bit rows, from the bits of the codes."""
    c, s = m.codes.long(), m.scales[..., :m.codes.shape[-1] // 32].long()
    e, f = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e > 0, (8 + f) * torch.exp2(e.double() - 10), f * 2.0 ** -9)
    v = torch.where((c & 127) == 127, torch.full_like(v, float("nan")), v) * torch.where(c >= 128, -1.0, 1.0)
    scale = torch.where(s == 255, torch.full_like(s, 1).double() * float("nan"), torch.exp2(s.double() - 127))
    return (v.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def check8(m: B.Mx8Rows, x, off):
    """8-bit rows of f64 values `x` that the kernel knew to within `off` (>= 0, same shape)."""
    s = m.scales[..., :x.shape[-1] // 32].double()
    scale = torch.exp2(s - 127)
    blocks = lambda t: t.unflatten(-1, (-1, 32))             # noqa: E731
    amax, slack = blocks(x.abs()).amax(-1), blocks(off).amax(-1)
    assert (amax - slack <= 448 * scale).all(), "a scale is too small"
    assert ((amax + slack > 224 * scale) | (s == 0)).all(), "a scale is too large"
    half = torch.maximum(2.0 ** -4 * x.abs(), (scale * 2.0 ** -10).repeat_interleave(32, -1))
    err = (values8(m) - x).abs()
    assert (err <= half + 1.07 * off).all(), float((err - half).max())


def within(got, want, bound):
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, worst {float((err - bound).max())} over the bound"
