"""The microscaled 4-bit format written out once more for the tests, in numpy and 64 bits: a value is
rounded by comparing its distances to the grid, nothing is shared with the kernels."""
import numpy as np
import torch

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
BLOCK = 32


def pitch(cols: int) -> int:
    return -(-(cols // BLOCK) // 16) * 16


def scale_bytes(x: np.ndarray) -> np.ndarray:
    """[..., K] f64 -> [..., K/32] scale bytes."""
    b = np.abs(x.reshape(*x.shape[:-1], -1, BLOCK))
    a = b.max(-1)                                        # NaN if the block has one
    out = np.full(a.shape, 255, np.int64)
    fine = np.isfinite(a)
    pos = fine & (a > 0)
    out[fine] = 0
    # a = m * 2^e with m in [0.5, 1): floor(log2 a) = e - 1
    out[pos] = np.clip(np.frexp(a[pos])[1] - 1 - 2 + 127, 0, 254)
    return out


def round_codes(x: np.ndarray, s: np.ndarray) -> np.ndarray:
    """Codes of [..., K] values under given scale bytes: nearest grid point, ties to the even code."""
    b = x.reshape(*x.shape[:-1], -1, BLOCK)
    with np.errstate(invalid="ignore"):
        m = np.abs(b) * 2.0 ** (127.0 - s[..., None])
        d = np.abs(m[..., None] - GRID)                  # exact: both are short binary numbers
        best = np.where(m >= 6, 7, np.argmin(d, -1))     # argmin takes the lower of two equal distances
    up = np.minimum(best + 1, 7)
    tie = (best % 2 == 1) & (best < 7) & (np.take_along_axis(d, best[..., None], -1) == np.take_along_axis(d, up[..., None], -1))[..., 0]
    code = np.where(tie, up, best) | (np.signbit(b).astype(np.int64) << 3)
    code = np.where(s[..., None] == 255, 0, code)
    return code.reshape(x.shape)


def quantize(x: np.ndarray):
    """[..., K] f64 -> (codes [..., K/2] u8, scales [..., pitch] u8 with zero padding)."""
    s = scale_bytes(x)
    c = round_codes(x, s)
    packed = (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)
    scales = np.zeros((*x.shape[:-1], pitch(x.shape[-1])), np.uint8)
    scales[..., :s.shape[-1]] = s
    return packed, scales


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The f64 values of 4-bit rows."""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    v = np.where(c & 8, -1.0, 1.0) * GRID[c & 7]
    s = scales[..., :v.shape[-1] // BLOCK].astype(np.float64)
    f = np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return (v.reshape(*v.shape[:-1], -1, BLOCK) * f[..., None]).reshape(v.shape)


def random_rows(rows: int, K: int, seed: int, spread: float = 0.0) -> np.ndarray:
    """f64 rows that are bf16 numbers; `spread`: standard deviation of a log2 magnitude per block."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, K))
    if spread:
        x *= np.repeat(2.0 ** np.round(spread * rng.standard_normal((rows, K // BLOCK))), BLOCK, axis=1)
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def segments(counts, order=None):
    """(counts, offsets [P+1]) int32 for slots laid out one after the other, in `order` where given."""
    counts = np.asarray(counts, np.int32)
    offsets = np.zeros(counts.size + 1, np.int32)
    at = 0
    for p in (range(counts.size) if order is None else order):
        offsets[p] = at
        at += counts[p]
    offsets[-1] = at
    return counts, offsets
