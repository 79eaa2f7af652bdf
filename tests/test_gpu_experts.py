"""The experts' products on bf16 rows and their gradients against the formulas in 64 bits, slot by slot, at the sizes,
layouts and values where a tile, a pair of tiles or a K = 16 ends."""
import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu

# (rows of each slot, n_in = n_out = H, n_hidden = I): tiles have 256 features and at most 256 rows, stages 64 of K; up to 64 and
# up to 128 rows in the longest segment the ring is another one.
SIZES = [
    ([1], 8, 16), ([0, 1, 0], 64, 16), ([3, 0, 64, 17, 1], 136, 48), ([65, 20, 5], 264, 144), ([15, 16, 17, 31, 33], 512, 128),
    ([66], 8, 16), ([130, 0, 257], 72, 272), ([700, 3, 129, 1], 1032, 80), ([256, 255, 512, 511], 256, 128), ([2100], 64, 32), ([0, 300, 0], 320, 640),
]
IDS = [f"{sum(c)}x{h}x{i}" for c, h, i in SIZES]


def _spans(counts, offsets):
    return [(p, o, o + c) for p, (c, o) in enumerate(zip(counts, offsets.tolist()))]


def _sigmoid_bound(g):
    """Relative error of the kernels' sigmoid: the hardware's exp and reciprocal, and a rounded argument."""
    return (g.abs() + 8) * 2.0 ** -23


@pytest.mark.parametrize("kept", ["no", "16", "8"])
@pytest.mark.parametrize("counts,H,I", SIZES, ids=IDS)
def test_forward(counts, H, I, kept):
    P = len(counts)
    r = U.make_router(P)
    n_, off, n = U.layout(counts, gap=3, order=list(range(P))[::-1])
    a, gate_up, down = U.bf16(n, H, seed=1), U.bf16(P, 2 * I, H, seed=2, scale=H ** -0.5), U.bf16(P, H, I, seed=3, scale=I ** -0.5)
    used = torch.zeros(n, dtype=torch.bool, device="cuda")
    for _, s, e in _spans(counts, off):
        used[s:e] = True
    a[~used] = float("nan")                                    # rows of no segment
    h, y = torch.full((n, I), -7.0, dtype=torch.bfloat16, device="cuda"), torch.full((n, H), -7.0, dtype=torch.bfloat16, device="cuda")
    z = None
    if kept == "16":
        z = torch.full((n, 2 * I), -7.0, dtype=torch.bfloat16, device="cuda")
    elif kept == "8":
        z = B.mx8_empty(n, 2 * I)
        z.codes.fill_(9); z.scales.fill_(0)
    assert r.expert_ffn(a, n_, off, gate_up, down, y, h, z) is y
    torch.cuda.synchronize()
    assert r.device_status() == 0
    for t in (h, y) + ((z,) if kept == "16" else ()):
        assert (t[~used] == -7).all()
    if kept == "8":
        assert (z.codes[~used] == 9).all() and (z.scales[~used] == 0).all()
    for p, s, e in _spans(counts, off):
        if s == e:
            continue
        x, w = a[s:e].double(), gate_up[p].double()
        v, dv = x @ w.T, U.sum_bound(H, x.abs() @ w.abs().T)
        g, u, dg, du = v[:, 0::2], v[:, 1::2], dv[:, 0::2], dv[:, 1::2]
        silu = g * torch.sigmoid(g)
        # |d silu / dg| < 1.1
        bound = 1.1 * (dg * u.abs() + silu.abs() * du + 1.1 * dg * du) + silu.abs() * u.abs() * _sigmoid_bound(g)
        U.within(h[s:e], silu * u, (1 + 2.0 ** -8) * bound + 2.0 ** -8 * (silu * u).abs() + 1e-36)
        if kept == "16":
            U.within(z[s:e], v, (1 + 2.0 ** -8) * dv + 2.0 ** -8 * v.abs())
        elif kept == "8":
            U.check8(B.Mx8Rows(z.codes[s:e], z.scales[s:e]), v, dv)
        hs, d = h[s:e].double(), down[p].double()
        want = hs @ d.T
        U.within(y[s:e], want, U.sum_bound(I, hs.abs() @ d.abs().T) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs())
    r.close()


@pytest.mark.parametrize("kept", ["16", "8"])
@pytest.mark.parametrize("counts,H,I", SIZES, ids=IDS)
def test_backward(counts, H, I, kept):
    P = len(counts)
    r = U.make_router(P)
    n_, off, n = U.layout(counts, gap=5, order=list(range(P))[1:] + [0])
    a, dy = U.bf16(n, H, seed=1), U.bf16(n, H, seed=4)
    gate_up, down = U.bf16(P, 2 * I, H, seed=2, scale=H ** -0.5), U.bf16(P, H, I, seed=3, scale=I ** -0.5)
    used = torch.zeros(n, dtype=torch.bool, device="cuda")
    for _, s, e in _spans(counts, off):
        used[s:e] = True
    for t in (a, dy):
        t[~used] = float("nan")
    zv = U.bf16(n, 2 * I, seed=5, scale=3.0)
    if kept == "8":
        codes = torch.randint(0, 256, (n, 2 * I), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(6))
        codes[(codes & 127) == 127] = 3
        z = B.Mx8Rows(codes, torch.full((n, B._mx_pitch(2 * I)), 120, dtype=torch.uint8, device="cuda"))
        zv = U.values8(z)
    else:
        zv[~used] = float("nan")
        z = zv
    full = lambda cols: torch.full((n, cols), -7.0, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    dz, h, d_rows = full(2 * I), full(I), full(H)
    r.expert_gated_backward(dy, n_, off, down, z, dz, h)
    r.expert_rows_backward(dz, n_, off, gate_up, d_rows)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    for t in (dz, h, d_rows):
        assert (t[~used] == -7).all()
    dz[~used] = float("nan"); h[~used] = float("inf")
    grads = [r.expert_weight_backward(dz, a, n_, off, dtype=t) for t in (torch.bfloat16, torch.float32)]
    d_down = r.expert_weight_backward(dy, h, n_, off)
    before = torch.randn(P, 2 * I, H, device="cuda")
    added = r.expert_weight_backward(dz, a, n_, off, before.clone(), add=True)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    for p, s, e in _spans(counts, off):
        if s == e:
            assert not grads[0][p].any() and not grads[1][p].any() and not d_down[p].any() and torch.equal(added[p], before[p])
            continue
        g, u, w = zv[s:e, 0::2].double(), zv[s:e, 1::2].double(), down[p].double()
        sg, t = torch.sigmoid(g), dy[s:e].double()
        dh, ddh = t @ w, U.sum_bound(H, t.abs() @ w.abs())
        slope = u * (sg + g * sg * torch.sigmoid(-g))
        # the two terms of the slope, each with the sigmoid's error, that of 1 - s being absolute
        off_slope = u.abs() * sg * ((1 + g.abs()) * _sigmoid_bound(g) + g.abs() * (_sigmoid_bound(g) + 2.0 ** -22))
        for got, f, df in ((dz[s:e, 0::2], slope, off_slope), (dz[s:e, 1::2], g * sg, (g * sg).abs() * _sigmoid_bound(g))):
            bound = ddh * f.abs() + (dh.abs() + ddh) * (df + 2.0 ** -21 * f.abs())
            U.within(got, dh * f, (1 + 2.0 ** -8) * bound + 2.0 ** -8 * (dh * f).abs() + 1e-34)
        hv = g * sg * u
        U.within(h[s:e], hv, (2.0 ** -8 + 2.0 ** -21) * hv.abs() + hv.abs() * _sigmoid_bound(g) + 1e-34)
        d, m = dz[s:e].double(), gate_up[p].double()
        U.within(d_rows[s:e], d @ m, U.sum_bound(2 * I, d.abs() @ m.abs()) * (1 + 2.0 ** -8) + 2.0 ** -8 * (d @ m).abs())
        for got, left, right in ((grads[0][p], d, a[s:e].double()), (grads[1][p], d, a[s:e].double()), (d_down[p], t, h[s:e].double())):
            want, half = left.T @ right, U.HALF[got.dtype]
            bound = U.sum_bound(e - s, left.abs().T @ right.abs())
            U.within(got, want, (1 + half) * bound + half * want.abs())
        # one rounding of the sum with what was there
        total = grads[1][p].double() + before[p].double()
        U.within(added[p], total, 2.0 ** -24 * total.abs())
    r.close()


def test_fp32_gradients_of_many_rows():
    """Sums of 960 rows at a time: 20000 rows are as near as cutting off in 60 steps of K = 16 leaves them, plus a rounding for
    each of the 21 pieces.  (In one accumulator they would be off by twenty times as much.)"""
    r = U.make_router(1)
    n_, off, n = U.layout([20000])
    dy, a = U.bf16(n, 64, seed=1).abs(), U.bf16(n, 72, seed=2).abs()      # all of one sign: cutting off adds up
    got = r.expert_weight_backward(dy, a, n_, off, dtype=torch.float32)[0].double()
    want = dy.double().T @ a.double()
    assert ((got - want).abs() <= (U.sum_bound(960, 1.0) + 21 * 2.0 ** -24) * want).all()
    r.close()


def test_fp32_gradients_beside_longer_segments():
    """Segments of one piece beside ones of two, of none, and alone in a call: the same bits, whichever way the call's sums go."""
    counts = [961, 0, 45, 960, 1500, 1, 530]
    P = len(counts)
    r = U.make_router(P)
    n_, off, n = U.layout(counts, gap=3)
    dy, a = U.bf16(n, 272, seed=1), U.bf16(n, 520, seed=2)
    before = torch.randn(P, 272, 520, device="cuda")
    got = r.expert_weight_backward(dy, a, n_, off, dtype=torch.float32)
    added = r.expert_weight_backward(dy, a, n_, off, before.clone(), add=True)
    assert torch.equal(added, torch.where(torch.tensor(counts, device="cuda")[:, None, None] > 0, got + before, before))
    short = torch.where(n_ > 960, torch.zeros_like(n_), n_)       # the same buffer, no segment of two pieces
    alone = r.expert_weight_backward(dy, a, short, off, dtype=torch.float32)
    for p, s, e in _spans(counts, off):
        if e - s <= 960:
            assert torch.equal(got[p], alone[p])
            few, where = torch.zeros_like(n_), torch.zeros_like(off)   # a buffer that no segment of two pieces fits
            few[p] = e - s
            assert torch.equal(got[p], r.expert_weight_backward(dy[s:e], a[s:e], few, where, dtype=torch.float32)[p])
        want, size = dy[s:e].double().T @ a[s:e].double(), dy[s:e].double().abs().T @ a[s:e].double().abs()
        U.within(got[p], want, (1 + 2.0 ** -24) * (U.sum_bound(min(e - s, 960), size) + 2 * 2.0 ** -24 * size) + 2.0 ** -24 * want.abs())
    assert r.device_status() == 0
    r.close()


def test_values_at_the_edge():
    """Gates beyond exp's range, infinities and NaN stay in their row; a large gate is the identity, a very negative one 0."""
    r = U.make_router(1)
    n_, off, n = U.layout([6])
    H, I = 16, 16
    a = torch.zeros(n, H, device="cuda").bfloat16()
    a[:, 0] = torch.tensor([1.0, -1.0, float("inf"), float("nan"), 0.0, 2.0])
    gate_up = torch.zeros(1, 2 * I, H, device="cuda").bfloat16()
    gate_up[0, 0::2, 0], gate_up[0, 1::2, 0] = 1e4, 1.0
    z = B.mx8_empty(n, 2 * I)
    h = r.expert_gated(a, n_, off, gate_up, z=z)
    torch.cuda.synchronize()
    # 1e4 is 9984 in bf16
    assert (h[0] == 9984).all() and (h[1] == 0).all() and (h[4] == 0).all() and (h[5] == 39936).all()
    assert not torch.isfinite(h[2:4]).any() and (z.scales[2:4, 0] == 255).all() and (z.codes[2:4] == 0).all()
    assert (z.scales[4] == 0)[0] and (z.codes[4] == 0).all()
    dy = torch.ones(n, H, device="cuda").bfloat16()
    down = torch.zeros(1, H, I, device="cuda").bfloat16()
    down[0, 0] = 1.0
    kept = torch.zeros(n, 2 * I, device="cuda").bfloat16()
    kept[:, 0::2] = torch.tensor([200.0, -200.0, 0.0, -87.0, 87.0, float("nan")], device="cuda")[:, None].bfloat16()
    kept[:, 1::2] = 3.0
    dz, h = r.expert_gated_backward(dy, n_, off, down, kept)
    torch.cuda.synchronize()
    # dz of the gate: u s (1 + g (1 - s)); of the up-projection: g s
    assert (dz[0, 0::2] == 3).all() and (dz[0, 1::2] == 200).all() and (dz[1] == 0).all()
    assert (dz[2, 0::2] == 1.5).all() and (dz[2, 1::2] == 0).all() and (h[2] == 0).all()
    assert torch.isfinite(dz[3:5]).all() and (dz[4, 0::2] == 3).all() and torch.isnan(dz[5]).all()
    r.close()


@pytest.mark.parametrize("most", [1.75, 1.0, 1.9921875])
def test_scales_of_kept_sums_at_their_steps(most):
    """The largest sum of a block, at every place of it, a little below, at and above `most` times a power of two, up to the
    largest that is finite: the scale is the smallest that will do.  The sums are exact: two terms that 24 bits hold."""
    P, I = 32, 16                                            # slot p has its largest at p
    rows = [(2.0 ** e, s * 2.0 ** e) for e in (-100, -7, 0, 1, 120, 127) for s in (-1, 0, 1)]
    r = U.make_router(P)
    n_, off, n = U.layout([len(rows)] * P)
    a = torch.zeros(n, 16, device="cuda").bfloat16()
    a[:, :2] = torch.tensor(rows * P)
    gate_up = torch.zeros(P, 2 * I, 16, device="cuda").bfloat16()
    gate_up[:, :, 0] = 0.25
    gate_up[torch.arange(P), torch.arange(P), 0] = most
    gate_up[torch.arange(P), torch.arange(P), 1] = 2.0 ** -20
    z = B.mx8_empty(n, 2 * I)
    r.expert_gated(a, n_, off, gate_up, z=z)
    torch.cuda.synchronize()
    want = torch.bmm(a.double().view(P, -1, 16), gate_up.double().transpose(1, 2)).view(n, 2 * I)
    assert want.float().isfinite().all() and (want.float() == want).all()
    U.check8(z, want, torch.zeros_like(want))
    r.close()


def test_segments_from_device_memory_are_cut():
    """Counts and offsets that leave the row buffer: segments are cut or dropped, nothing beyond the buffers is touched."""
    r = U.make_router(4)
    H, I, n = 64, 32, 40
    guard = 64
    i32 = dict(dtype=torch.int32, device="cuda")
    counts, off = torch.tensor([10, 100, -5, 7], **i32), torch.tensor([0, 30, 12, -3], **i32)
    a, gate_up = U.bf16(n + guard, H, seed=1), U.bf16(4, 2 * I, H, seed=2)
    whole = torch.full((n + guard, I), -7.0, dtype=torch.bfloat16, device="cuda")
    h = whole[:n]
    r.expert_gated(a[:n], counts, off, gate_up, h)
    dw = r.expert_weight_backward(a[:n], a[:n], counts, off, dtype=torch.float32)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    assert (whole[10:30] == -7).all() and (whole[n:] == -7).all() and not (whole[:10] == -7).any() and not (whole[30:40] == -7).any()
    x = a[:n].double()
    for p, (s, e) in enumerate(((0, 10), (30, 40), (0, 0), (0, 0))):
        U.within(dw[p], x[s:e].T @ x[s:e], U.sum_bound(16, x[s:e].abs().T @ x[s:e].abs()))
    r.close()


def test_no_rows():
    r = U.make_router(3)
    counts, off = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    gate_up, down = U.bf16(3, 64, 48, seed=1), U.bf16(3, 48, 32, seed=2)
    for n in (0, 5, 500):                                      # an empty buffer, and buffers with no segment in them
        a = U.bf16(n, 48, seed=3)
        y = torch.full((n, 48), -7.0, dtype=torch.bfloat16, device="cuda")
        z = torch.zeros(n, 64, dtype=torch.bfloat16, device="cuda")
        r.expert_ffn(a, counts, off, gate_up, down, y, z=z)
        assert (y == -7).all()
        _, d_gate_up, d_down = r.expert_ffn_backward(a, a, counts, off, gate_up, down, z)
        assert d_gate_up.shape == gate_up.shape and not d_gate_up.any() and not d_down.any()
        kept = torch.ones(3, 64, 48, device="cuda")
        r.expert_weight_backward(z, a, counts, off, kept, add=True)
        assert (kept == 1).all()
    assert r.device_status() == 0
    r.close()


@pytest.mark.parametrize("counts", [[40, 3, 0, 17], [300, 30, 700, 1]], ids=["short", "long"])
def test_calls_repeat_bit_for_bit_and_in_graphs(counts):
    """Eagerly, on another stream, and captured and replayed over other counts, between eager calls of the same context."""
    r = U.make_router(4)
    H, I = 136, 80
    n_, off, n = U.layout(counts)
    a, dy = U.bf16(n, H, seed=1), U.bf16(n, H, seed=2)
    gate_up, down = U.bf16(4, 2 * I, H, seed=3, scale=H ** -0.5), U.bf16(4, H, I, seed=4, scale=I ** -0.5)

    def step(z):
        y = r.expert_ffn(a, n_, off, gate_up, down, z=z)
        return (y, *r.expert_ffn_backward(dy, a, n_, off, gate_up, down, z, grad_dtype=torch.float32))

    z = B.mx8_empty(n, 2 * I)
    want = step(z)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step(B.mx8_empty(n, 2 * I))
    graph = torch.cuda.CUDAGraph()
    zg = B.mx8_empty(n, 2 * I)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step(zg)
    graph.replay()
    torch.cuda.synchronize()
    for w, o, g in zip(want, other, got):
        assert torch.equal(w, o) and torch.equal(w, g)
    # the same graph, other segments in the same rows: what an eager call computes for them
    n_.copy_(n_.flip(0)); off.copy_(torch.cat((n_.new_zeros(1), n_.cumsum(0)[:-1])).int())
    graph.replay()
    want = step(z)
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert torch.equal(w, g)
    assert r.device_status() == 0
    del graph
    r.close()


def test_a_rows_sums_do_not_depend_on_its_tile():
    """The same segments beside one that makes the ring another one, and in a longer buffer."""
    P, H, I = 6, 520, 176
    r = U.make_router(P)
    short, extra = [5, 64, 33, 0, 17], 700
    n1, off1, n = U.layout(short + [0])
    n2, off2, m = U.layout(short + [extra])
    a = U.bf16(m + 50, H, seed=1)
    gate_up, down = U.bf16(P, 2 * I, H, seed=3, scale=H ** -0.5), U.bf16(P, H, I, seed=4, scale=I ** -0.5)
    calls = []
    for rows, counts, off in ((a[:n], n1, off1), (a, n2, off2)):
        z = torch.empty(rows.shape[0], 2 * I, dtype=torch.bfloat16, device="cuda")
        y = r.expert_ffn(rows, counts, off, gate_up, down, z=z)
        dz, h = r.expert_gated_backward(rows, counts, off, down, z)
        calls.append((z, y, dz, h, r.expert_rows_backward(dz, counts, off, gate_up)))
    torch.cuda.synchronize()
    for one, two in zip(*calls):
        assert torch.equal(one, two[:n])
    r.close()


def test_the_end_of_a_segment_under_load():
    """Odd segments between rows of NaN, many times over with all SMs busy: lines behind a segment that were not zero in time
    would be NaN in its gradient."""
    P = 96
    r = U.make_router(P)
    counts = [(37 * p) % 190 + 1 for p in range(P)]
    n_, off, n = U.layout(counts, gap=1)
    dy, a = U.bf16(n, 512, seed=1), U.bf16(n, 768, seed=2)
    inside = torch.zeros(n, dtype=torch.bool, device="cuda")
    for _, s, e in _spans(counts, off):
        inside[s:e] = True
    dy[~inside] = float("nan"); a[~inside] = float("inf")
    first = r.expert_weight_backward(dy, a, n_, off, dtype=torch.float32)
    for _ in range(60):
        again = r.expert_weight_backward(dy, a, n_, off, dtype=torch.float32)
    torch.cuda.synchronize()
    assert torch.isfinite(first).all() and torch.equal(first, again)
    for p, s, e in _spans(counts, off)[::13]:
        left, right = dy[s:e].double(), a[s:e].double()
        U.within(first[p], left.T @ right, U.sum_bound(e - s, left.abs().T @ right.abs()))
    r.close()


def test_two_contexts_at_once():
    P, H, I = 8, 512, 256
    n_, off, n = U.layout([90] * P)
    a, gate_up, down = U.bf16(n, H, seed=1), U.bf16(P, 2 * I, H, seed=2, scale=H ** -0.5), U.bf16(P, H, I, seed=3, scale=I ** -0.5)
    routers, streams = [U.make_router(P) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    want = routers[0].expert_ffn(a, n_, off, gate_up, down)
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for r, s in zip(routers, streams):
            with torch.cuda.stream(s):
                got.append(r.expert_ffn(a, n_, off, gate_up, down))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got) and all(r.device_status() == 0 for r in routers)
    for r in routers:
        r.close()


def test_thousands_of_slots_and_wide_matrices():
    """As many slots as a context takes at 512 experts, few of them with rows, where their table takes a stage's place; and more
    features than a wave has tiles."""
    P, H, I = 2000, 72, 48
    r = B.MoeRouter(B.make_config(512, 1, H, 16, P // 8, 8, 8), [p % 512 if p < 2000 else -1 for p in range(P)], None, [1.0] * P)
    counts = [0] * P
    for p, n in ((0, 3), (7, 300), (1023, 1), (1024, 65), (1999, 40)):
        counts[p] = n
    n_, off, n = U.layout(counts)
    a, gate_up, down = U.bf16(n, H, seed=1), U.bf16(P, 2 * I, H, seed=2, scale=H ** -0.5), U.bf16(P, H, I, seed=3, scale=I ** -0.5)
    z = torch.empty(n, 2 * I, dtype=torch.bfloat16, device="cuda")
    y = r.expert_ffn(a, n_, off, gate_up, down, z=z)
    d_rows, d_gate_up, d_down = r.expert_ffn_backward(a, a, n_, off, gate_up, down, z, grad_dtype=torch.float32)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    few = U.make_router(5)
    at = torch.tensor([0, 7, 1023, 1024, 1999], device="cuda")
    args = (n_[at].contiguous(), off[at].contiguous())
    y2 = few.expert_ffn(a, *args, gate_up[at].contiguous(), down[at].contiguous())
    want = few.expert_ffn_backward(a, a, *args, gate_up[at].contiguous(), down[at].contiguous(), z, grad_dtype=torch.float32)
    assert torch.equal(y, y2) and torch.equal(d_rows, want[0]) and torch.equal(d_gate_up[at], want[1]) and torch.equal(d_down[at], want[2])
    rest = torch.ones(P, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert not d_gate_up[rest].any() and not d_down[rest].any()
    few.close(); r.close()
    r = U.make_router(1)
    n_, off, n = U.layout([130])
    a, w = U.bf16(n, 40, seed=1), U.bf16(1, 40_008, 40, seed=2)
    y = r.expert_product(a, n_, off, w)
    back = r.expert_rows_backward(y, n_, off, w)
    dw = r.expert_weight_backward(y, a, n_, off)
    torch.cuda.synchronize()
    x, m, t = a.double(), w[0].double(), y.double()
    U.within(y, x @ m.T, U.sum_bound(40, x.abs() @ m.abs().T) * 1.01 + 2.0 ** -8 * (x @ m.T).abs())
    U.within(back, t @ m, U.sum_bound(40_008, t.abs() @ m.abs()) * 1.01 + 2.0 ** -8 * (t @ m).abs())
    U.within(dw[0], t.T @ x, U.sum_bound(130, t.abs().T @ x.abs()) * 1.01 + 2.0 ** -8 * (t.T @ x).abs())
    assert r.device_status() == 0
    r.close()


def test_a_long_sum_is_no_reason_to_give_up():
    """8 million rows in one segment: a tile takes longer than most steps, and the waits for it are counted in polls."""
    r = U.make_router(1)
    n_, off, n = U.layout([8_000_001])
    a, dy = (torch.ones(n, 8, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dy[:, 3] = 0
    for dtype in (torch.float32, torch.bfloat16):
        dw = r.expert_weight_backward(dy, a, n_, off, dtype=dtype)[0].double()
        torch.cuda.synchronize()
        assert r.device_status() == 0 and not dw[3].any()
        # whole numbers below 2^24: nothing is cut off
        assert ((dw[:3] - 8_000_001).abs() <= U.HALF[dtype] * 8_000_001).all() and (dw[4:] == dw[0, 0]).all()
    r.close()
    del a, dy
    torch.cuda.empty_cache()


def test_offsets_past_32_bits():
    """A segment at the end of row buffers of 5 GB, and a slot at the end of 9 GB of matrices."""
    H, I, n = 4096, 2056, 600_000
    r = U.make_router(2)
    i32 = dict(dtype=torch.int32, device="cuda")
    counts, off = torch.tensor([0, 9], **i32), torch.tensor([0, n - 9], **i32)
    a, y = (torch.empty(n, H, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    a[n - 9:] = U.bf16(9, H, seed=1)
    w = U.bf16(2, H, H, seed=2, scale=H ** -0.5)
    r.expert_product(a, counts, off, w, y)
    want = r.expert_product(a[n - 9:].contiguous(), counts, torch.tensor([0, 0], **i32), w)
    z = B.mx8_empty(n, 2 * H)
    gate_up = U.bf16(2, 2 * H, H, seed=3, scale=H ** -0.5)
    h = r.expert_gated(a, counts, off, gate_up, y.clone(), z)[n - 9:].clone()
    z2 = B.mx8_empty(9, 2 * H)
    h2 = r.expert_gated(a[n - 9:].contiguous(), counts, torch.tensor([0, 0], **i32), gate_up, z=z2)
    torch.cuda.synchronize()
    # tiles of 64 and of 256 rows give the same bits
    assert torch.equal(y[n - 9:], want) and torch.equal(h, h2)
    assert torch.equal(z.codes[n - 9:], z2.codes) and torch.equal(z.scales[n - 9:], z2.scales)
    r.close()
    del a, y, z, h
    torch.cuda.empty_cache()
    P = 512
    r = U.make_router(P)
    counts, off = (torch.zeros(P, **i32) for _ in range(2))
    counts[P - 1] = 20
    a, dy = U.bf16(20, H, seed=4), U.bf16(20, I, seed=5)
    dw = torch.full((P, I, H), -7.0, dtype=torch.bfloat16, device="cuda")
    r.expert_weight_backward(dy, a, counts, off, dw)
    torch.cuda.synchronize()
    left, right = dy.double(), a.double()
    U.within(dw[P - 1], left.T @ right, 2.0 ** -8 * (left.T @ right).abs() + U.sum_bound(20, left.abs().T @ right.abs()))
    assert not dw[:P - 1].any()
    dw[P - 1] = dw[P - 1] * 2.0 ** -5
    x = r.expert_rows_backward(dy, counts, off, dw)
    want = dy.double() @ dw[P - 1].double()
    U.within(x, want, (2.0 ** -8 + 2.0 ** -15) * want.abs() + 1.01 * U.sum_bound(I, dy.double().abs() @ dw[P - 1].double().abs()))
    r.close()
    del dw
    torch.cuda.empty_cache()
