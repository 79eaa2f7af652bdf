"""Calls of the 4-bit layer and of the gradients that the documentation allows and that are easy to forget: no tokens,
the smallest rows, dense-FFN routing, a compacted rank order, lost experts, launches without overlap, and buffers
whose offsets pass 32 bits."""
import numpy as np
import pytest
import torch

import mx_util as M
from gpu_util import make_router, to_dev
from paper_2602_21140_b200 import binding as B
from paper_2602_21140_b200 import workloads as W

pytestmark = pytest.mark.gpu


def _weights(P, N, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return B.mx_quantize(torch.randn(P, N, K, device="cuda", generator=g, dtype=torch.bfloat16) * K ** -0.5)


def _tiny(T=64, H=256, I=64):
    wl = W.WORKLOADS["tiny"]
    inp = W.make_inputs(wl, T=T, H=H)
    router = make_router(wl, inp, max_tokens=T, hidden=H)
    # replicas of an expert share its weights
    s2e = torch.from_numpy(np.maximum(inp["slot_to_expert"], 0)).long().cuda()
    of = lambda m: B.MxRows(m.codes[s2e], m.scales[s2e])      # noqa: E731
    gate_up, down = of(_weights(wl.E, 2 * I, H, 1)), of(_weights(wl.E, H, I, 2))
    return wl, inp, router, to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16), gate_up, down


def test_no_tokens():
    wl, inp, router, logits, x, gate_up, down = _tiny()
    H, k = x.shape[1], wl.k
    assert router.mx_step(logits[:0], x[:0], gate_up, down).shape == (0, H)
    d_buf, d_w = router.combine_backward(x[:0], x[:0])
    dx, d_logits = router.dispatch_backward(logits[:0], d_buf, d_w)
    assert d_buf.shape == (0, H) and d_w.shape == (0, k) and dx.shape == (0, H) and d_logits.shape == (0, wl.E)
    want = router.mx_step(logits, x, gate_up, down)           # and the next step is an ordinary one
    assert torch.equal(router.mx_step(logits, x, gate_up, down), want) and torch.isfinite(want).all()
    assert router.device_status() == 0
    router.close()


@pytest.mark.parametrize("E,k,H,T", [(1, 1, 8, 1), (2, 2, 8, 300), (5, 3, 16, 77), (512, 16, 8, 40), (3, 2, 24, 1)])
def test_gradients_of_the_smallest_rows(E, k, H, T):
    """Bounds as in test_gpu_backward."""
    r = B.MoeRouter(B.make_config(E, k, H, T, 1, E, 1), range(E), None, [0.75] * E)
    g = torch.Generator(device="cuda").manual_seed(E)
    logits = torch.randn(T, E, device="cuda", generator=g)
    out = r.dispatch(logits, torch.randn(T, H, device="cuda", generator=g).bfloat16())
    buf, dy = (torch.randn(n, H, device="cuda", generator=g).bfloat16() for n in (T * k, T))
    d_buf, d_w = r.combine_backward(buf, dy)
    dx, d_logits = r.dispatch_backward(logits, d_buf, d_w)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    dst, ids, w = out.dst_row.long().view(T, k), out.topk_ids.long(), out.topk_weights.double()
    prod = buf.double()[dst] * dy.double()[:, None]
    assert ((d_w.double() - 0.75 * prod.sum(-1)).abs() <= (H / 256 + 34) * 2.0 ** -24 * 0.75 * prod.abs().sum(-1)).all()
    want = (0.75 * w)[..., None] * dy.double()[:, None]
    assert ((d_buf.double()[dst] - want).abs() <= 2.0 ** -8 * want.abs()).all()
    rows = d_buf.double()[dst]
    assert ((dx.double() - rows.sum(1)).abs() <= 2.0 ** -8 * rows.sum(1).abs() + k * 2.0 ** -24 * rows.abs().sum(1)).all()
    gd = d_w.double()
    got = d_logits.double().gather(1, ids)
    want = w * (gd - (w * gd).sum(1, keepdim=True))
    # w itself is within 1e-6 of summing to one
    assert ((got - want).abs() <= w * (gd.abs() + (w * gd.abs()).sum(1, keepdim=True)) * (16 * k * 2.0 ** -24 + 1e-6)).all()
    assert d_logits.double().abs().sum() == got.abs().sum()   # zero everywhere else
    r.close()


def test_dense_ffn_routing():
    """Tokens dealt over replicated groups of shards, with one shard lost: every shard's network and their sum."""
    k, groups, T, H, I = 2, 3, 40, 64, 32
    E = k * groups
    r = B.MoeRouter(B.make_config(E, k, H, T, E, 1, 1, B.MOE_ROUTE_DENSE_TP), range(E), None, [1.0] * E)
    r.set_failed_ranks([3])
    x = torch.randn(T, H, device="cuda").bfloat16()
    logits = torch.zeros(T, E, device="cuda")
    one_gu, one_dn = _weights(k, 2 * I, H, 3), _weights(k, H, I, 4)
    rep = lambda m: B.MxRows(m.codes.repeat(groups, 1, 1), m.scales.repeat(groups, 1, 1))      # noqa: E731
    gate_up, down = rep(one_gu), rep(one_dn)
    out, rows = r.mx_dispatch(logits, x)
    buf = r.mx_expert_ffn(rows, out.slot_counts, out.slot_offsets, gate_up, down)
    y = r.mx_step(logits, x, gate_up, down)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    dst, slot = out.dst_row.long().view(T, k), out.topk_slot.long()
    assert (slot != 3).all() and (slot != 2).all()            # the whole group of the lost shard is skipped
    want = buf.double()[dst].sum(1)
    assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + k * 2.0 ** -24 * buf.double()[dst].abs().sum(1)).all()
    # all groups hold the same shards: a token's rows do not depend on the group that it went to
    other = r.mx_step(logits, x.roll(1, 0), gate_up, down).roll(-1, 0)
    assert torch.equal(other, y)
    r.close()


def test_rank_order_and_lost_experts():
    """A compacted, permuted rank order moves the segments (offsets are not monotone in the slot any more) and nothing
    else; lost experts have no rows."""
    wl, inp, router, logits, x, gate_up, down = _tiny()
    dy = torch.randn_like(x)

    def run():
        out, rows = router.mx_dispatch(logits, x)
        buf = router.mx_expert_ffn(rows, out.slot_counts, out.slot_offsets, gate_up, down)
        y = router.combine(buf, x.shape[0])
        d_buf, d_w = router.combine_backward(buf, dy)
        dst = out.dst_row.long()
        return (y, d_w, buf[dst], d_buf[dst], *router.dispatch_backward(logits, d_buf, d_w)), out
    lost = np.zeros(wl.E, np.uint8)
    lost[1] = 1
    router.set_failed_ranks([2])
    router.set_failed_experts(lost)
    want, out0 = run()
    assert (out0.topk_ids != 1).all()
    alive = [q for q in range(wl.R) if q != 2]
    router.set_rank_order(alive[::-1])
    got, out1 = run()
    torch.cuda.synchronize()
    assert not torch.equal(out0.slot_offsets, out1.slot_offsets)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert router.device_status() == 0
    router.close()


def test_launches_without_overlap():
    wl, inp, router, logits, x, gate_up, down = _tiny()
    dy = torch.randn_like(x)

    def run():
        y = router.mx_step(logits, x, gate_up, down)
        d_buf, d_w = router.combine_backward(x.repeat_interleave(wl.k, 0), dy)
        return (y, d_buf, d_w, *router.dispatch_backward(logits, d_buf, d_w))
    want = [t.clone() for t in run()]
    router.set_tuning(B.MOE_TUNE_PDL, 0)
    for a, b in zip(run(), want):
        assert torch.equal(a, b)
    router.close()


@pytest.fixture
def gib():
    """gib(n): skip unless n GiB are free; what the test took goes back to the device afterwards."""
    def need(n):
        if torch.cuda.mem_get_info()[0] < n * 2 ** 30:
            pytest.skip("not enough free device memory")
    torch.cuda.empty_cache()
    yield need
    torch.cuda.empty_cache()


def test_rows_past_32_bits(gib):
    """9 GB of bf16 rows, 2.4 GB of codes; the last rows lie past 2^32 elements."""
    gib(24)
    rows, K = 70000, 65536
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    at = [0, 32767, 32768, 65535, 65536, 69999]
    part = torch.from_numpy(M.random_rows(len(at), K, 5, 3.0)).to(torch.bfloat16)
    x[at] = part.cuda()
    m = B.mx_quantize(x)
    codes, scales = M.quantize(part.double().numpy())
    assert np.array_equal(m.codes[at].cpu().numpy(), codes) and np.array_equal(m.scales[at].cpu().numpy(), scales)
    x.fill_(1.0)
    B.mx_dequantize(m, torch.bfloat16, out=x)
    assert torch.equal(x[at].double().cpu(), torch.from_numpy(M.values(codes, scales)))
    assert (x[1:32767] == 0).all() and (x[65537:69999] == 0).all()


def test_products_past_32_bits(gib):
    """Weights of 4.3 GB, of which three slots are used, and 4.6 GB of y."""
    gib(24)
    P, N, K, rows = 66, 32768, 4096, 70000
    r = B.MoeRouter(B.make_config(P, 1, 64, 16, P, 1, 1), range(P), None, [1.0] * P)
    w = B.MxRows(torch.full((P, N, K // 2), 0x22, dtype=torch.uint8, device="cuda"), torch.full((P, N, M.pitch(K)), 127, dtype=torch.uint8, device="cuda"))
    a = B.MxRows(torch.zeros((rows, K // 2), dtype=torch.uint8, device="cuda"), torch.full((rows, M.pitch(K)), 127, dtype=torch.uint8, device="cuda"))
    counts, offsets = torch.zeros(P, dtype=torch.int32, device="cuda"), torch.zeros(P + 1, dtype=torch.int32, device="cuda")
    used = {0: (0, 40), 31: (300, 33), 65: (rows - 77, 77)}
    g = torch.Generator(device="cuda").manual_seed(3)
    for p, (first, n) in used.items():
        counts[p], offsets[p] = n, first
        part = B.mx_quantize(torch.randn(n, K, device="cuda", generator=g))
        a.codes[first:first + n], a.scales[first:first + n] = part.codes, part.scales
        few = B.mx_quantize(torch.randn(256, K, device="cuda", generator=g) * K ** -0.5)
        w.codes[p, :128], w.codes[p, -128:], w.scales[p, :128], w.scales[p, -128:] = few.codes[:128], few.codes[128:], few.scales[:128], few.scales[128:]
    y = torch.full((rows, N), -7.0, dtype=torch.bfloat16, device="cuda")
    r.mx_expert_product(a, counts, offsets, w, y)
    h = r.mx_expert_gated(a, counts, offsets, w)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    val = lambda c, s: torch.from_numpy(M.values(c.cpu().numpy(), s.cpu().numpy()))      # noqa: E731
    for p, (first, n) in used.items():
        av = val(a.codes[first:first + n], a.scales[first:first + n])
        for cols in (slice(0, 128), slice(N - 128, N)):
            wv = val(w.codes[p, cols], w.scales[p, cols])
            want, mag = av @ wv.T, av.abs() @ wv.abs().T
            err = (y[first:first + n, cols].double().cpu() - want).abs()
            assert (err <= (K / 64 + 64) * 2.0 ** -23 * mag + 2.0 ** -8 * want.abs()).all()
            z = torch.nn.functional.silu(want[:, 0::2]) * want[:, 1::2]
            c = slice(cols.start // 2, cols.stop // 2)
            got = B.mx_dequantize(B.MxRows(h.codes[first:first + n], h.scales[first:first + n]), torch.float32)[:, c].double().cpu()
            # half of the largest step (2 of 4..6) under the block's scale, and the sums' own errors far below
            step = z.view(n, -1, 32).abs().amax(-1, keepdim=True).log2().floor().exp2() / 4
            assert ((got - z).view(n, -1, 32).abs() <= 2.001 * step).all()
    gap = torch.ones(rows, dtype=torch.bool)
    for first, n in used.values():
        gap[first:first + n] = False
    assert (y[gap.nonzero().flatten()[::997].cuda()] == -7).all() and (y[40] == -7).all() and (y[rows - 78] == -7).all()
    r.close()


def test_dispatch_and_gradients_past_32_bits(gib):
    """A send buffer of 4.8 GB of codes, rows of 4.6 GB in the gradients."""
    gib(60)
    E, k, H = 16, 8, 7168
    T = 42000
    r = B.MoeRouter(B.make_config(E, k, H, T, E, 1, 1), range(E), None, [1.0] * E)
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(T, E, device="cuda", generator=g)
    x = torch.randn(T, H, device="cuda", generator=g, dtype=torch.bfloat16)
    out = r.dispatch(logits, x)
    dst = out.dst_row.long().view(T, k)
    dx, _ = r.dispatch_backward(None, out.send_buf)
    d_buf, d_w = r.combine_backward(out.send_buf, x)
    torch.cuda.synchronize()
    assert r.device_status() == 0
    for part in (slice(0, 500), slice(T // 2, T // 2 + 500), slice(T - 500, T)):
        xs = x[part].double()
        assert torch.equal(dx[part], (8 * xs).bfloat16())                        # the sum of k copies, exact
        want = out.topk_weights[part].double()[..., None] * xs[:, None]
        assert ((d_buf[dst[part].flatten()].double().view(-1, k, H) - want).abs() <= 2.0 ** -8 * want.abs()).all()
        sq = (xs * xs).sum(-1, keepdim=True)
        assert ((d_w[part].double() - sq).abs() <= (H / 256 + 34) * 2.0 ** -24 * sq).all()
    r.close()
    del out, dx, d_buf, d_w, dst
    torch.cuda.empty_cache()
    T = 168000
    r = B.MoeRouter(B.make_config(E, k, H, T, E, 1, 1), range(E), None, [1.0] * E)
    logits = torch.randn(T, E, device="cuda", generator=g)
    x = x.repeat(4, 1)
    out, rows = r.mx_dispatch(logits, x)
    one = B.mx_quantize(x[:T // 4])
    dst = out.dst_row.long().view(T, k)
    for part in (slice(0, 2000), slice(T - 2000, T)):
        t = torch.arange(part.start, part.stop, device="cuda") % (T // 4)
        for j in range(k):
            assert torch.equal(rows.codes[dst[part, j]], one.codes[t]) and torch.equal(rows.scales[dst[part, j]], one.scales[t])
    assert r.device_status() == 0
    r.close()
