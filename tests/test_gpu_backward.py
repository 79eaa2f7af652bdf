"""Gradients of combine and dispatch against the formulas in 64 bits, and of the formulas against differences.

Bounds: d_expert_buf is one fp32 product rounded to bf16 (2^-8 relative covers half a bf16 step of 2^-9 and
the fp32 roundings).  d_weights is an fp32 sum of H exact-in-fp32 products of bf16 numbers (16 significant
bits): with fused adds its error is at most (H / lanes + log) roundings, bounded by (H / 256 + 32) * 2^-24 of
sum |a b|, and a last product.  dx is k fp32 additions and one rounding.  d_logits is a handful of fp32
operations of magnitude w (|g| + sum w |g|): 16 k of 2^-24 of that; sigmoid_spec is within 3e-7 of the sigmoid."""
import numpy as np
import pytest
import torch

from gpu_util import make_router, to_dev
from paper_2602_21140_b200 import binding as B
from paper_2602_21140_b200 import workloads as W

pytestmark = pytest.mark.gpu

CASES = [("tiny", 1, 8), ("tiny", 128, 256), ("mixtral", 65, 4096), ("dsv3", 33, 7168), ("dsv3", 700, 72), ("kimi", 70, 264),
         ("qwen3", 257, 1000), ("mixtral", 3, 16392)]


def _forward(name, T, H, route_scale=1.0, score=None):
    wl = W.WORKLOADS[name]
    inp = W.make_inputs(wl, T=T, H=H)
    router = make_router(wl, inp, max_tokens=T, hidden=H, route_scale=route_scale)
    router.set_failed_ranks(wl.failure_sets[-1])
    logits, x = to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16)
    out = router.dispatch(logits, x)
    return wl, inp, router, logits, x, out


def _weights(logits, ids, sigmoid, scale):
    """w [T,k] from f64 logits at fixed ids."""
    lg = logits.gather(1, ids)
    u = torch.sigmoid(lg) if sigmoid else torch.exp(lg - lg.max(1, keepdim=True).values.detach())
    return scale * u / u.sum(1, keepdim=True)


@pytest.mark.parametrize("name,T,H", CASES)
def test_combine_backward(name, T, H):
    wl, inp, router, logits, x, out = _forward(name, T, H)
    n = T * wl.k
    g = torch.Generator(device="cuda").manual_seed(T)
    buf = torch.randn(n, H, device="cuda", generator=g).bfloat16()
    dy = torch.randn(T, H, device="cuda", generator=g).bfloat16()
    d_buf = torch.full((n, H), float("nan"), device="cuda", dtype=torch.bfloat16)
    d_buf, d_w = router.combine_backward(buf, dy, d_buf)
    torch.cuda.synchronize()
    dst = out.dst_row.long().view(T, wl.k)
    scale = to_dev(inp["slot_scale"]).double()[out.topk_slot.long()]
    coef = out.topk_weights.double() * scale
    want = torch.empty(n, H, dtype=torch.float64, device="cuda")
    want[dst.flatten()] = (coef[..., None] * dy.double()[:, None]).flatten(0, 1)
    assert ((d_buf.double() - want).abs() <= 2.0 ** -8 * want.abs()).all()
    prod = buf.double()[dst] * dy.double()[:, None]
    want_w, mag = scale * prod.sum(-1), scale.abs() * prod.abs().sum(-1)
    assert ((d_w.double() - want_w).abs() <= (H / 256 + 34) * 2.0 ** -24 * mag).all()
    router.close()


@pytest.mark.parametrize("route_scale", [1.0, 2.5])
@pytest.mark.parametrize("name,T,H", CASES)
def test_dispatch_backward(name, T, H, route_scale):
    wl, inp, router, logits, x, out = _forward(name, T, H, route_scale)
    sigmoid = wl.score_func == W.SIGMOID
    g = torch.Generator(device="cuda").manual_seed(T)
    d_send = torch.randn(T * wl.k, H, device="cuda", generator=g).bfloat16()
    d_w = torch.randn(T, wl.k, device="cuda", generator=g)
    d_logits = torch.full((T, wl.E), float("nan"), device="cuda")
    dx, d_logits = router.dispatch_backward(logits, d_send, d_w, d_logits=d_logits)
    torch.cuda.synchronize()
    dst, ids = out.dst_row.long().view(T, wl.k), out.topk_ids.long()
    rows = d_send.double()[dst]
    want, mag = rows.sum(1), rows.abs().sum(1)
    assert ((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + wl.k * 2.0 ** -24 * mag).all()
    leaf = logits.double().requires_grad_()
    w = _weights(leaf, ids, sigmoid, route_scale)
    (w * d_w.double()).sum().backward()
    wm = w.detach()
    bound = wm * (d_w.double().abs() + (wm * d_w.double().abs()).sum(1, keepdim=True) / route_scale)
    tol = torch.zeros(T, wl.E, dtype=torch.float64, device="cuda").scatter_(1, ids, bound * (16 * wl.k * 2.0 ** -24 + 3e-7))
    assert ((d_logits.double() - leaf.grad).abs() <= tol).all()
    # without gate gradients: the rows alone, the same bits
    dx2, none = router.dispatch_backward(None, d_send)
    assert none is None and torch.equal(dx2, dx)
    router.close()


@pytest.mark.parametrize("E,k,H,T", [(16, 1, 40, 70), (24, 3, 8200, 9), (64, 6, 2048, 333), (32, 16, 264, 41), (8, 8, 64, 5)])
def test_any_number_of_experts_per_token(E, k, H, T):
    """The kernels that are not built for one k, one token with every expert, rows of more than one ring slot; on a
    stream of its own."""
    cfg = B.make_config(E, k, H, T, E, 1, 1, B.MOE_SCORE_SIGMOID, route_scale=1.5)
    scale = np.linspace(0.5, 1.5, E).astype(np.float32)
    router = B.MoeRouter(cfg, range(E), np.zeros(E, np.float32), scale)
    g = torch.Generator(device="cuda").manual_seed(E)
    logits = torch.randn(T, E, device="cuda", generator=g)
    x, dy = (torch.randn(T, H, device="cuda", generator=g).bfloat16() for _ in range(2))
    buf, d_send = (torch.randn(T * k, H, device="cuda", generator=g).bfloat16() for _ in range(2))
    d_w = torch.randn(T, k, device="cuda", generator=g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = router.dispatch(logits, x)
        d_buf, got_w = router.combine_backward(buf, dy)
        dx, d_logits = router.dispatch_backward(logits, d_send, d_w)
    side.synchronize()
    assert router.device_status() == 0
    dst, ids = out.dst_row.long().view(T, k), out.topk_ids.long()
    sc = torch.from_numpy(scale).cuda().double()[out.topk_slot.long()]
    prod = buf.double()[dst] * dy.double()[:, None]
    assert ((got_w.double() - sc * prod.sum(-1)).abs() <= (H / 256 + 34) * 2.0 ** -24 * sc * prod.abs().sum(-1)).all()
    want = torch.empty(T * k, H, dtype=torch.float64, device="cuda")
    want[dst.flatten()] = ((out.topk_weights.double() * sc)[..., None] * dy.double()[:, None]).flatten(0, 1)
    assert ((d_buf.double() - want).abs() <= 2.0 ** -8 * want.abs()).all()
    rows = d_send.double()[dst]
    assert ((dx.double() - rows.sum(1)).abs() <= 2.0 ** -8 * rows.sum(1).abs() + k * 2.0 ** -24 * rows.abs().sum(1)).all()
    leaf = logits.double().requires_grad_()
    w = _weights(leaf, ids, True, 1.5)
    (w * d_w.double()).sum().backward()
    wm, gm = w.detach(), d_w.double().abs()
    tol = torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter_(
        1, ids, wm * (gm + (wm * gm).sum(1, keepdim=True) / 1.5) * (16 * k * 2.0 ** -24 + 3e-7))
    assert ((d_logits.double() - leaf.grad).abs() <= tol).all()
    router.close()


def test_formula_against_differences():
    """d loss / d logits and d x by central differences of the forward formula in 64 bits (T, E small)."""
    for name in ("tiny", "dsv3"):
        wl, inp, router, logits, x, out = _forward(name, 4, 64, 1.5)
        sigmoid = wl.score_func == W.SIGMOID
        T, k, H = 4, wl.k, 64
        g = torch.Generator(device="cuda").manual_seed(3)
        dy = torch.randn(T, H, device="cuda", generator=g).bfloat16()
        # an "expert" that squares its rows: buf = send^2, so d_send = 2 send d_buf
        send = out.send_buf.double()
        buf = (send ** 2).bfloat16()
        d_buf, d_w = router.combine_backward(buf, dy)
        d_send = (2 * send * d_buf.double()).bfloat16()
        dx, d_logits = router.dispatch_backward(logits, d_send, d_w)
        ids, slot = out.topk_ids.long(), out.topk_slot.long()
        scale = to_dev(inp["slot_scale"]).double()[slot]

        def loss(lg, xx):
            w = _weights(lg, ids, sigmoid, 1.5) * scale
            y = (w.sum(1, keepdim=True)) * xx ** 2           # every expert squares the same row
            return (y * dy.double()).sum()
        lg0, x0, h = logits.double(), x.double(), 1e-5
        for t in range(T):
            for e in list(ids[t, :2].tolist()) + [int(ids[t].max()) // 2]:
                step = torch.zeros_like(lg0); step[t, e] = h
                diff = (loss(lg0 + step, x0) - loss(lg0 - step, x0)) / (2 * h)
                if e not in ids[t].tolist():
                    assert d_logits[t, e] == 0 and abs(diff) < 1e-9
                else:
                    # buf is rounded to bf16 before the dot product: 2^-8 of sum |buf dy| times the weight's slope
                    mag = (x0[t] ** 2 * dy[t].double().abs()).sum() * scale[t].max() * 1.5
                    assert abs(d_logits[t, e].double() - diff) <= 2.0 ** -8 * 2 * mag
            for c in (0, 17, 63):
                step = torch.zeros_like(x0); step[t, c] = h
                diff = (loss(lg0, x0 + step) - loss(lg0, x0 - step)) / (2 * h)
                # d_buf, d_send and dx are each rounded to bf16
                assert abs(dx[t, c].double() - diff) <= 4 * 2.0 ** -8 * diff.abs() + 1e-6
        router.close()


def test_after_a_dispatch_of_4_bit_rows_and_in_a_graph():
    wl = W.WORKLOADS["dsv3"]
    T, H = 50, 96
    inp = W.make_inputs(wl, T=T, H=H)
    router = make_router(wl, inp, max_tokens=T, hidden=H)
    logits, x = to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16)
    n = T * wl.k
    buf, dy = torch.randn(n, H, device="cuda").bfloat16(), torch.randn(T, H, device="cuda").bfloat16()
    out, _ = router.mx_dispatch(logits, x)
    d_buf, d_w = router.combine_backward(buf, dy)
    dx, d_logits = router.dispatch_backward(logits, d_buf, d_w)
    got = [torch.zeros_like(t) for t in (d_buf, d_w, dx, d_logits)]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        router.combine_backward(buf, dy, got[0], got[1])
        router.dispatch_backward(logits, got[0], got[1], got[2], got[3])
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, (d_buf, d_w, dx, d_logits)):
        assert torch.equal(a, b)
    assert router.device_status() == 0
    router.close()


def test_logits_at_the_edges():
    """Saturated sigmoids keep their slope (1 - s without cancellation), masked logits get 0."""
    E, k, H, T = 8, 2, 32, 3
    for sigmoid in (0, 1):
        cfg = B.make_config(E, k, H, T, 4, 2, 1, sigmoid)
        router = B.MoeRouter(cfg, list(range(E)), None, [1.0] * E)
        lg = torch.full((T, E), float("-inf"), device="cuda")
        lg[0, [1, 5]] = torch.tensor([30.0, 25.0], device="cuda")
        lg[1, [0, 7]] = torch.tensor([-30.0, -40.0], device="cuda")
        lg[2, [2, 3]] = torch.tensor([20.0, -20.0], device="cuda")
        out = router.dispatch(lg, torch.zeros(T, H, device="cuda", dtype=torch.bfloat16))
        d_w = torch.tensor([[1.0, -2.0], [0.5, 3.0], [-1.0, 1.0]], device="cuda")
        _, d = router.dispatch_backward(lg, out.send_buf, d_w)
        # The 64-bit value without cancellation: w_j sum_i w_i (g_j - g_i) (the w add up to 1), times the slope
        # sigmoid(-l).  (Differentiating u / sum(u) in 64 bits gives 0 for the 8e-18 of the last row: its terms
        # are 1 - 1 at 2^-53.)
        ids, g = out.topk_ids.long(), d_w.double()
        w = _weights(lg.double(), ids, sigmoid, 1.0)
        part = w * (w[:, None, :] * (g[:, :, None] - g[:, None, :])).sum(2)
        if sigmoid:
            part = part * torch.sigmoid(-lg.double().gather(1, ids))
        want = torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter_(1, ids, part)
        # k = 2: one difference, so every step is relative: under 40 fp32 roundings, and 3e-7 of the spec's sigmoid
        # in each of w and the slope
        assert ((d.double() - want).abs() <= (40 * 2.0 ** -24 + 3 * 3e-7) * want.abs()).all()
        assert (d[lg == float("-inf")] == 0).all()
        router.close()


def test_guard_zones():
    wl, inp, router, logits, x, out = _forward("kimi", 37, 264)
    T, H, n = 37, 264, 37 * wl.k
    d_send = torch.randn(n, H, device="cuda").bfloat16()
    dy, d_w = torch.randn(T, H, device="cuda").bfloat16(), torch.randn(T, wl.k, device="cuda")
    made = {}
    for name, shape, dt in (("d_buf", (n, H), torch.bfloat16), ("d_w", (T, wl.k), torch.float32), ("dx", (T, H), torch.bfloat16),
                            ("d_logits", (T, wl.E), torch.float32)):
        m = int(np.prod(shape))
        whole = torch.full((m + 128,), -3.0, dtype=dt, device="cuda")
        made[name] = (whole, whole[64:64 + m].view(shape))
    router.combine_backward(d_send, dy, made["d_buf"][1], made["d_w"][1])
    router.dispatch_backward(logits, d_send, d_w, made["dx"][1], made["d_logits"][1])
    torch.cuda.synchronize()
    for whole, _ in made.values():
        assert (whole[:64] == -3).all() and (whole[-64:] == -3).all()
    router.close()


def test_refusals():
    wl, inp, router, logits, x, out = _forward("tiny", 8, 64)
    n = 8 * wl.k
    buf, dy = torch.zeros(n, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(8, 64, device="cuda", dtype=torch.bfloat16)
    d_w = torch.zeros(8, wl.k, device="cuda")
    bad = [
        lambda: router.combine_backward(buf, dy[:7]),                               # rows of another T
        lambda: router.combine_backward(buf[:, :56], dy),
        lambda: router.combine_backward(buf, dy, buf),                              # in place
        lambda: router.combine_backward(buf.float(), dy),
        lambda: router.combine_backward(buf.cpu(), dy),
        lambda: router.dispatch_backward(logits, buf[:n - wl.k]),                   # T - 1 tokens
        lambda: router.dispatch_backward(logits, buf[:n - 1]),
        lambda: router.dispatch_backward(logits, buf, d_w.double()),
        lambda: router.dispatch_backward(logits, buf, None, None, torch.zeros(8, wl.E, device="cuda")),
        lambda: router.dispatch_backward(logits[:, :4], buf, d_w),
    ]
    for call in bad:
        with pytest.raises(B.MoeError):
            call()
    assert B.moe_combine_backward(router._ctx, buf.data_ptr() + 2, dy.data_ptr(), 8, dy.data_ptr(), d_w.data_ptr()) == B.MOE_ERR_INVALID_ARG
    assert B.moe_combine_backward(router._ctx, 0, dy.data_ptr(), 8, buf.data_ptr(), d_w.data_ptr()) == B.MOE_ERR_INVALID_ARG
    router.close()
    fresh = make_router(wl, inp, max_tokens=8, hidden=64)
    with pytest.raises(B.MoeError):
        fresh.combine_backward(buf, dy)                                             # nothing was dispatched
    with pytest.raises(B.MoeError):
        fresh.dispatch_backward(logits, buf)
    fresh.close()
    sig = W.WORKLOADS["dsv3"]
    si = W.make_inputs(sig, T=4, H=64)
    r = make_router(sig, si, max_tokens=4, hidden=64)
    o = r.dispatch(to_dev(si["logits"]), to_dev(si["x"], torch.bfloat16))
    with pytest.raises(B.MoeError):                                                 # sigmoid scores need the logits
        r.dispatch_backward(None, o.send_buf, torch.zeros(4, 8, device="cuda"))
    r.close()
    dense = B.MoeRouter(B.make_config(4, 2, 64, 8, 4, 1, 1, B.MOE_ROUTE_DENSE_TP), range(4), None, [1.0] * 4)
    o = dense.dispatch(torch.zeros(8, 4, device="cuda"), x)
    dx, none = dense.dispatch_backward(None, o.send_buf)
    assert none is None and torch.equal(dx, (2 * x.float()).bfloat16())
    with pytest.raises(B.MoeError):                                                 # its weights are constants
        dense.dispatch_backward(torch.zeros(8, 4, device="cuda"), o.send_buf, torch.zeros(8, 2, device="cuda"))
    dense.close()
