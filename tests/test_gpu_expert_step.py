"""A layer with experts in 16 bits as it is trained: norm, dispatch, experts, combine, and back, with what is kept in 8 bits."""
import pytest
import torch

import expert_util as U
from paper_2602_21140_b200 import binding as B

pytestmark = pytest.mark.gpu

E, K, H, I = 12, 3, 256, 96


def _layer(T, sigmoid=False, failed=(), spare=4):
    """E experts on P = E + spare slots of 4 ranks, the first ones twice."""
    P = E + spare
    s2e = [p if p < E else p - E for p in range(P)]
    cfg = B.make_config(E, K, H, max(T, 1), 4, P // 4, 2, int(sigmoid))
    r = B.MoeRouter(cfg, s2e, [0.0] * E if sigmoid else None, [1.0] * P)
    r.set_failed_ranks(failed)
    w = [U.bf16(E, 2 * I, H, seed=1, scale=H ** -0.5), U.bf16(E, H, I, seed=2, scale=I ** -0.5)]
    return r, s2e, [m[torch.tensor(s2e, device="cuda")].contiguous() for m in w]


@pytest.mark.parametrize("T,failed", [(1, ()), (37, (1,)), (700, (3,))])
def test_redispatch_is_the_dispatch_of_the_kept_values(T, failed):
    r, _, _ = _layer(T, failed=failed)
    logits, x = torch.randn(T, E, device="cuda"), U.bf16(T, H, seed=3)
    y8 = B.rms_norm(x, torch.ones(H, device="cuda"), keep=True).y8
    want = r.dispatch(logits, B.mx8_dequantize(y8)).send_buf
    whole = torch.full((T * K + 3, H), -7.0, dtype=torch.bfloat16, device="cuda")
    got = r.redispatch(y8, whole[:T * K])
    assert torch.equal(got, want) and (whole[T * K:] == -7).all()
    r.mx_dispatch(logits, x)                                    # after a dispatch of 4-bit rows as well
    assert torch.equal(r.redispatch(y8), want)
    with pytest.raises(B.MoeError):
        r.redispatch(B.mx8_empty(T + 1, H))
    r.close()


@pytest.mark.parametrize("T", [1, 37, 3000])
def test_rows_of_many_widths(T):
    """Rows shorter and longer than a warp's piece."""
    for width in (32, 1024, 1056, 7168):
        r = B.MoeRouter(B.make_config(4, 2, width, T, 1, 4, 1), range(4), None, [1.0] * 4)
        logits, x = torch.randn(T, 4, device="cuda"), U.bf16(T, width, seed=3)
        y8 = B.rms_norm(x, torch.ones(width, device="cuda"), keep=True).y8
        want = r.dispatch(logits, B.mx8_dequantize(y8)).send_buf
        assert torch.equal(r.redispatch(y8), want)
        r.close()


@pytest.mark.parametrize("T,sigmoid", [(1, False), (50, True), (2000, False)])
def test_a_step_and_its_gradients(T, sigmoid):
    """expert_step and expert_step_backward are the operators one after the other, and the whole agrees with the layer's
    gradients in 64 bits to what its roundings to bf16 (five on the longest way, two of them of sums) and to 8 bits allow."""
    r, s2e, (gate_up, down) = _layer(T, sigmoid, failed=(2,))
    logits, stream, res = torch.randn(T, E, device="cuda"), U.bf16(T, H, seed=3), U.bf16(T, H, seed=4)
    norm_w = 1 + 0.1 * torch.randn(H, device="cuda")
    dy, d_stream = U.bf16(T, H, seed=5), U.bf16(T, H, seed=6)
    P, n = r.num_slots, T * K
    out, buf, z = r.alloc_outputs(T), torch.empty(n, H, dtype=torch.bfloat16, device="cuda"), B.mx8_empty(n, 2 * I)
    norm = B.rms_norm(stream, norm_w, res, keep=True)
    y = r.expert_step(logits, norm.y, gate_up, down, out, buf=buf, z=z)
    dx, d_logits, d_gate_up, d_down = r.expert_step_backward(logits, dy, norm.y8, out, buf, z, gate_up, down, grad_dtype=torch.float32)
    d_h, d_norm = B.rms_norm_backward(dx, norm.h, norm.rstd, norm_w, d_stream)
    torch.cuda.synchronize()
    assert r.device_status() == 0

    # step by step
    o2 = r.dispatch(logits, norm.y)
    b2 = r.expert_ffn(o2.send_buf, o2.slot_counts, o2.slot_offsets, gate_up, down)
    assert torch.equal(b2, buf) and torch.equal(r.combine(b2, T), y)
    d_buf, d_w = r.combine_backward(buf, dy)
    rows = r.redispatch(norm.y8)
    d_rows, g1, g2 = r.expert_ffn_backward(d_buf, rows, o2.slot_counts, o2.slot_offsets, gate_up, down, z, grad_dtype=torch.float32)
    dx2, dl2 = r.dispatch_backward(logits, d_rows, d_w)
    for a, b in ((g1, d_gate_up), (g2, d_down), (dx2, dx), (dl2, d_logits)):
        assert torch.equal(a, b)

    # the layer in 64 bits, differentiated by autograd
    leaf = lambda t: t.double().clone().requires_grad_()       # noqa: E731
    h, l, wg, wd, wn = leaf(norm.h), leaf(logits), leaf(gate_up), leaf(down), leaf(norm_w)
    xn = h * (h.square().mean(1, keepdim=True) + 1e-6).rsqrt() * wn
    u = (torch.sigmoid(l) if sigmoid else torch.exp(l)).gather(1, out.topk_ids.long())
    w = u / u.sum(1, keepdim=True)
    total = 0
    for j in range(K):
        slot = out.topk_slot[:, j].long()
        for p in slot.unique().tolist():
            t = slot == p
            v = xn[t] @ wg[p].T
            e = (torch.nn.functional.silu(v[:, 0::2]) * v[:, 1::2]) @ wd[p].T
            total = total + (w[t, j, None] * e * dy[t].double()).sum()
    (total + (h * d_stream.double()).sum()).backward()
    # An element of the 8-bit rows is off by 2^-4 of itself at most, uniformly 2^-4 / sqrt(3) or less in the mean: what is
    # linear in them (all gradients are, in z and in the rows) by the same part of its norm at most, twice on the way to d_gate_up.
    for got, want, part in ((dx_of(d_h, d_stream), h.grad - d_stream.double(), 0.1), (d_norm, wn.grad, 0.1), (d_logits, l.grad, 0.02),
                            (d_gate_up, wg.grad, 0.15), (d_down, wd.grad, 0.1)):
        assert float((got.double() - want).norm()) <= part * float(want.norm()) + 1e-12
    # with everything kept in 16 bits: roundings of 2^-9 in the mean
    z16 = torch.empty(n, 2 * I, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(r.expert_step(logits, norm.y, gate_up, down, out, buf=buf, z=z16), y)
    dx, d_logits, d_gate_up, d_down = r.expert_step_backward(logits, dy, out.send_buf, out, buf, z16, gate_up, down, grad_dtype=torch.float32)
    d_h, d_norm = B.rms_norm_backward(dx, norm.h, norm.rstd, norm_w, d_stream)
    for got, want in ((dx_of(d_h, d_stream), h.grad - d_stream.double()), (d_norm, wn.grad), (d_logits, l.grad), (d_gate_up, wg.grad), (d_down, wd.grad)):
        assert float((got.double() - want).norm()) <= 0.015 * float(want.norm()) + 1e-12
    r.close()


def dx_of(d_h, d_stream):
    return d_h.double() - d_stream.double()


def test_gradients_against_differences():
    """One slot's network: the loss in 64 bits at the matrices a little to either side."""
    r = U.make_router(1)
    n_, off, n = U.layout([70])
    a, dy = U.bf16(n, 64, seed=1), U.bf16(n, 64, seed=2)
    gate_up, down = U.bf16(1, 96, 64, seed=3, scale=0.125), U.bf16(1, 64, 48, seed=4, scale=0.14)
    z = torch.empty(n, 96, dtype=torch.bfloat16, device="cuda")
    r.expert_ffn(a, n_, off, gate_up, down, z=z)
    grads = r.expert_ffn_backward(dy, a, n_, off, gate_up, down, z, grad_dtype=torch.float32)

    def loss(x, g, d):
        v = x @ g[0].T
        return (((torch.nn.functional.silu(v[:, 0::2]) * v[:, 1::2]) @ d[0].T) * dy.double()).sum()

    at, e = [t.double() for t in (a, gate_up, down)], 2.0 ** -18
    for i, got in enumerate(grads):
        for s in range(3):
            u = torch.randn(at[i].shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(s))
            up, dn = list(at), list(at)
            up[i], dn[i] = at[i] + e * u, at[i] - e * u
            diff = (loss(*up) - loss(*dn)) / (2 * e)
            # z, h, dz and the result are rounded by 2^-8 of themselves at most, and each of them scales a term of the sum
            assert abs(float((u * got.double()).sum() - diff)) <= 4 * 2.0 ** -8 * float((u * got.double()).abs().sum())
    r.close()


def test_a_backward_pass_captured_while_an_eager_graph_of_the_same_leaves_lives():
    r, _, (gate_up, down) = _layer(64)
    logits, x, dy = torch.randn(64, E, device="cuda"), U.bf16(64, H, seed=3), U.bf16(64, H, seed=4)
    leaf = x.clone().requires_grad_()
    alive = (leaf.float() ** 2).sum()                           # an autograd graph of the same tensor, not run yet
    out, buf, z = r.alloc_outputs(64), torch.empty(64 * K, H, dtype=torch.bfloat16, device="cuda"), B.mx8_empty(64 * K, 2 * I)
    xd = leaf.detach()

    def step():
        y = r.expert_step(logits, xd, gate_up, down, out, buf=buf, z=z)
        return (y, *r.expert_step_backward(logits, dy, out.send_buf, out, buf, z, gate_up, down))

    want = step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    alive.backward()
    assert torch.isfinite(leaf.grad).all()
    del graph
    r.close()


def test_another_dispatch_in_between_is_refused():
    r, _, (gate_up, down) = _layer(32)
    logits, x, dy = torch.randn(32, E, device="cuda"), U.bf16(32, H, seed=3), U.bf16(32, H, seed=4)
    out, buf, z = r.alloc_outputs(32), torch.empty(32 * K, H, dtype=torch.bfloat16, device="cuda"), B.mx8_empty(32 * K, 2 * I)
    r.expert_step(logits, x, gate_up, down, out, buf=buf, z=z)
    want = r.expert_step_backward(logits, dy, out.send_buf, out, buf, z, gate_up, down)
    r.dispatch(logits.flip(0).contiguous(), x)
    with pytest.raises(B.MoeError):
        r.expert_step_backward(logits, dy, out.send_buf, out, buf, z, gate_up, down)
    r.expert_step(logits, x, gate_up, down, out, buf=buf, z=z)
    got = r.expert_step_backward(logits, dy, out.send_buf, out, buf, z, gate_up, down)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    r.close()


def test_no_tokens_and_dense_routing():
    r, _, (gate_up, down) = _layer(8)
    logits, x = torch.randn(0, E, device="cuda"), torch.empty(0, H, dtype=torch.bfloat16, device="cuda")
    out, buf, z = r.alloc_outputs(0), x.clone(), B.mx8_empty(0, 2 * I)
    out.slot_counts.zero_(); out.slot_offsets.zero_()           # a dispatch of no tokens writes nothing
    assert r.expert_step(logits, x, gate_up, down, out, buf=buf, z=z).shape == (0, H)
    dx, d_logits, d_gate_up, d_down = r.expert_step_backward(logits, x, B.mx8_empty(0, H), out, buf, z, gate_up, down)
    assert dx.shape == (0, H) and d_logits.shape == (0, E) and not d_gate_up.any() and not d_down.any()
    r.close()
    k, groups, T = 2, 3, 40
    n = k * groups
    r = B.MoeRouter(B.make_config(n, k, H, T, n, 1, 1, B.MOE_ROUTE_DENSE_TP), range(n), None, [1.0] * n)
    r.set_failed_ranks([3])
    gate_up, down = U.bf16(n, 2 * I, H, seed=1, scale=H ** -0.5), U.bf16(n, H, I, seed=2, scale=I ** -0.5)
    logits, x, dy = torch.zeros(T, n, device="cuda"), U.bf16(T, H, seed=3), U.bf16(T, H, seed=4)
    out, buf, z = r.alloc_outputs(T), torch.empty(T * k, H, dtype=torch.bfloat16, device="cuda"), B.mx8_empty(T * k, 2 * I)
    r.expert_step(logits, x, gate_up, down, out, buf=buf, z=z)
    dx, d_logits, _, d_down = r.expert_step_backward(None, dy, out.send_buf, out, buf, z, gate_up, down)
    torch.cuda.synchronize()
    assert d_logits is None and torch.isfinite(dx).all() and not d_down[3].any() and d_down[0].any() and r.device_status() == 0
    r.close()
