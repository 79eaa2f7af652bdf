"""Dispatch with 4-bit rows: the same routing as moe_dispatch (checked against the oracle), the rows against
the format written out in 64 bits; and the whole layer, dispatch -> experts -> combine."""
import numpy as np
import pytest
import torch

import mx_util as M
import oracle
from gpu_util import check_dispatch, make_router, to_dev
from paper_2602_21140_b200 import binding as B
from paper_2602_21140_b200 import workloads as W
from util import oracle_cfg

pytestmark = pytest.mark.gpu


def _x64(inp):
    return W.bf16_bits_to_f32(inp["x"]).astype(np.float64)


def _check(wl, inp, failed, out, rows):
    bias = inp["bias"] if wl.score_func == W.SIGMOID else None
    ref = oracle.dispatch(oracle_cfg(wl), inp["slot_to_expert"], failed, bias, inp["logits"], inp["x"])
    check_dispatch(out, ref, check_send=False)
    codes, scales = M.quantize(_x64(inp))
    src = ref["src_index"] // wl.k
    assert np.array_equal(rows.codes.cpu().numpy(), codes[src])
    assert np.array_equal(rows.scales.cpu().numpy(), scales[src])
    return ref


@pytest.mark.parametrize("name,T,H", [("tiny", 1, 32), ("tiny", 128, 256), ("dsv3", 33, 7168), ("kimi", 65, 544), ("qwen3", 257, 1056),
                                      ("mixtral", 100, 4096), ("dsv3", 2500, 96), ("mixtral", 2400, 2080)])
def test_rows_and_routing(name, T, H):
    wl = W.WORKLOADS[name]
    inp = W.make_inputs(wl, T=T, H=H)
    router = make_router(wl, inp, max_tokens=T, hidden=H)
    logits, x = to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16)
    for failed in wl.failure_sets[:2]:
        router.set_failed_ranks(failed)
        out, rows = router.mx_dispatch(logits, x)
        torch.cuda.synchronize()
        assert router.device_status() == 0
        _check(wl, inp, failed, out, rows)
    router.close()


def test_non_finite_rows():
    wl = W.WORKLOADS["tiny"]
    inp = W.make_inputs(wl, T=20, H=256)
    for t, bits in ((3, 0x7F80), (9, 0x7FC0), (11, 0xFF80)):
        inp["x"][t, 40] = bits
    router = make_router(wl, inp, max_tokens=20, hidden=256)
    out, rows = router.mx_dispatch(to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16))
    _check(wl, inp, (), out, rows)
    router.close()


def test_guard_zones_and_no_tokens():
    wl = W.WORKLOADS["qwen3"]
    T, H = 37, 1056
    inp = W.make_inputs(wl, T=T, H=H)
    router = make_router(wl, inp, max_tokens=T, hidden=H)
    n, p = T * wl.k, M.pitch(H)
    c = torch.full((n * H // 2 + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.full((n * p + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    rows = B.MxRows(c[32:-32].view(n, H // 2), s[32:-32].view(n, p))
    out, _ = router.mx_dispatch(to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16), rows=rows)
    _check(wl, inp, (), out, rows)
    for t in (c, s):
        assert (t[:32] == 0xAB).all() and (t[-32:] == 0xAB).all()
    empty = router.mx_dispatch(torch.empty(0, wl.E, device="cuda"), torch.empty(0, H, device="cuda", dtype=torch.bfloat16))
    assert empty[1].codes.shape == (0, H // 2)
    assert router.combine(torch.empty(0, H, device="cuda", dtype=torch.bfloat16), 0).shape == (0, H)
    router.close()


def _layer(wl, inp, T, H, I, seed):
    """Weights of every slot (replicas of an expert share theirs) and the layer's output in 64 bits."""
    gu = M.random_rows(wl.E * 2 * I, H, seed).reshape(wl.E, 2 * I, H) * H ** -0.5
    dn = M.random_rows(wl.E * H, I, seed + 1).reshape(wl.E, H, I) * I ** -0.5
    s2e = np.maximum(inp["slot_to_expert"], 0)
    pair = []
    for w in (gu, dn):
        c, s = M.quantize(w)
        pair.append((B.MxRows(torch.from_numpy(c[s2e]).cuda(), torch.from_numpy(s[s2e]).cuda()), M.values(c, s)))
    return pair


def _expected(wl, inp, ref, gu, dn):
    """(y, bound): every chosen expert in 64 bits.  The 4-bit rounding of h can fall the other way where the
    kernel's h is off by its error e; such an element moves by at most one step, a third of its block's
    largest magnitude, so y moves by at most |down| @ (that step) where the bracket of h is not one value."""
    x = M.values(*M.quantize(_x64(inp)))
    T, H = x.shape
    K = H
    y, tol = np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        for j in range(wl.k):
            e, slot = ref["topk_ids"][t, j], ref["topk_slot"][t, j]
            coef = float(np.float32(ref["topk_weights"][t, j]) * np.float32(inp["slot_scale"][slot]))
            s = gu[e] @ x[t]
            mag = (K / 64 + 64) * 2.0 ** -23 * (np.abs(gu[e]) @ np.abs(x[t]))
            g, u = s[0::2], s[1::2]
            silu = g / (1 + np.exp(-g))
            h = silu * u
            err = 1.1 * mag[0::2] * (np.abs(u) + mag[1::2]) + np.abs(silu) * mag[1::2] + (8 + np.abs(g)) * 2.0 ** -23 * np.abs(h)
            hq = M.values(*M.quantize(h))
            lo, hi = M.values(*M.quantize(h - err)), M.values(*M.quantize(h + err))
            flip = np.maximum(np.abs(lo - hq), np.abs(hi - hq))
            out = dn[e] @ hq
            moved = np.abs(dn[e]) @ flip + (h.size / 64 + 64) * 2.0 ** -23 * (np.abs(dn[e]) @ np.abs(hq))
            y[t] += coef * out
            tol[t] += abs(coef) * (moved + 2.0 ** -8 * np.abs(out))          # the expert's row is bf16
    return y, tol + 2.0 ** -8 * np.abs(y) + wl.k * 2.0 ** -24 * np.abs(y)


def test_whole_layer():
    """dispatch -> gated product -> product -> combine, with a failed rank, eagerly and as a replayed graph
    across remaps."""
    wl = W.WORKLOADS["tiny"]
    T, H, I = 96, 256, 160
    inp = W.make_inputs(wl, T=T, H=H)
    router = make_router(wl, inp, max_tokens=T, hidden=H)
    (gate_up, gu), (down, dn) = _layer(wl, inp, T, H, I, 21)
    logits, x = to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16)
    out, y = router.alloc_outputs(T, send_buf=False), torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        router.mx_step(logits, x, gate_up, down, out, y)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            router.mx_step(logits, x, gate_up, down, out, y)
    torch.cuda.synchronize()
    for failed in ((), (2,), (4,), ()):
        router.set_failed_ranks(failed)
        g.replay()
        torch.cuda.synchronize()
        assert router.device_status() == 0
        ref = oracle.dispatch(oracle_cfg(wl), inp["slot_to_expert"], failed, None, inp["logits"], inp["x"])
        check_dispatch(out, ref, check_send=False)
        want, tol = _expected(wl, inp, ref, gu, dn)
        err = np.abs(y.double().cpu().numpy() - want)
        assert (err <= tol).all(), (err / tol).max()
        again = y.clone()
        assert torch.equal(router.mx_step(logits, x, gate_up, down), again)      # eager: the same bits
    router.close()


def test_two_graphs_and_two_streams():
    """Two contexts whose layers are captured separately and replayed at the same time do not disturb each other."""
    wl = W.WORKLOADS["tiny"]
    T, H, I = 128, 512, 96
    made = []
    for seed in (1, 2):
        inp = W.make_inputs(wl, T=T, H=H, seed=seed)
        router = make_router(wl, inp, max_tokens=T, hidden=H)
        (gate_up, _), (down, _) = _layer(wl, inp, T, H, I, seed)
        logits, x = to_dev(inp["logits"]), to_dev(inp["x"], torch.bfloat16)
        want = router.mx_step(logits, x, gate_up, down).clone()
        y, out = torch.zeros_like(want), router.alloc_outputs(T, send_buf=False)
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            router.mx_step(logits, x, gate_up, down, out, y)
        made.append((router, g, s, y, want, (gate_up, down, logits, x, out)))
    for _ in range(20):
        for _, g, s, *_ in made:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for router, _, _, y, want, _ in made:
        assert torch.equal(y, want) and router.device_status() == 0
        router.close()


def test_two_graphs_of_one_context():
    """Two layers' steps captured from one context, of different lengths, replayed in turn on one stream."""
    wl = W.WORKLOADS["tiny"]
    H, I = 256, 64
    inp = W.make_inputs(wl, T=128, H=H)
    router = make_router(wl, inp, max_tokens=128, hidden=H)
    (gate_up, _), (down, _) = _layer(wl, inp, 128, H, I, 5)
    made = []
    s = torch.cuda.Stream()
    for T in (128, 37):
        logits, x = to_dev(inp["logits"][:T]), to_dev(inp["x"][:T], torch.bfloat16)
        want = router.mx_step(logits, x, gate_up, down).clone()
        y, out = torch.zeros_like(want), router.alloc_outputs(T, send_buf=False)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            router.mx_step(logits, x, gate_up, down, out, y)
        made.append((g, y, want, logits, x, out))
    for _ in range(5):
        for g, *_ in made:
            g.replay()
        torch.cuda.synchronize()
        for _, y, want, *_ in made:
            assert torch.equal(y, want)
            y.zero_()
    assert router.device_status() == 0
    router.close()
