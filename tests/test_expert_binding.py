"""CPU-only: what the binding and the C entry points of the 16-bit experts, the norm and redispatch refuse.  Tensors are
stand-ins that claim to be on a device; the C calls of the binding's tests are replaced and only note that they were reached."""
import os
import subprocess

import pytest
import torch

import test_drains
from paper_2602_21140_b200 import binding as B
from paper_2602_21140_b200 import build as build_mod
from test_mx_binding import Fake as FakeTensor

T, H, E, K, R, S, I = 8, 64, 8, 2, 4, 2, 48
P, N = R * S, T * K
BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class Fake(FakeTensor):
    """Each somewhere else."""
    _next = 1 << 30

    def __init__(self, *args, **kwargs):
        super().__init__(*args, **kwargs)
        Fake._next += 1 << 30
        self._at = Fake._next

    def data_ptr(self):
        return self._at

    def element_size(self):
        return {U8: 1, BF: 2, torch.float16: 2}.get(self.dtype, 4)

    def new_empty(self, shape, dtype=None):
        return Fake(shape, dtype or self.dtype, self._device)


class Row(Fake):
    device = None

    def stride(self, d):
        return 1 if d else self.shape[-1] + 8


@pytest.fixture
def router(monkeypatch):
    monkeypatch.setattr(torch, "empty_like", lambda t, dtype=None: type(t)(t.shape, dtype or t.dtype))
    r = B.MoeRouter.__new__(B.MoeRouter)
    r.cfg = B.make_config(E, K, H, 64, R, S)
    r.device, r._ctx, r._latest = torch.device("cuda", 0), None, None
    r.reached = []
    for name in B.EXPORTED_SYMBOLS:
        if hasattr(B, name) and not name.endswith(("pitch", "string", "workspace")):
            monkeypatch.setattr(B, name, lambda *a, _n=name: r.reached.append(_n) or B.MOE_OK)
    monkeypatch.setattr(B, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(B, "_on_device", lambda index, call, *args: call(*args))
    monkeypatch.setattr(B.MoeRouter, "_stream", lambda self: 0)
    return r


def rows8(*shape):
    return B.Mx8Rows(Fake(shape, U8), Fake((*shape[:-1], B._mx_pitch(shape[-1])), U8))


def good():
    return dict(rows=Fake((N, H), BF), slot_counts=Fake((P,), I32), slot_offsets=Fake((P + 1,), I32), gate_up=Fake((P, 2 * I, H), BF),
                down=Fake((P, H, I), BF))


def variants(t):
    s = tuple(t.shape)
    yield "type", Fake(s, F32 if t.dtype is not F32 else BF)
    yield "device", Fake(s, t.dtype, device=1)
    yield "CPU", Fake(s, t.dtype, device=-1)
    yield "strides", Fake(s, t.dtype, contiguous=False)
    for d in range(len(s)):
        yield f"dimension {d}", Fake(s[:d] + (s[d] - 1,) + s[d + 1:], t.dtype)
    yield "rank", Fake((1, *s), t.dtype)


FORWARD = [("expert_gated", ("rows", "slot_counts", "slot_offsets", "gate_up"), {"h": (N, I), "z": (N, 2 * I)}),
           ("expert_product", ("rows", "slot_counts", "slot_offsets", "gate_up"), {"y": (N, 2 * I)}),
           ("expert_rows_backward", ("rows", "slot_counts", "slot_offsets", "down"), {"d_rows": (N, I)}),
           ("expert_gated_backward", ("rows", "slot_counts", "slot_offsets", "down", "z"), {"dz": (N, 2 * I), "h": (N, I)})]


@pytest.mark.parametrize("name,inputs,outputs", FORWARD, ids=[f[0] for f in FORWARD])
def test_every_argument_of_a_product_is_looked_at(router, name, inputs, outputs):
    have = {**good(), "z": Fake((N, 2 * I), BF)}
    call, args = getattr(router, name), [have[i] for i in inputs]
    outs = {k: Fake(s, BF) for k, s in outputs.items()}
    call(*args)
    call(*args, **outs)
    assert len(router.reached) == 2
    for i, key in enumerate(inputs):
        for what, bad in variants(args[i]):
            # fewer rows are fewer rows everywhere, longer offsets are fine, and the features of a result that is not given are
            # whatever the matrix has (multiples of 8 are the C call's to check)
            free = {"expert_product": ("gate_up", "dimension 1"), "expert_rows_backward": ("down", "dimension 2")}.get(name)
            if (key, what) in (("slot_offsets", "dimension 0"), free) or (key == "rows" and what == "dimension 0" and "z" not in inputs):
                continue
            with pytest.raises((B.MoeError, ValueError)):
                call(*args[:i], bad, *args[i + 1:])
    for key, t in outs.items():
        for what, bad in variants(t):
            with pytest.raises((B.MoeError, ValueError)):
                call(*args, **{**outs, key: bad})
    assert len(router.reached) == 2


def test_what_is_kept_is_of_the_right_form(router):
    g = good()
    args = (g["rows"], g["slot_counts"], g["slot_offsets"])
    router.expert_gated(*args, g["gate_up"], z=rows8(N, 2 * I))
    router.expert_gated_backward(*args, g["down"], rows8(N, 2 * I))
    for bad in (rows8(N, 2 * I + 32), rows8(N - 1, 2 * I), B.Mx8Rows(Fake((N, 2 * I), U8), Fake((N, 32), U8)), Fake((N, 2 * I), U8)):
        with pytest.raises(B.MoeError):
            router.expert_gated(*args, g["gate_up"], z=bad)
        with pytest.raises(B.MoeError):
            router.expert_gated_backward(*args, g["down"], bad)
    for hidden in (8, 24, 0):                                   # not a multiple of 16
        with pytest.raises(B.MoeError):
            router.expert_gated(*args, Fake((P, 2 * hidden, H), BF))
    assert len(router.reached) == 2


def test_weight_gradients(router):
    g = good()
    dy, args = Fake((N, I), BF), (g["slot_counts"], g["slot_offsets"])
    router.expert_weight_backward(dy, g["rows"], *args)
    router.expert_weight_backward(dy, g["rows"], *args, Fake((P, I, H), F32), add=True)
    for bad in (dict(add=True), dict(dtype=torch.float16), dict(d_weight=Fake((P, I, H), torch.float16)), dict(d_weight=Fake((P, H, I), BF)),
                dict(d_weight=Fake((P - 1, I, H), F32)), dict(d_weight=Fake((P, I, H), F32, contiguous=False))):
        with pytest.raises(B.MoeError):
            router.expert_weight_backward(dy, g["rows"], *args, **bad)
    for what, bad in variants(dy):
        if what != "dimension 1":
            with pytest.raises(B.MoeError):
                router.expert_weight_backward(bad, g["rows"], *args)
    assert router.reached == ["moe_expert_weight_backward"] * 2


def test_a_network_is_refused_before_its_first_launch(router):
    g = good()
    dy = Fake((N, H), BF)
    args = dict(rows=g["rows"], slot_counts=g["slot_counts"], slot_offsets=g["slot_offsets"], gate_up=g["gate_up"], down=g["down"])
    outs = dict(y=Fake((N, H), BF), h=Fake((N, I), BF), z=rows8(N, 2 * I))
    router.expert_ffn(**args)
    router.expert_ffn(**args, **outs)
    assert router.reached == ["moe_expert_gated", "moe_expert_product"] * 2
    router.reached.clear()
    for name, t in [*args.items(), *outs.items()]:
        for what, bad in variants(t) if name != "z" else [("rows", rows8(N - 1, 2 * I)), ("columns", rows8(N, 4 * I)), ("a tensor", Fake((N, I), BF))]:
            if (name, what) in (("slot_offsets", "dimension 0"), ("down", "dimension 1")):
                continue
            with pytest.raises((B.MoeError, ValueError, AttributeError)):
                router.expert_ffn(**{**args, **outs, name: bad})
    whole = Fake((2 * N, 2 * I), BF)
    y = Fake((N, H), BF)
    y._at = whole._at + 64
    with pytest.raises(B.MoeError):                             # y over what is kept
        router.expert_ffn(**args, y=y, z=_at((N, 2 * I), whole._at))
    assert router.reached == []
    args = dict(dy=dy, **args, z=rows8(N, 2 * I))
    outs = dict(d_rows=Fake((N, H), BF), d_gate_up=Fake((P, 2 * I, H), F32), d_down=Fake((P, H, I), F32))
    router.expert_ffn_backward(**args)
    router.expert_ffn_backward(**args, **outs, add=True)
    router.expert_ffn_backward(**args, grad_dtype=F32)
    steps = ["moe_expert_gated_backward", "moe_expert_weight_backward", "moe_expert_weight_backward", "moe_expert_rows_backward"]
    assert router.reached == steps * 3
    router.reached.clear()
    for name, t in [*args.items(), *outs.items()]:
        for what, bad in variants(t) if name != "z" else [("rows", rows8(N - 1, 2 * I)), ("columns", rows8(N, 4 * I)), ("none", None)]:
            if (name, what) in (("slot_offsets", "dimension 0"), ("d_gate_up", "type"), ("d_down", "type")):
                continue
            with pytest.raises((B.MoeError, ValueError, AttributeError)):
                router.expert_ffn_backward(**{**args, **outs, name: bad})
    for bad in (dict(add=True), dict(add=True, grad_dtype=F32), dict(add=True, d_down=outs["d_down"]), dict(grad_dtype=torch.float16),
                dict(add=True, d_gate_up=Fake((P, 2 * I, H), BF), d_down=outs["d_down"])):
        with pytest.raises(B.MoeError):
            router.expert_ffn_backward(**args, **bad)
    for name, t in outs.items():                                # over any input or another output
        for other in [*args.values(), *[o for o in outs.values() if o is not t]]:
            place = _at(t.shape, (other.codes if isinstance(other, B.Mx8Rows) else other)._at, t.dtype)
            with pytest.raises(B.MoeError):
                router.expert_ffn_backward(**{**args, **outs, name: place})
    assert router.reached == []


def _at(shape, address, dtype=BF):
    t = Fake(shape, dtype)
    t._at = address
    return t


def _out(tokens=T):
    n = tokens * K
    return B.DispatchBuffers(Fake((tokens, K), I32), Fake((tokens, K), F32), Fake((tokens, K), I32), Fake((P,), I32), Fake((P + 1,), I32),
                             Fake((R,), I32), Fake((R + 1,), I32), Fake((n,), I32), Fake((n,), I32), Fake((n, H), BF))


def test_a_step_is_refused_before_its_first_launch(router):
    g, logits, x = good(), Fake((T, E), F32), Fake((T, H), BF)
    fine = dict(out=_out(), y=Fake((T, H), BF), buf=Fake((N, H), BF), z=rows8(N, 2 * I))
    router.expert_step(logits, x, g["gate_up"], g["down"], **fine)
    assert router.reached == ["moe_dispatch", "moe_expert_gated", "moe_expert_product", "moe_combine"]
    router.reached.clear()
    short = _out()
    short.send_buf = Fake((N - 1, H), BF)
    none = _out()
    none.send_buf = None
    for bad in (dict(out=_out(T - 1)), dict(out=short), dict(out=none), dict(y=Fake((T - 1, H), BF)), dict(y=Fake((T, H), F32)),
                dict(buf=Fake((N, H - 8), BF)), dict(z=rows8(N, I * 2 + 32)), dict(z=Fake((N, I), BF))):
        with pytest.raises(B.MoeError):
            router.expert_step(logits, x, g["gate_up"], g["down"], **{**fine, **bad})
    for gate_up, down in ((Fake((P, 2 * I, H + 8), BF), g["down"]), (g["gate_up"], Fake((P, H, I + 16), BF)), (Fake((P, 16, H), BF), Fake((P, H, 8), BF)),
                          (Fake((P - 1, 2 * I, H), BF), g["down"])):
        with pytest.raises(B.MoeError):
            router.expert_step(logits, x, gate_up, down, **fine)
        with pytest.raises(B.MoeError):
            router.expert_step_backward(logits, x, fine["buf"], fine["out"], fine["buf"], fine["z"], gate_up, down)
    for bad_logits, bad_x in ((Fake((T, E - 1), F32), x), (logits, Fake((T, H - 8), BF)), (logits, Fake((T - 1, H), BF)), (Fake((T, E), BF), x)):
        with pytest.raises(B.MoeError):
            router.expert_step(bad_logits, bad_x, g["gate_up"], g["down"], **fine)
    with pytest.raises(B.MoeError):
        router.redispatch(rows8(T, H + 32))
    with pytest.raises(B.MoeError):
        router.redispatch(rows8(T, H), Fake((N - 1, H), BF))
    assert router.reached == []


def test_norm_arguments(router, monkeypatch):
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: Row((shape,) if isinstance(shape, int) else shape, dtype))
    x, w = Row((T, H), BF), Row((H,), BF)
    router_reached = router.reached
    B.rms_norm(x, w, keep=True)
    B.rms_norm(Row((T, H), BF, contiguous=False), Row((H,), F32), x)
    for bad in ((Row((T, H), torch.int32), w, None), (x, Row((H - 1,), BF), None), (x, Row((H,), torch.float64), None), (x, w, Row((T, H), F32)),
                (x, w, Row((T - 1, H), BF)), (x, w, Row((T, H), BF, device=1)), (Row((T, H), BF, device=-1), w, None),
                (Row((2, T, H), BF, contiguous=False), w, None)):
        with pytest.raises(B.MoeError):
            B.rms_norm(bad[0], bad[1], bad[2])
    out = B.RmsNormOut(Row((T, H), BF), Row((T, H), BF), Row((T,), F32), None)
    with pytest.raises(B.MoeError):
        B.rms_norm(x, w, out=out, keep=True)
    for field, bad in (("y", Row((T, H), F32)), ("h", Row((T - 1, H), BF)), ("rstd", Row((T,), BF))):
        with pytest.raises(B.MoeError):
            B.rms_norm(x, w, x, out=B.RmsNormOut(**{**vars(out), field: bad}))
    args = (x, Row((T, H), BF), Row((T,), F32), Row((H,), F32))
    B.rms_norm_backward(*args, dh=x)
    for i, t in enumerate(args):
        for what, bad in variants(t):
            if (i, what) != (3, "type"):
                with pytest.raises((B.MoeError, ValueError)):
                    B.rms_norm_backward(*args[:i], Row(bad.shape, bad.dtype, bad._device, bad._contiguous), *args[i + 1:])
    for more in (dict(dh=Row((T, H), F32)), dict(dx=Row((T - 1, H), BF)), dict(d_weight=Row((H,), BF)), dict(d_weight=Row((H + 8,), F32))):
        with pytest.raises(B.MoeError):
            B.rms_norm_backward(*args, **more)
    assert router_reached == ["moe_rms_norm"] * 2 + ["moe_rms_norm_backward"]


def test_values_of_8_bit_rows(router):
    m = rows8(T, H)
    B.mx8_dequantize(m, out=Row((T, H), BF, contiguous=False))
    for bad, out in ((rows8(T, H), Row((T, H), F32)), (rows8(T, H), Row((T, H + 32), BF)), (rows8(T, H), Row((T, H), BF, device=-1)),
                     (B.Mx8Rows(Fake((T, H), U8), Fake((T, H // 32), U8)), None), (B.mx_empty(T, H, device="cpu"), None), (B.mx8_empty(T, H, device="cpu"), None),
                     (B.mx8_empty(T, H, device="cpu"), torch.empty(T, H, dtype=BF))):
        with pytest.raises(B.MoeError):
            B.mx8_dequantize(bad, out=out)
    assert router.reached == ["moe_kept_dequantize"]


A = 1 << 30                  # 16-byte aligned; refused calls never look at it
BAD, OK, CAP, CUDA = B.MOE_ERR_INVALID_ARG, B.MOE_OK, B.MOE_ERR_CAPACITY, B.MOE_ERR_CUDA


@pytest.fixture(scope="module")
def built():
    build_mod.build_library()


def _norm(x=A, xs=64, res=0, rs=64, dt=0, rows=4, cols=64, w=A + (1 << 20), wdt=0, eps=1e-6, h=0, y=A + (2 << 20), rstd=A + (3 << 20), c=0, s=0):
    return B.moe_rms_norm(x, xs, res, rs, dt, rows, cols, w, wdt, eps, h, y, rstd, c, s)


def _back(dy=A, dh=0, h=A + (1 << 20), rstd=A + (2 << 20), dt=0, rows=4, cols=64, w=A + (3 << 20), wdt=0, dx=A + (4 << 20), dw=A + (5 << 20),
          ws=A + (6 << 20), n=None):
    return B.moe_rms_norm_backward(dy, dh, h, rstd, dt, rows, cols, w, wdt, dx, dw, ws, B.moe_rms_norm_backward_workspace(rows, cols) if n is None else n)


@pytest.mark.parametrize("args", [dict(dt=3), dict(dt=-1), dict(rows=-1), dict(cols=0), dict(cols=12), dict(cols=16392, xs=16392), dict(xs=63), dict(xs=68),
                                  dict(wdt=3), dict(wdt=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(x=0), dict(w=0), dict(y=0), dict(x=A + 8),
                                  dict(y=A + (2 << 20) + 2), dict(c=A + 8192), dict(s=A + 8192), dict(c=A + 8192, s=A + 16384, cols=40, xs=40),
                                  dict(res=A + 4096), dict(res=A + 4096, h=A + 8192, rs=60), dict(y=A + 496), dict(y=A), dict(rstd=A + 16), dict(h=A + 16),
                                  dict(h=A, xs=128), dict(c=A + 8192, s=A + 8192 + 240), dict(y=A + (1 << 20) - 400), dict(res=A + 4096, h=A + 4096 + 16)])
def test_norm_is_refused(built, args):
    assert _norm(**args) == BAD


@pytest.mark.parametrize("args", [dict(dt=3), dict(cols=12), dict(cols=16392), dict(wdt=3), dict(dy=0), dict(h=0), dict(rstd=0), dict(w=0), dict(dx=0),
                                  dict(dw=0), dict(ws=0), dict(ws=A + (6 << 20) + 8), dict(dx=A + 16), dict(dx=A + (1 << 20) - 16), dict(dw=A + 64),
                                  dict(dw=A + (4 << 20) + 64), dict(ws=A + (5 << 20)), dict(dx=A + (3 << 20)), dict(rows=0, dw=0)])
def test_norm_backward_is_refused(built, args):
    assert _back(**args) == BAD


def test_norm_sizes(built):
    assert _norm(rows=0, x=0, w=0, y=0) == OK
    assert _norm(rows=1 << 31) == CAP and _back(n=4) == CAP
    need = B.moe_rms_norm_backward_workspace
    assert need(0, 64) == 0 and need(1, 64) == 256 and need(4, 12) == 0 and need(4, 16392) == 0
    assert need(1 << 30, 7168) <= 8 * 148 * 7168 * 4
    if torch.cuda.is_available():
        return
    # these pass the checks: without a GPU they end at the launch
    assert _norm() == _norm(res=A + 4096, h=A + 4096) == _norm(res=A + 4096, h=A) == _norm(xs=128, c=A + (7 << 20), s=A + (8 << 20)) == CUDA
    assert _back() == _back(dx=A) == _back(dx=A + (1 << 20)) == _back(dh=A + (7 << 20), dx=A + (7 << 20)) == CUDA


def test_context_calls_without_a_context(built):
    assert B.moe_expert_product(None, A, 1, A, A, A, 8, 8, A) == BAD
    assert B.moe_expert_gated(None, A, 1, A, A, A, 16, 8, A) == BAD
    assert B.moe_expert_rows_backward(None, A, 1, A, A, A, 8, 8, A) == BAD
    assert B.moe_expert_gated_backward(None, A, 1, A, A, A, 8, 16, A, 0, A, A) == BAD
    assert B.moe_expert_weight_backward(None, A, A, 1, A, A, 8, 8, A, 0, 0) == BAD
    assert B.moe_redispatch(None, A, A, 1, A) == BAD
    for args, status in (((A, A, 1, 40, A, 0, 40), BAD), ((A, A, 1, 32, A + 2, 0, 32), BAD), ((A, A, 1, 32, A + 16, 0, 32), BAD), ((A, A, 0, 32, 0, 0, 32), OK),
                         ((A, A + 4096, 1 << 40, 32, A, 0, 32), CAP)):
        assert B.moe_kept_dequantize(*args) == status


def test_every_other_wait_gives_up():
    test_drains.test_every_other_wait_gives_up("expert_product.cu")


def test_sizes_that_the_kernels_numbers_cannot_hold_are_refused(tmp_path):
    src, exe = tmp_path / "limits.cu", tmp_path / "limits"
    products = [(1, 8, 8, 1, 1), (1, 1 << 30, 8, 1, 1), (1, 8, 1 << 30, 1, 1), (1, (1 << 30) + 8, 8, 1, 0), ((1 << 30) + 1, 8, 8, 1, 0), (1 << 30, 1 << 30, 8, 1, 0),
                (1, 1 << 25, 32, 4096, 0), (1, 1 << 20, 1 << 20, 1, 0)]
    grads = [(1, 8, 8, 1, 1), (1 << 30, 8192, 8192, 4096, 1), (1, 1 << 22, 1 << 14, 1, 1), (1, 1 << 22, 1 << 15, 512, 0), (1, (1 << 30) + 8, 8, 1, 0),
             (1, 1 << 20, 1 << 20, 1, 0), ((1 << 30) + 1, 8, 8, 1, 0)]
    body = "".join(f'printf("%d ", (int)expert_product_fits({r}ll, {n}ll, {k}ll, {p}));' for r, n, k, p, _ in products)
    body += "".join(f'printf("%d ", (int)weight_grad_fits({r}ll, {m}ll, {n}ll, {p}));' for r, m, n, p, _ in grads)
    # a tile's number, its rows and features rounded up to a tile, and the tiles that a CTA looks ahead stay ints
    body += 'printf("%d", (int)((long long)kMaxFeatures + 4 * 256 < (1ll << 31) && (long long)kMaxRows + 2 * 256 < (1ll << 31) && kTooManyTiles + 64 * 148 > 0));'
    src.write_text('#include <stdio.h>\n#include "expert_product.h"\nusing namespace moe;\nint main()\n{\n' + body + "\nreturn 0;\n}\n")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_21140_b200", "csrc")
    subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", csrc, "-o", str(exe), str(src)])
    got = subprocess.check_output([str(exe)], text=True).split()
    assert [int(v) for v in got] == [c[4] for c in products] + [c[4] for c in grads] + [1]
