"""CPU-only: calls that launch several operators are refused before the first launch where any of them would be, or where one of
them would write what another reads.  Tensors are stand-ins, and so are the C calls, which refuse as the C code does."""
import itertools
import os
import subprocess

import pytest
import torch

from paper_2602_21140_b200 import binding as B
from test_expert_binding import BF, E, F32, H, I, I32, K, N, P, T, U8, Fake, _at, _out, good, router, rows8  # noqa: F401

OK, BAD, CAP = B.MOE_OK, B.MOE_ERR_INVALID_ARG, B.MOE_ERR_CAPACITY


def _meet(outputs, inputs):
    spans = [(a, a + n) for a, n in inputs if a]
    for a, n in outputs:
        if a and n:
            if any(a < e and s < a + n for s, e in spans if s < e):
                return True
            spans.append((a, a + n))
    return False


def _askew(*pointers):
    return any(p and p % 16 for p in pointers)


def _sizes(rows, n_out, n_in):
    if n_out < 8 or n_out % 8 or n_in < 8 or n_in % 8:
        return BAD
    for n, k in ((n_out, n_in), (n_in, n_out)):
        if max(rows, n, k) > 1 << 30 or (n + 127) // 128 * (P + rows // 32) >= 1 << 29 or n * k * 2 >= 1 << 39:
            return CAP
    return OK


def _kept(rows, cols, z, s):
    return [(z or 0, rows * cols * (1 if s else 2)), (s or 0, rows * B._mx_pitch(cols) if s else 0)]


class C:
    """The C entry points of a network, as far as they refuse."""

    def __init__(self):
        self.launched, self.score = [], B.MOE_SCORE_SOFTMAX

    def _done(self, name, st):
        if st == OK:
            self.launched.append(name)
        return st

    def gated(self, ctx, a, rows, counts, offsets, w, hidden, n_in, h, z=0, s=0, stream=0):
        st = _sizes(rows, 2 * hidden, n_in) if hidden >= 16 and hidden % 16 == 0 else BAD
        if st == OK and rows:
            bad = not h or _askew(a, w, h, z, s) or _meet([(h, rows * hidden * 2), *_kept(rows, 2 * hidden, z, s)],
                                                          [(a, rows * n_in * 2), (w, P * hidden * n_in * 4), (counts, P * 4), (offsets, P * 4)])
            st = BAD if bad else OK
        return self._done("gated", st)

    def product(self, ctx, a, rows, counts, offsets, w, n_out, n_in, y, stream=0):
        st = _sizes(rows, n_out, n_in)
        if st == OK and rows:
            bad = not y or _askew(a, w, y) or _meet([(y, rows * n_out * 2)], [(a, rows * n_in * 2), (w, P * n_out * n_in * 2), (counts, P * 4), (offsets, P * 4)])
            st = BAD if bad else OK
        return self._done("product", st)

    def gated_backward(self, ctx, dy, rows, counts, offsets, w, n_out, hidden, z, s, dz, h, stream=0):
        st = _sizes(rows, n_out, hidden) if hidden >= 16 and hidden % 16 == 0 else BAD
        if st == OK and rows:
            bad = not z or not dz or not h or _askew(dy, w, z, s, dz, h) or _meet(
                [(dz, rows * hidden * 4), (h, rows * hidden * 2)],
                [(dy, rows * n_out * 2), (w, P * n_out * hidden * 2), *_kept(rows, 2 * hidden, z, s), (counts, P * 4), (offsets, P * 4)])
            st = BAD if bad else OK
        return self._done("gated_backward", st)

    def weight_backward(self, ctx, dy, a, rows, counts, offsets, n_out, n_in, dw, dtype, add, stream=0):
        if n_out < 8 or n_out % 8 or n_in < 8 or n_in % 8 or (add and dtype != B.MOE_DTYPE_F32):
            return BAD
        if max(rows, n_out, n_in) > 1 << 30 or (n_out + 255) // 256 * ((n_in + 255) // 256) >= (1 << 29) // P or n_out * n_in * 4 >= 1 << 39:
            return CAP
        size = P * n_out * n_in * (4 if dtype == B.MOE_DTYPE_F32 else 2)
        bad = not dw or _askew(dw)
        if rows:
            bad = bad or _askew(dy, a) or _meet([(dw, size)], [(dy, rows * n_out * 2), (a, rows * n_in * 2), (counts, P * 4), (offsets, P * 4)])
        return self._done("weight_backward", BAD if bad else OK)

    def rows_backward(self, ctx, dy, rows, counts, offsets, w, n_out, n_in, da, stream=0):
        st = _sizes(rows, n_out, n_in)
        if st == OK and rows:
            bad = not da or _askew(dy, w, da) or _meet([(da, rows * n_in * 2)],
                                                       [(dy, rows * n_out * 2), (w, P * n_out * n_in * 2), (counts, P * 4), (offsets, P * 4)])
            st = BAD if bad else OK
        return self._done("rows_backward", st)

    def dispatch(self, ctx, logits, x, tokens, out, stream=0):
        return self._done("dispatch", BAD if tokens and _askew(logits, x, out.send_buf) else OK)

    def combine_backward(self, ctx, buf, dy, tokens, d_buf, d_weights, stream=0):
        return self._done("combine_backward", BAD if tokens and _askew(buf, dy, d_buf) else OK)

    def redispatch(self, ctx, codes, scales, tokens, send, stream=0):
        return self._done("redispatch", BAD if tokens and _askew(codes, scales, send) else OK)

    def dispatch_backward(self, ctx, logits, d_send, d_weights, tokens, dx, d_logits, stream=0):
        bad = bool(d_weights) != bool(d_logits) or (d_logits and self.score == B.MOE_ROUTE_DENSE_TP)
        bad = bad or (tokens and (_askew(d_send, dx, d_logits) or (d_logits and self.score == B.MOE_SCORE_SIGMOID and not logits)))
        return self._done("dispatch_backward", BAD if bad else OK)

    def combine(self, ctx, buf, tokens, y, stream=0):
        return self._done("combine", BAD if tokens and _askew(buf, y) else OK)


@pytest.fixture
def c(router, monkeypatch):  # noqa: F811
    c = C()
    monkeypatch.setattr(B, "moe_expert_gated", c.gated)
    monkeypatch.setattr(B, "moe_expert_product", c.product)
    for name in ("dispatch", "combine", "combine_backward", "redispatch", "dispatch_backward"):
        monkeypatch.setattr(B, "moe_" + name, getattr(c, name))
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: Fake((shape,) if isinstance(shape, int) else shape, dtype))
    for name in ("gated_backward", "weight_backward", "rows_backward"):
        monkeypatch.setattr(B, "moe_expert_" + name, getattr(c, name))
    return c


def _forward():
    g = good()
    return {**g, "y": Fake((N, H), BF), "h": Fake((N, I), BF), "z": rows8(N, 2 * I)}


def _moved(args, name, address):
    """The same arguments, with `name` (of 8-bit rows "z.codes", "z.scales") at another address."""
    key, _, part = name.partition(".")
    t = getattr(args[key], part) if part else args[key]
    moved = _at(t.shape, address, t.dtype)
    if part:
        z = args[key]
        moved = B.Mx8Rows(moved, z.scales) if part == "codes" else B.Mx8Rows(z.codes, moved)
    return {**args, key: moved}


def _tensor(args, name):
    key, _, part = name.partition(".")
    return getattr(args[key], part) if part else args[key]


def test_a_network_runs_with_its_buffers_apart(router, c):  # noqa: F811
    for more in itertools.product((False, True), (False, True), (None, "8", "16")):
        args = _forward()
        y, h, kept = more
        args["y"], args["h"] = args["y"] if y else None, args["h"] if h else None
        args["z"] = {None: None, "8": args["z"], "16": Fake((N, 2 * I), BF)}[kept]
        router.expert_ffn(**args)
    assert c.launched == ["gated", "product"] * 12
    args = _forward()
    router.expert_ffn(**{**args, "y": args["rows"]})           # y in the place of the rows, which are read no more
    empty = dict(rows=Fake((0, H), BF), y=_at((0, H), args["down"]._at), z=None, h=None)
    router.expert_ffn(**{**args, **empty})                      # a buffer without rows shares no byte
    assert c.launched == ["gated", "product"] * 14


@pytest.mark.parametrize("kept", ["8", "16"])
def test_a_networks_outputs_lie_nowhere_else(router, c, kept):  # noqa: F811
    args = _forward()
    outputs = ["y", "h"] + (["z.codes", "z.scales"] if kept == "8" else ["z"])
    if kept == "16":
        args["z"] = Fake((N, 2 * I), BF)
    for out in outputs:
        for other in ["rows", "gate_up", "down", "slot_counts", "slot_offsets"] + [o for o in outputs if o != out]:
            t = _tensor(args, other)
            for address in (t._at, t._at + t.numel() * t.element_size() - 16, t._at - 16):
                if (out, other) == ("y", "rows") or address % 16:
                    continue
                with pytest.raises(B.MoeError):
                    router.expert_ffn(**_moved(args, out, address))
    assert c.launched == []


def test_a_networks_alignment_and_sizes(router, c):  # noqa: F811
    args = _forward()
    for name in ("rows", "gate_up", "down", "y", "h", "z.codes", "z.scales"):
        for off in (2, 8):
            with pytest.raises(B.MoeError):
                router.expert_ffn(**_moved(args, name, _tensor(args, name)._at + off))
    router.expert_ffn(**_moved(args, "slot_counts", args["slot_counts"]._at + 4))
    assert c.launched == ["gated", "product"]
    c.launched.clear()
    plain = {k: args[k] for k in ("rows", "slot_counts", "slot_offsets", "gate_up", "down")}
    for n_out in (12, 4, 0, 7):
        with pytest.raises(B.MoeError):
            router.expert_ffn(**{**plain, "down": Fake((P, n_out, I), BF)})
    for n_in in (12, 4, 0):
        with pytest.raises(B.MoeError):
            router.expert_ffn(**{**plain, "rows": Fake((N, n_in), BF), "gate_up": Fake((P, 2 * I, n_in), BF)})
    for n, n_out in ((N, (1 << 30) + 8), ((1 << 30) + 1, H), (1 << 30, 1 << 22)):
        with pytest.raises(B.MoeError) as e:
            router.expert_ffn(**{**plain, "rows": Fake((n, H), BF), "down": Fake((P, n_out, I), BF)})
        assert e.value.status == CAP
    assert c.launched == []


STEP = ["dispatch", "gated", "product", "combine"]
BACKWARD = ["gated_backward", "weight_backward", "weight_backward", "rows_backward"]


def _step(kept="8"):
    g = good()
    return dict(logits=Fake((T, E), F32), x=Fake((T, H), BF), gate_up=g["gate_up"], down=g["down"], out=_out(), y=Fake((T, H), BF), buf=Fake((N, H), BF),
                z=rows8(N, 2 * I) if kept == "8" else Fake((N, 2 * I), BF))


INDEX = ["topk_ids", "topk_weights", "topk_slot", "slot_counts", "slot_offsets", "rank_counts", "rank_offsets", "dst_row", "src_index"]


def test_a_step_runs_with_its_buffers_apart(router, c):  # noqa: F811
    args = _step()
    router.expert_step(**args)
    router.expert_step(**{**args, "out": None, "y": None, "buf": None, "z": None})
    router.expert_step(**{**args, "y": args["x"]})
    router.expert_step(**{**args, "buf": args["out"].send_buf})
    router.expert_step(**{**args, "y": _at((T, H), args["out"].send_buf._at)})
    assert c.launched == STEP * 5


@pytest.mark.parametrize("kept", ["8", "16"])
def test_a_steps_outputs_lie_nowhere_else(router, c, kept):  # noqa: F811
    """Seen before the dispatch, which would become the latest one."""
    args = _step(kept)
    outputs = ["y", "buf"] + (["z.codes", "z.scales"] if kept == "8" else ["z"])
    fine = {("y", "x"), ("y", "out.send_buf"), ("buf", "out.send_buf")}
    for o in outputs:
        for other in ["logits", "x", "gate_up", "down", "out.send_buf"] + ["out." + i for i in INDEX] + [q for q in outputs if q != o]:
            if (o, other) not in fine:
                with pytest.raises(B.MoeError):
                    router.expert_step(**_moved(args, o, _tensor(args, other)._at))
    for name in outputs + ["gate_up", "down"]:
        with pytest.raises(B.MoeError):
            router.expert_step(**_moved(args, name, _tensor(args, name)._at + 8))
    askew = _out()
    askew.send_buf = _at((N, H), askew.send_buf._at + 8)
    with pytest.raises(B.MoeError):
        router.expert_step(**{**args, "out": askew})
    assert c.launched == [] and router._latest is None


def _step_backward(args, rows):
    return dict(logits=args["logits"], dy=Fake((T, H), BF), rows=rows, out=args["out"], buf=args["buf"], z=args["z"], gate_up=args["gate_up"],
                down=args["down"], d_gate_up=Fake((P, 2 * I, H), F32), d_down=Fake((P, H, I), F32))


ALL_BACK = ["combine_backward", "redispatch", *BACKWARD, "dispatch_backward"]


def test_a_steps_gradients_are_refused_before_one_is_written(router, c):  # noqa: F811
    """With add=True a caller that tries again must not have added anything."""
    args = _step()
    router.expert_step(**args)
    c.launched.clear()
    from8, from16 = _step_backward(args, rows8(T, H)), _step_backward(args, args["out"].send_buf)
    router.expert_step_backward(**from8, add=True)
    router.expert_step_backward(**from16, add=True)
    router.expert_step_backward(**{**from8, "logits": None}, add=True)   # softmax: logits are for masked ones only
    without = [s for s in ALL_BACK if s != "redispatch"]
    assert c.launched == ALL_BACK + without + ALL_BACK
    c.launched.clear()
    for back in (from8, from16):
        for bad in (Fake((T, E - 1), F32), Fake((T, E), BF), Fake((T - 1, E), F32), Fake((T, E), F32, device=1), Fake((T, E), F32, contiguous=False)):
            with pytest.raises(B.MoeError):
                router.expert_step_backward(**{**back, "logits": bad}, add=True)
        for grad in ("d_gate_up", "d_down"):
            others = ["logits", "dy", "buf", "gate_up", "down", "z.codes", "z.scales"] + ["out." + i for i in INDEX]
            for other in others + (["rows.codes", "rows.scales"] if back is from8 else ["rows"]):
                with pytest.raises(B.MoeError):
                    router.expert_step_backward(**_moved(back, grad, _tensor(back, other)._at), add=True)
            with pytest.raises(B.MoeError):
                router.expert_step_backward(**_moved(back, grad, back[grad]._at + 4), add=True)
    router.cfg.score_func = c.score = B.MOE_SCORE_SIGMOID
    with pytest.raises(B.MoeError):
        router.expert_step_backward(**{**from8, "logits": None}, add=True)
    assert not set(c.launched) & {*BACKWARD, "dispatch_backward"}


def test_outputs_in_the_place_of_the_rows_that_a_backward_pass_asks_for(router, c):  # noqa: F811
    """buf over the send buffer leaves no rows but those in 8 bits."""
    args = _step()
    args["buf"] = args["out"].send_buf
    router.expert_step(**args)
    c.launched.clear()
    for rows in (args["out"].send_buf, _at((N, H), args["buf"]._at), _at((N, H), args["buf"]._at + 2 * H)):
        with pytest.raises(B.MoeError):
            router.expert_step_backward(**_step_backward(args, rows))
    assert c.launched == []
    router.expert_step_backward(**_step_backward(args, rows8(T, H)))
    assert c.launched == ALL_BACK


def _printed(tmp_path, header, expressions):
    """The values of C++ expressions of ints."""
    src, exe = tmp_path / "values.cu", tmp_path / "values"
    body = "".join(f'printf("%d ", (int)({e}));' for e in expressions)
    src.write_text(f'#include <stdio.h>\n#include "{header}"\nusing namespace moe;\nint main()\n{{\n{body}\nreturn 0;\n}}\n')
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_21140_b200", "csrc")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", csrc,
                           "-o", str(exe), str(src)])
    return [int(v) for v in subprocess.check_output([str(exe)], text=True).split()]


SPREAD = [(n, n_in, cols, n_out, P_) for n in (1, 4096, 1 << 30, (1 << 30) + 1) for n_in in (8, 1 << 15, 1 << 19, 1 << 24) for cols in (32, 1 << 20, 1 << 25)
          for n_out in (8, 1 << 15, 1 << 23, 1 << 30, (1 << 30) + 8) for P_ in (1, 36, 4096)]


def _backward():
    g = good()
    return {"dy": Fake((N, H), BF), **g, "z": rows8(N, 2 * I), "d_rows": Fake((N, H), BF), "d_gate_up": Fake((P, 2 * I, H), F32),
            "d_down": Fake((P, H, I), F32)}


def test_buffers_without_rows_lie_anywhere(router, c):  # noqa: F811
    """Slices of no rows of buffers that are in use."""
    args = _backward()
    for name in ("gate_up", "down", "d_gate_up", "d_down"):
        inside = args[name]._at + 64
        none = dict(dy=_at((0, H), inside), rows=_at((0, H), inside), d_rows=_at((0, H), inside), z=_at((0, 2 * I), inside))
        router.expert_ffn_backward(**{**args, **none}, add=True)
    assert c.launched == BACKWARD * 4


def test_a_networks_gradients_alignment_and_sizes(router, c):  # noqa: F811
    """Nothing is added to one matrix's gradient in a call that another operator refuses."""
    args = _backward()
    router.expert_ffn_backward(**args, add=True)
    assert c.launched == BACKWARD
    c.launched.clear()
    for name in ("dy", "rows", "gate_up", "down", "z.codes", "z.scales", "d_rows", "d_gate_up", "d_down"):
        for off in (4, 8):
            with pytest.raises(B.MoeError):
                router.expert_ffn_backward(**_moved(args, name, _tensor(args, name)._at + off), add=True)
    plain = {k: args[k] for k in ("dy", "rows", "slot_counts", "slot_offsets", "gate_up", "down", "z")}
    for n_out in (12, 4, 0):
        with pytest.raises(B.MoeError):
            router.expert_ffn_backward(**{**plain, "dy": Fake((N, n_out), BF), "down": Fake((P, n_out, I), BF)})
    for n_in in (12, 4, 0):
        with pytest.raises(B.MoeError):
            router.expert_ffn_backward(**{**plain, "rows": Fake((N, n_in), BF), "gate_up": Fake((P, 2 * I, n_in), BF)})
    wide = 1 << 23                                             # its gradient's tiles are more than eight slots may have
    for more in (dict(dy=Fake((N, (1 << 30) + 8), BF), down=Fake((P, (1 << 30) + 8, I), BF)),
                 dict(rows=Fake((N, 1 << 20), BF), gate_up=Fake((P, wide, 1 << 20), BF), down=Fake((P, H, wide // 2), BF), z=Fake((N, wide), BF))):
        with pytest.raises(B.MoeError) as e:
            router.expert_ffn_backward(**{**plain, **more})
        assert e.value.status == CAP
    assert c.launched == []


def test_the_sizes_that_the_binding_lets_through_are_those_of_the_c_code(tmp_path):
    want = _printed(tmp_path, "expert_product.h", [" && ".join(f"expert_product_fits({n}ll, {a}ll, {b}ll, {p})" for x, y in ((cols, n_in), (n_out, cols // 2))
                                                               for a, b in ((x, y), (y, x))) for n, n_in, cols, n_out, p in SPREAD])
    got = [B._network_status(*sizes) for sizes in SPREAD]
    assert got == [OK if w else CAP for w in want] and 0 < sum(want) < len(want)
    grads = _printed(tmp_path, "expert_product.h", [" && ".join(f"weight_grad_fits({n}ll, {a}ll, {b}ll, {p})" for a, b in ((cols, n_in), (n_out, cols // 2)))
                                                    for n, n_in, cols, n_out, p in SPREAD])
    got = [B._network_status(*sizes, True) for sizes in SPREAD]
    both = [w and g for w, g in zip(want, grads)]
    assert got == [OK if b else CAP for b in both] and sum(both) < sum(want)
