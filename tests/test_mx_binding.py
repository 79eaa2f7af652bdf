"""CPU-only: what the binding of the 4-bit dispatch lets through to the C call, which cannot know a buffer's size.
Tensors are stand-ins that claim to be on a device; the C calls are replaced and only note that they were reached."""
import dataclasses

import pytest
import torch

from paper_2602_21140_b200 import binding as B


class Fake:
    """As much of a CUDA tensor as the binding looks at."""

    def __init__(self, shape, dtype, device=0, contiguous=True):
        self.shape, self.dtype, self._device, self._contiguous = torch.Size(shape), dtype, device, contiguous
        self.is_cuda = device >= 0

    def is_contiguous(self):
        return self._contiguous

    def get_device(self):
        return self._device

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def new_empty(self, shape, dtype=None):
        return Fake(shape, dtype or self.dtype, self._device)


T, H, E, K, R, S = 8, 64, 8, 2, 4, 2


@pytest.fixture
def router(monkeypatch):
    r = B.MoeRouter.__new__(B.MoeRouter)
    r.cfg = B.make_config(E, K, H, 64, R, S)
    r.device, r._ctx, r._latest = torch.device("cuda", 0), None, None
    reached = []
    for name in ("moe_mx_dispatch", "moe_mx_expert_gated", "moe_mx_expert_product", "moe_combine"):
        monkeypatch.setattr(B, name, lambda *a, _n=name: reached.append(_n) or B.MOE_OK)
    monkeypatch.setattr(B, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(B, "_on_device", lambda index, call, *args: call(*args))
    monkeypatch.setattr(B.MoeRouter, "_stream", lambda self: 0)
    r.reached = reached
    return r


def _out(tokens=T, device=0, ranks=R, slots=R * S, k=K):
    i, f, n = torch.int32, torch.float32, tokens * k
    return B.DispatchBuffers(Fake((tokens, k), i, device), Fake((tokens, k), f, device), Fake((tokens, k), i, device),
                             Fake((slots,), i, device), Fake((slots + 1,), i, device), Fake((ranks,), i, device),
                             Fake((ranks + 1,), i, device), Fake((n,), i, device), Fake((n,), i, device), None)


def _inputs():
    return Fake((T, E), torch.float32), Fake((T, H), torch.bfloat16)


def test_buffers_of_this_dispatch_pass(router):
    router.mx_dispatch(*_inputs(), _out())
    router.mx_dispatch(*_inputs(), _out(tokens=T + 3))       # allocated for more tokens than come this time
    assert router.reached == ["moe_mx_dispatch"] * 2


@pytest.mark.parametrize("out", [_out(tokens=T - 1), _out(device=1), _out(device=-1), _out(ranks=2), _out(slots=7),
                                 _out(k=1)], ids=["smaller T", "other device", "CPU", "fewer ranks", "fewer slots", "smaller k"])
def test_buffers_of_another_dispatch_are_refused(router, out):
    with pytest.raises(B.MoeError):
        router.mx_dispatch(*_inputs(), out)
    assert router.reached == []


@pytest.mark.parametrize("field", [f.name for f in dataclasses.fields(B.DispatchBuffers) if f.name != "send_buf"])
def test_every_buffer_is_looked_at(router, field):
    good = getattr(_out(), field)
    for bad in (Fake(good.shape, torch.int64), Fake(good.shape, good.dtype, contiguous=False), Fake(good.shape, good.dtype, device=1),
                Fake(tuple(good.shape)[:-1] + (good.shape[-1] - 1,), good.dtype)):
        with pytest.raises(B.MoeError):
            router.mx_dispatch(*_inputs(), dataclasses.replace(_out(), **{field: bad}))
    assert router.reached == []


def _rows(*shape):
    pitch = (shape[-1] // 32 + 15) // 16 * 16
    return B.MxRows(Fake((*shape[:-1], shape[-1] // 2), torch.uint8), Fake((*shape[:-1], pitch), torch.uint8))


I = 96


def _step(router, y=None, gate_up=None, down=None):
    router.mx_step(*_inputs(), gate_up or _rows(R * S, 2 * I, H), down or _rows(R * S, H, I), _out(), y)


def test_a_whole_step_passes(router):
    _step(router, Fake((T, H), torch.bfloat16))
    assert router.reached == ["moe_mx_dispatch", "moe_mx_expert_gated", "moe_mx_expert_product", "moe_combine"]


@pytest.mark.parametrize("args", [
    dict(y=Fake((T - 1, H), torch.bfloat16)), dict(y=Fake((T, H - 32), torch.bfloat16)), dict(y=Fake((T, H), torch.float32)),
    dict(y=Fake((T, H), torch.bfloat16, device=1)), dict(y=Fake((T, H), torch.bfloat16, contiguous=False)),
    dict(down=_rows(R * S, H - 32, I)), dict(down=_rows(R * S, H, I - 32)), dict(gate_up=_rows(R * S * 2 * I, H)),
    dict(down=_rows(R * S * H, I)), dict(gate_up=_rows(R * S - 1, 2 * I, H)), dict(gate_up=_rows(R * S, 2 * I, H + 32)),
    dict(gate_up=_rows(R * S, 2 * I - 32, H))],
    ids=["rows of y", "columns of y", "type of y", "device of y", "strides of y", "features", "hidden", "flat gate_up", "flat down", "slots", "columns",
         "half a block of pairs"])
def test_a_step_is_refused_before_its_first_launch(router, args):
    """Above all a y that the combine, which takes its size on trust, would write past its end."""
    with pytest.raises(B.MoeError):
        _step(router, **args)
    assert router.reached == []


def test_a_router_stays_on_the_device_that_it_was_made_on(monkeypatch):
    """device="cuda" means the device that is current when the context is made, not at the first 4-bit call."""
    import contextlib
    current = [1]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(B.MoeRouter, "_stream", lambda self: 0)
    monkeypatch.setattr(B, "moe_route_init", lambda *a: (B.MOE_OK, object()))
    monkeypatch.setattr(B, "moe_route_destroy", lambda ctx: B.MOE_OK)
    r = B.MoeRouter(B.make_config(E, K, H, 64, R, S), range(R * S), None, [1.0] * (R * S), device="cuda")
    current[0] = 0
    assert r._index() == 1 and r.device == torch.device("cuda", 1)
    r.close()
