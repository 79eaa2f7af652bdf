"""CPU-only: which buffers a norm writes when its output object is used again.  Tensors are stand-ins; the C call notes what it
is given."""
import pytest
import torch

from paper_2602_21140_b200 import binding as B
from test_expert_binding import BF, F32, H, T, Row, router  # noqa: F401 (a fixture)


@pytest.fixture
def calls(router, monkeypatch):  # noqa: F811
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: Row((shape,) if isinstance(shape, int) else shape, dtype))
    seen = []

    def norm(x, xs, res, rs, dt, rows, cols, w, wdt, eps, h, y, rstd, codes, scales, stream):
        seen.append(dict(x=x, res=res, h=h, y=y, codes=codes))
        return B.MOE_OK

    monkeypatch.setattr(B, "moe_rms_norm", norm)
    return seen


def _norm(x, res=None, **more):
    return B.rms_norm(x, Row((H,), BF), res, **more)


def test_a_callers_rows_are_no_output_of_a_later_call(calls):
    """Without a residual h is x itself; with the same `out` a later call has to write its h somewhere else."""
    x, x2, res = (Row((T, H), BF) for _ in range(3))
    out = _norm(x)
    assert out.h is x and calls[-1]["h"] == 0
    assert _norm(x2, res, out=out) is out
    assert calls[-1]["h"] not in (0, x.data_ptr(), x2.data_ptr(), res.data_ptr()) and out.h.data_ptr() == calls[-1]["h"]
    mine = out.h
    assert _norm(x, out=out).h is x and calls[-1]["h"] == 0
    _norm(x2, out=out)
    assert out.h is x2
    _norm(x, res, out=out)                                     # its own buffer again
    assert out.h is mine and calls[-1]["h"] == mine.data_ptr()


def test_a_given_buffer_for_h_outlives_a_call_without_a_residual(calls):
    x, res, h = (Row((T, H), BF) for _ in range(3))
    out = B.RmsNormOut(Row((T, H), BF), h, Row((T,), F32))
    _norm(x, out=out)
    assert out.h is x
    _norm(x, res, out=out)
    assert out.h is h and calls[-1]["h"] == h.data_ptr()
    _norm(x, out=out)
    out.h = res                                                # in the residual's place, as the caller says
    _norm(x, res, out=out)
    assert out.h is res and calls[-1]["h"] == calls[-1]["res"] == res.data_ptr()


def test_the_caller_may_put_the_same_rows_there(calls):
    """h in the residual's place, where the residual is the x of the call before."""
    stream, branch = Row((T, H), BF), Row((T, H), BF)
    out = _norm(stream)
    _norm(branch, stream, out=out)                             # not said: somewhere else
    assert calls[-1]["h"] not in (stream.data_ptr(), branch.data_ptr())
    out = _norm(stream)
    out.h = stream
    _norm(branch, stream, out=out)
    assert calls[-1]["h"] == calls[-1]["res"] == stream.data_ptr() and out.h is stream
    again = B.RmsNormOut(**vars(_norm(stream)))                # a copy knows it as well
    _norm(branch, stream, out=again)
    assert calls[-1]["h"] != stream.data_ptr()


def test_the_stream_of_a_stack_of_layers(calls):
    """x of one call is the h of the one before."""
    x, res = Row((T, H), BF), Row((T, H), BF)
    out = _norm(x, res)
    h = out.h
    _norm(out.h, out=out)
    assert out.h is h
    _norm(x, res, out=out)
    assert out.h is h and calls[-1]["h"] == h.data_ptr()


def test_a_refused_call_changes_nothing(calls):
    x, h = Row((T, H), BF), Row((T, H), BF)
    out = B.RmsNormOut(Row((T, H), BF), h, Row((T,), F32))
    with pytest.raises(B.MoeError):
        _norm(x, out=out, keep=True)                           # there is no buffer for the 8-bit rows
    with pytest.raises(B.MoeError):
        _norm(Row((T - 1, H), BF), out=out)
    assert out.h is h and not calls
    borrowed = _norm(x)
    with pytest.raises(B.MoeError):
        _norm(x, Row((T, H), F32), out=borrowed)
    assert borrowed.h is x and len(calls) == 1
