"""What the C entry points of the head's losses and of the rotary positions refuse, a field at a time, with the outputs as they were."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2412_12487_gb300 import Echo
from paper_2412_12487_gb300 import echo as E

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
INVALID, UNSUPPORTED = 1, 9


@pytest.fixture(scope="module")
def echo():
    with Echo(0) as e:
        yield e


def _call(echo, name, desc):
    rc = getattr(echo.lib, name)(echo.h, C.byref(desc))
    torch.cuda.synchronize()
    return rc


def _refused(echo, name, make, outs, changes):
    for out in outs:
        out.fill_(7)
    for field, value, code in changes:
        d = make()
        if isinstance(field, tuple):
            getattr(d, field[0])[field[1]] = value
        else:
            setattr(d, field, value)
        assert _call(echo, name, d) == code, (field, value)
        assert all((o == 7).all() for o in outs), (field, value)
    assert _call(echo, name, make()) == 0
    assert getattr(echo.lib, name)(echo.h, None) == INVALID


def _head():
    t = {"x": torch.randn((6, 16), device="cuda"), "w": torch.randn((9, 16), device="cuda"), "labels": torch.arange(6, device="cuda"),
         "ids": torch.randint(0, 9, (6, 3), device="cuda"), "t": torch.randn((6, 3), device="cuda"), "g": torch.ones(6, device="cuda"),
         "lse": torch.full((6,), 5.0, device="cuda")}
    return t, {k: v.data_ptr() for k, v in t.items()}


COMMON = [("n_tokens", -1, INVALID), ("hidden", 0, INVALID), ("vocab_rows", -1, INVALID), ("vocab_start", -1, INVALID), ("x", None, INVALID), ("weight", None, INVALID),
          ("x_stride", -1, INVALID), ("weight_stride", -1, INVALID), ("type", 3, INVALID), ("id_bits", 16, INVALID), ("scale", math.nan, INVALID),
          ("hidden", 2 ** 24 + 1, UNSUPPORTED), ("n_tokens", 2 ** 30 + 1, UNSUPPORTED), ("vocab_rows", 2 ** 30 + 1, UNSUPPORTED), ("x_stride", 2 ** 58, INVALID)]


def test_cross_entropy(echo):
    t, p = _head()
    out = [torch.empty(6, device="cuda") for _ in range(3)]
    host = np.zeros(200, np.float32)
    make = lambda: E.CrossEntropyDesc(6, 16, 9, 0, p["x"], p["w"], p["labels"], *(o.data_ptr() for o in out), 16, 16, 0, 64, 1.0)  # noqa: E731
    _refused(echo, "echo_cross_entropy", make, out, COMMON + [("labels", None, INVALID), ("labels", p["labels"] + 4, INVALID), ("x", p["x"] + 2, INVALID),
                                                             ("loss", out[0].data_ptr() + 1, INVALID), ("lse", host.ctypes.data, INVALID), ("x", host.ctypes.data, INVALID)])
    d = make()
    d.loss = d.target = None  # each may be missing
    out[1].fill_(0)
    assert _call(echo, "echo_cross_entropy", d) == 0 and (out[1] != 0).all()


def test_cross_entropy_grad(echo):
    t, p = _head()
    out = [torch.empty((6, 16), device="cuda"), torch.empty((9, 16), device="cuda")]
    a, b = (o.data_ptr() for o in out)
    make = lambda: E.CrossEntropyGradDesc(6, 16, 9, 0, p["g"], None, p["x"], p["w"], p["labels"], p["lse"], a, b, 16, 16, 16, 16, 0, 0, 64, 0, 1.0)  # noqa: E731
    _refused(echo, "echo_cross_entropy_grad", make, out, COMMON + [("labels", None, INVALID), ("dloss", None, INVALID), ("lse", None, INVALID), ("dx_stride", 15, INVALID),
                                                                  ("dweight_stride", 3, INVALID), ("dweight_type", -1, INVALID), ("dlse", p["g"] + 1, INVALID), ("dx", a + 2, INVALID)])


def test_distill(echo):
    t, p = _head()
    out = [torch.empty(6, device="cuda") for _ in range(3)]
    make = lambda: E.DistillDesc(6, 16, 9, 0, 3, p["x"], p["w"], p["ids"], p["t"], None, *(o.data_ptr() for o in out), 16, 16, 0, 64, 0, 1.0, 2.0)  # noqa: E731
    more = [("n_top", 0, INVALID), ("n_top", 257, UNSUPPORTED), ("temperature", 0.0, INVALID), ("temperature", -1.0, INVALID), ("temperature", math.inf, INVALID),
            ("logits", None, INVALID), ("ids", None, INVALID), ("logits_type", 5, INVALID), ("teacher_lse", 8, INVALID)]
    _refused(echo, "echo_distill", make, out, COMMON + more)
    grads = [torch.empty((6, 16), device="cuda"), torch.empty((9, 16), device="cuda")]
    a, b = (o.data_ptr() for o in grads)
    make = lambda: E.DistillGradDesc(6, 16, 9, 0, 3, p["g"], None, p["x"], p["w"], p["ids"], p["t"], None, p["lse"], a, b, 16, 16, 16, 16, 0, 0, 64, 0, 0, 1.0, 2.0)  # noqa: E731
    _refused(echo, "echo_distill_grad", make, grads, COMMON + more + [("dloss", None, INVALID), ("lse", None, INVALID)])


@pytest.mark.parametrize("name", ["echo_rotary", "echo_rotary_grad"])
def test_rotary(echo, name):
    x, out = torch.randn((2, 5, 4, 16), device="cuda"), torch.empty((2, 5, 4, 16), device="cuda")
    at, f = torch.arange(10, device="cuda"), np.ones(4)
    bad = np.array([1.0, 2.0, 2.0 ** 33, 1.0])
    make = lambda: E.RotaryDesc(2, 5, (4, 0), (x.data_ptr(), None), (out.data_ptr(), None), (320, 0), (64, 0), (16, 0), (320, 0), (64, 0), (16, 0),  # noqa: E731
                                at.data_ptr(), 5, f.ctypes.data, 16, 8, 0, 64, 0, 1.0)
    _refused(echo, name, make, [out], [
        ("n_batch", -1, INVALID), ("n_tokens", -1, INVALID), (("heads", 0), -1, INVALID), (("heads", 1), 1, INVALID), (("heads", 0), 65536, UNSUPPORTED), ("dim", 0, INVALID),
        ("dim", 7, INVALID), ("dim", 65537, UNSUPPORTED), ("rot", 0, INVALID), ("rot", 7, INVALID), ("rot", 18, INVALID), ("type", 9, INVALID), ("id_bits", 8, INVALID),
        ("scale", math.inf, INVALID), ("frequencies", None, INVALID), ("frequencies", bad.ctypes.data, INVALID), ("positions", None, INVALID), ("positions_stride", -1, INVALID),
        (("x", 0), None, INVALID), (("out", 0), x.data_ptr() + 2, INVALID), (("x_stride", 0), -1, INVALID), (("out_head_stride", 0), 15, INVALID), (("out_stride", 0), 63, INVALID),
        (("out_batch_stride", 0), 0, INVALID), (("x_batch_stride", 0), 2 ** 60, INVALID)])
