"""CPU tests of the operators' entry points: what they do without a device or a context."""
import ctypes as C

import pytest

from paper_2412_12487_gb300 import build as B
from paper_2412_12487_gb300 import echo as E

OPS = {"echo_embed": E.EmbedDesc, "echo_embed_grad": E.EmbedGradDesc, "echo_layer_norm": E.LayerNormDesc,
       "echo_layer_norm_grad": E.LayerNormGradDesc, "echo_orthogonalize": E.OrthogonalizeDesc}


@pytest.mark.parametrize("name", sorted(OPS))
def test_no_context_is_refused(name):
    B.build()
    lib = E.load_library()
    assert getattr(lib, name)(None, C.byref(OPS[name]())) == 1
    assert getattr(lib, name)(None, None) == 1


def test_no_context_has_no_stream():
    B.build()
    s = C.c_void_p()
    assert E.load_library().echo_stream_get(None, C.byref(s)) == 1


def test_views_as_rows_and_batches():
    torch = pytest.importorskip("torch")
    x = torch.arange(120.0).view(4, 5, 6)
    t, rows, stride = E._matrix(x)
    assert t is x and (rows, stride) == (20, 6)
    t, rows, stride = E._matrix(x[:, :, :4])
    assert (rows, stride) == (20, 6) and t.data_ptr() == x.data_ptr()
    v = x[:, :3, :4]  # rows not a fixed distance apart
    t, rows, stride = E._matrix(v)
    assert (rows, stride) == (12, 4) and torch.equal(t, v)
    with pytest.raises(E.EchoError):
        E._matrix(v, out=True)
    assert E._matrix(x[:0])[1:] == (0, 6)
    assert E._matrix(torch.zeros(7))[1:] == (1, 7)
    t, batch, rs, bs = E._batch(x[1:, 1:4, 2:])
    assert (batch, rs, bs) == (3, 6, 30) and t.data_ptr() == x[1:, 1:4, 2:].data_ptr()
    assert E._batch(x[0].t())[1:] == (1, 5, 30)
    with pytest.raises(E.EchoError):
        E._batch(x[0].t(), out=True)


def test_element_types():
    torch = pytest.importorskip("torch")
    assert [E._type(t) for t in (torch.float32, torch.bfloat16, torch.float16)] == [0, 1, 2]
    with pytest.raises(E.EchoError):
        E._type(torch.float64)
