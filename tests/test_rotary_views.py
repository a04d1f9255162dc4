"""Queries and keys without heads, tokens or elements, as the binding sees them."""
import pytest

from paper_2412_12487_gb300 import echo as E

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("shape", [(1, 2, 3, 0, 6), (2, 0, 3, 4, 6), (2, 3, 0, 4, 6), (2, 3, 4, 0, 0), (2, 3, 0, 0, 6), (1, 1, 2, 3, 0, 8)])
@pytest.mark.parametrize("out", [False, True])
def test_views_without_elements(shape, out):
    tokens = 1
    for s in shape[:-2]:
        tokens *= s
    t, batch, n, strides = E._heads(torch.zeros(shape), out)
    assert (batch, n, len(strides)) == (1, tokens, 3) and t.shape[-2:] == shape[-2:]


@pytest.mark.gpu
@pytest.mark.parametrize("strided", [False, True])
def test_calls_without_heads_or_tokens(strided):
    """Of five dimensions, as of four: nothing to turn in one array, the other as ever."""
    f = E.rotary_frequencies(6)
    at = torch.arange(6, device="cuda").view(1, 2, 3)
    k = torch.randn((1, 2, 3, 4, 8), device="cuda")[..., :7 if strided else 8]
    with E.Echo(0) as e:
        want = e.rotary(k.reshape(6, 4, -1), None, at.view(6), f).view_as(k)
        none = k[:, :, :, :0]
        q, got = e.rotary(none, k, at, f)
        assert q.shape == none.shape and torch.equal(got, want)
        got, q = e.rotary(k, none, at, f, out=(torch.empty_like(k), torch.empty_like(none)))
        assert q.shape == none.shape and torch.equal(got, want)
        assert e.rotary(k[:, :0], k[:, :0], at[:, :0], f)[1].shape == (1, 0, 3, 4, k.shape[-1])
        assert e.rotary_grad(none, None, at, f).shape == none.shape
