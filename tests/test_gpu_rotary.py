"""Rotary positions and their gradient against a plain 64-bit implementation.

Tolerances, written down before the first run (U = 2^-24): an angle is within 2^-64 of a turn times the position, and a
fp32 number of half turns of at most 1 is within U / 2 of it, so that the angle is within pi U / 2; sine and cosine are
within 2 U of theirs, and scaled with one rounding: 5 U in all of the scale, for each of two products and a sum (2 U
more): 8 U of scale (|a| + |b|), and the output's rounding.
"""
import math

import numpy as np
import pytest

from paper_2412_12487_gb300 import Echo, EchoError, rotary_frequencies

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
UO = {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}


@pytest.fixture(scope="module")
def echo():
    with Echo(0) as e:
        yield e


def _randn(shape, seed, dtype=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _angles(positions, f):
    """Positions times frequencies modulo a turn, from exact integers: frequencies as fractions of 2^-200 turns."""
    from fractions import Fraction

    import sympy
    turn = Fraction(str(sympy.N(1 / (2 * sympy.pi), 90)))
    parts = [Fraction(float(x)) * turn for x in f]
    rows = [[float((int(p) * q) % 1) * 2 * math.pi for q in parts] for p in positions.reshape(-1).tolist()]
    return torch.tensor(rows, dtype=torch.float64, device="cuda").reshape(*positions.shape, len(f))


def _check(got, x, angle, interleaved, scale, back=False):
    rot = 2 * angle.shape[-1]
    scale = float(np.float32(scale))
    d = x.double()
    a, b = (d[..., 0:rot:2], d[..., 1:rot:2]) if interleaved else (d[..., :rot // 2], d[..., rot // 2:rot])
    c, s = torch.cos(angle)[..., None, :] * scale, torch.sin(angle)[..., None, :] * (-scale if back else scale)
    y0, y1, size = a * c - b * s, a * s + b * c, (a.abs() + b.abs()) * abs(scale)
    lay = (lambda p, q: torch.stack((p, q), -1).flatten(-2)) if interleaved else (lambda p, q: torch.cat((p, q), -1))
    want, tol = lay(y0, y1), lay(size, size) * 8 * U
    g = got.double()
    dtype = x.dtype
    assert got.dtype == dtype and got.shape == x.shape
    assert torch.equal(got[..., rot:], x[..., rot:])
    off = (g[..., :rot] - want).abs() - (tol + UO[dtype] * (want.abs() + tol) + TINY[dtype])
    assert off.numel() == 0 or float(off.max()) <= 0, float(off.max())


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,kv,dim,rot", [(1, 1, 1, 2, 2), (1, 32, 8, 128, 128), (7, 3, 1, 80, 20), (33, 5, 5, 65, 64), (130, 12, 12, 128, 128),
                                                     (9, 2, 1, 256, 256), (5, 3, 2, 600, 512), (3, 70, 1, 96, 2), (2, 1, 1, 7, 6), (300, 1, 1, 16, 4)])
def test_rotary(echo, dtype, interleaved, tokens, heads, kv, dim, rot):
    q, k = _randn((tokens, heads, dim), 1, dtype), _randn((tokens, kv, dim), 2, dtype)
    f = rotary_frequencies(rot)
    g = torch.Generator(device="cuda").manual_seed(3)
    for bits, far in ((torch.int64, 2 ** 40), (torch.int32, 2 ** 31 - 1), (torch.int64, 300)):
        at = torch.randint(-far, far, (tokens,), generator=g, device="cuda").to(bits)
        angle = _angles(at, f)
        got = echo.rotary(q, k, at, f, interleaved=interleaved, scale=1.25)
        _check(got[0], q, angle, interleaved, 1.25)
        _check(got[1], k, angle, interleaved, 1.25)
        back = echo.rotary_grad(q, k, at, f, interleaved=interleaved, scale=0.5)
        _check(back[0], q, angle, interleaved, 0.5, True)
        _check(back[1], k, angle, interleaved, 0.5, True)
        one = echo.rotary(q, None, at, f, interleaved=interleaved, scale=1.25)
        assert torch.equal(one, got[0])


def test_forms_and_strides(echo):
    f = rotary_frequencies(32, factor=4.0, length=2048)
    b, s, h, d = 3, 11, 6, 48
    for dtype in (BF16, F32):
        x = _randn((b, s, h, d), 4, dtype)
        at = torch.arange(s, device="cuda") + 100
        want = echo.rotary(x, None, at, f)
        _check(want, x, _angles(at.expand(b, s).contiguous(), f), False, 1.0)
        assert torch.equal(echo.rotary(x, None, at.expand(b, s), f), want)
        assert torch.equal(echo.rotary(x.view(b * s, h, d), None, at.repeat(b), f).view_as(x), want)
        assert torch.equal(echo.rotary(x[0, 0], None, at[0], f), want[0, 0])            # one token
        turned = x.transpose(1, 2).contiguous().transpose(1, 2)                          # heads before tokens
        assert torch.equal(echo.rotary(turned, None, at, f), want)
        out = torch.empty_like(turned)
        assert echo.rotary(turned, None, at, f, out=out) is out and torch.equal(out, want)
        five = x.view(1, b, s, h, d)
        assert torch.equal(echo.rotary(five, None, at.expand(1, b, s), f), want.view_as(five))
        # packed query, key and value: both parts in place, the values and the gaps stay
        packed = _randn((b, s, 10, d + 3), 5, dtype)
        keep = packed.clone()
        q, k = packed[:, :, :6, 1:1 + d], packed[:, :, 6:8, 1:1 + d]
        wq, wk = echo.rotary(q.contiguous(), k.contiguous(), at, f)
        got = echo.rotary(q, k, at, f, out=(q, k))
        assert got[0] is q and torch.equal(q, wq) and torch.equal(k, wk)
        assert torch.equal(packed[:, :, 8:], keep[:, :, 8:]) and torch.equal(packed[..., 0], keep[..., 0]) and torch.equal(packed[..., 1 + d:], keep[..., 1 + d:])
        wide = x[:1].expand(b, s, h, d)                                                  # the same rows for each batch
        assert torch.equal(echo.rotary(wide, None, at, f), echo.rotary(x[:1].contiguous(), None, at, f).expand(b, s, h, d))
    assert echo.rotary(x[:0], None, at, f).shape == (0, s, h, d)
    assert echo.rotary(x[:, :, :0], x, at, f)[1].shape == x.shape


def test_the_gradient_turns_back_and_is_the_derivative(echo):
    f = rotary_frequencies(64)
    q, k, dq = _randn((50, 4, 64), 6), _randn((50, 2, 64), 7), _randn((50, 4, 64), 8)
    at = torch.arange(50, device="cuda") * 1000003
    for inter in (False, True):
        y = echo.rotary(q, k, at, f, interleaved=inter)
        x = echo.rotary_grad(*y, at, f, interleaved=inter)
        size = q.double().abs().amax() * 2
        assert float((x[0].double() - q.double()).abs().max()) <= 40 * U * float(size)
        # a linear map: <dq, turn(q)> = <gradient(dq), q>
        g = echo.rotary_grad(dq, None, at, f, interleaved=inter, scale=1.5)
        left = (dq.double() * echo.rotary(q, None, at, f, interleaved=inter, scale=1.5).double()).sum()
        right = (g.double() * q.double()).sum()
        assert abs(float(left - right)) <= 40 * U * 1.5 * float((dq.double().abs() * size).sum())


def test_far_offsets_streams_and_graphs(echo):
    f = rotary_frequencies(128)
    at = torch.arange(4, device="cuda")
    big = torch.empty(2 ** 31 + 4096, dtype=BF16, device="cuda")  # a last batch beyond 32 bits of elements
    x = big.as_strided((2, 2, 2, 128), (2 ** 31, 256, 128, 1))
    x.copy_(_randn((2, 2, 2, 128), 9, BF16))
    want = echo.rotary(x.contiguous(), None, at.view(2, 2), f)
    assert torch.equal(echo.rotary(x, None, at.view(2, 2), f), want)
    assert echo.rotary(x, None, at.view(2, 2), f, out=x) is x and torch.equal(x, want)
    del big, x
    q = _randn((600, 6, 128), 10, BF16)
    at = torch.arange(600, device="cuda")
    want = echo.rotary(q, None, at, f)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = echo.rotary(q, None, at, f)
    side.synchronize()
    assert torch.equal(got, want)
    with torch.cuda.stream(side), Echo(0, stream=side) as own:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = own.rotary(q, None, at, f)
            again = own.rotary_grad(out, None, at, f)
        at += 7
        graph.replay()
        side.synchronize()
    assert torch.equal(out, echo.rotary(q, None, at, f)) and torch.equal(again, echo.rotary_grad(out, None, at, f))


def test_special_elements(echo):
    f = rotary_frequencies(8)
    x = _randn((3, 2, 12), 11)
    x[1, 0, 2], x[2, 1, 9] = math.nan, math.inf
    at = torch.tensor([5, 6, -2 ** 63], device="cuda")
    y = echo.rotary(x, None, at, f)
    assert torch.isnan(y[1, 0, [2, 6]]).all() and torch.isnan(y).sum() == 2 and y[2, 1, 9] == math.inf
    zero = echo.rotary(x[:1], None, torch.zeros(1, dtype=torch.int32, device="cuda"), f)
    assert torch.equal(zero, x[:1])


def test_refusals(echo):
    q, k = _randn((5, 4, 16), 12), _randn((5, 2, 16), 13)
    at, f = torch.arange(5, device="cuda"), rotary_frequencies(16)
    for call in (lambda: echo.rotary(q, k, at[:4], f),
                 lambda: echo.rotary(q, k[:4], at, f),
                 lambda: echo.rotary(q, k.to(BF16), at, f),
                 lambda: echo.rotary(q, k, at.float(), f),
                 lambda: echo.rotary(q.double(), None, at, f),
                 lambda: echo.rotary(q, k, at, rotary_frequencies(18)),
                 lambda: echo.rotary(q, k, at, f[:0]),
                 lambda: echo.rotary(q, k, at, f * math.nan),
                 lambda: echo.rotary(q, k, at, f * 1e11),
                 lambda: echo.rotary(q, k, at, f, scale=math.inf),
                 lambda: echo.rotary(q, k, at, f, out=(q,)),
                 lambda: echo.rotary(q, None, at, f, out=q[:1].expand(5, 4, 16)),
                 lambda: echo.rotary(q, None, at, f, out=torch.empty((5, 16, 4), device="cuda").transpose(1, 2)),
                 lambda: echo.rotary(q.cpu(), None, at, f),
                 lambda: rotary_frequencies(15),
                 lambda: rotary_frequencies(16, length=100, low=2, high=1)):
        with pytest.raises(EchoError) as err:
            call()
        assert err.value.code == 1, err.value
    with pytest.raises(EchoError) as err:
        echo.rotary(_randn((1, 1, 600), 14), None, at[:1], rotary_frequencies(600))
    assert err.value.code == 9
