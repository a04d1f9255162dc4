"""Operators of a training step against plain 64-bit implementations.

Tolerances are bounds on rounding, written down before the first run.  u = 2^-24 is fp32's unit roundoff, uo the output
type's (0 where the output is fp32 and its last rounding is counted with the others):

* lookup: one product in fp32 and one rounding.
* sums of n terms in fp32 (embedding gradient, weight gradients): each term takes part in at most n roundings, and in any
  tree far fewer; (n + 4) u times the sum of the terms' magnitudes holds for every order.
* layer norm: a row's sums run over at most 64 terms a thread and then a tree of at most 10 + 32 additions, so mean and
  variance are within 128 u of the magnitudes summed; the row's outputs inherit that, and the subtraction of the mean
  adds u times the largest element over the deviation.
* Newton-Schulz: a step multiplies an error by at most 3.9 (the largest slope of the quintic on [0, 1.2]) while the
  iterate grows by up to 3.44, and adds three products' roundings; five steps stay below 100 e of the result's norm,
  with e = 2^-22 for fp32 matrices and 2^-11 for 16-bit ones, and the output's own rounding.  An iterate of rank one
  starts at its final norm and does not grow: there the errors of each step are multiplied by all that follow, and the sum
  of 3.9^k over five steps is 1210.
"""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2412_12487_gb300 import Echo, EchoError
from paper_2412_12487_gb300 import echo as E
from paper_2412_12487_gb300 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
UO = {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}  # smallest step near zero


@pytest.fixture(scope="module")
def echo():
    with Echo(0) as e:
        yield e


def _randn(shape, seed, dtype=F32, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std + mean).to(dtype)


def _ids(n, lo, hi, seed, dtype=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(lo, hi, (n,), generator=g, device="cuda").to(dtype)


def _close(got, want, tol, dtype):
    """|got - want| <= tol + one rounding of the output, element by element; NaN and infinities alike."""
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    off = (got - want).abs() - (tol + UO[dtype] * (want.abs() + tol) + TINY[dtype])
    assert fine.sum() == 0 or float(torch.where(fine, off, torch.full_like(off, -1.0)).max()) <= 0, float(off[fine].max())


# -- embedding ---------------------------------------------------------------------------------
def _embed_ref(ids, table, scale, v0):
    row = ids.long() - v0
    mine = (row >= 0) & (row < table.shape[0])
    out = torch.zeros((*ids.shape, table.shape[1]), dtype=torch.float64, device="cuda")
    out[mine] = table.double()[row[mine]] * float(np.float32(scale))
    return out


@pytest.mark.parametrize("table_t,out_t", [(F32, F32), (F32, BF16), (BF16, BF16), (F16, F32), (BF16, F16), (F16, F16)])
@pytest.mark.parametrize("n,h,v,v0", [(1, 1, 1, 0), (3, 7, 5, 2), (33, 64, 40, 10), (257, 1030, 300, 0), (130, 4099, 64, 32), (64, 12288, 16, 8)])
def test_embed(echo, table_t, out_t, n, h, v, v0):
    table = _randn((v, h), 1, table_t)
    for bits in (torch.int64, torch.int32):
        ids = _ids(n, -2, v0 + v + 3, 2, bits)
        got = echo.embed(ids, table, scale=1.5, vocab_start=v0, dtype=out_t)
        assert got.dtype == out_t and got.shape == (n, h)
        want = _embed_ref(ids, table, 1.5, v0)
        _close(got, want, U * want.abs(), out_t)


def test_embed_no_tokens_no_rows_and_masked_rows(echo):
    table = _randn((4, 16), 3)
    assert echo.embed(torch.empty(0, dtype=torch.int64, device="cuda"), table).shape == (0, 16)
    ids = torch.tensor([0, -1, 2 ** 62, -2 ** 63, 2 ** 63 - 1, 3], device="cuda")
    assert torch.equal(echo.embed(ids, torch.empty((0, 16), device="cuda")), torch.zeros((6, 16), device="cuda"))
    table[1:3] = float("nan")  # rows that no token has
    out = echo.embed(ids, table, scale=float("inf"), vocab_start=0)
    assert torch.equal(out[1:5], torch.zeros((4, 16), device="cuda"))
    assert torch.equal(out[0], table[0] * float("inf"))


@pytest.mark.parametrize("h", [64, 65, 66])
def test_embed_strides_and_shapes(echo, h):
    base = _randn((10, h + 9), 4, BF16)
    table = base[:, 3:3 + h]  # odd address, rows apart
    ids = _ids(24, 0, 10, 5).view(2, 3, 4)
    out = torch.full((24, h + 5), 7.0, dtype=BF16, device="cuda")
    view = out[:, 1:1 + h]
    got = echo.embed(ids.view(-1), table, out=view)
    assert got.data_ptr() == view.data_ptr()
    assert torch.equal(view, table[ids.view(-1)])
    assert (out[:, 0] == 7).all() and (out[:, 1 + h:] == 7).all()
    assert torch.equal(echo.embed(ids, table), table[ids])
    assert torch.equal(echo.embed(ids.transpose(0, 2), table), table[ids.transpose(0, 2)])


def _embed_grad_ref(ids, dy, v, scale, v0, old=None):
    row = ids.reshape(-1).long() - v0
    dy = dy.reshape(-1, dy.shape[-1]).double()
    total = torch.zeros((v, dy.shape[-1]), dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    mine = (row >= 0) & (row < v)
    total.index_put_((row[mine],), dy[mine], accumulate=True)
    size.index_put_((row[mine],), dy[mine].abs(), accumulate=True)
    s = float(np.float32(scale))
    count = torch.bincount(row[mine], minlength=v)[:, None] if v else torch.zeros((0, 1), device="cuda")
    tol = (count + 4) * U * abs(s) * size
    if old is not None:
        total, tol = total * s + old.double(), tol + 2 * U * (total * s + old.double()).abs()
        return total, tol
    return total * s, tol


@pytest.mark.parametrize("dy_t,table_t", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,h,v,v0,spread", [(1, 1, 1, 0, 1), (1, 264, 9, 3, 9), (31, 7, 5, 0, 5), (33, 1030, 300, 100, 500), (1000, 264, 300, 0, 7),
                                             (9001, 72, 70001, 5, 70100), (2500, 1536, 40, 0, 1), (700, 2, 66000, 60000, 130000)])
def test_embed_grad(echo, dy_t, table_t, accumulate, n, h, v, v0, spread):
    # spread: ids in [0, spread), so that 1 gives every token the same row, and more than v0 + v some to other shards
    ids = _ids(n, 0, spread, 6, torch.int32 if n % 2 else torch.int64) + (v0 if spread == 1 else 0)
    dy = _randn((n, h), 7, dy_t)
    old = _randn((v, h), 8, table_t)
    out = old.clone() if accumulate else None
    got = echo.embed_grad(ids, dy, v, scale=0.75, vocab_start=v0, dtype=table_t, out=out, accumulate=accumulate)
    want, tol = _embed_grad_ref(ids, dy, v, 0.75, v0, old if accumulate else None)
    _close(got, want, tol, table_t)
    again = echo.embed_grad(ids, dy, v, scale=0.75, vocab_start=v0, dtype=table_t, out=old.clone() if accumulate else None, accumulate=accumulate)
    assert torch.equal(got, again)


def test_embed_grad_touches_only_its_rows(echo):
    dy = _randn((6, 40), 9)
    ids = torch.tensor([2, 7, -1, 2, 100, 2], device="cuda")
    dy[2] = float("nan")  # a masked token's and another shard's gradients reach nothing
    dy[4] = float("inf")
    out = torch.full((8, 40), float("nan"), device="cuda")
    out[2] = 1
    got = echo.embed_grad(ids, dy, 8, out=out, accumulate=True)
    assert got is out
    assert torch.isnan(out[[0, 1, 3, 4, 5, 6, 7]]).all()
    _close(out[2], 1 + dy[[0, 3, 5]].double().sum(0), 16 * U * (1 + dy[[0, 3, 5]].abs().double().sum(0)), F32)
    out = echo.embed_grad(ids, dy, 8, out=out)  # overwritten: no old value is left
    assert torch.equal(out[[0, 1, 3, 4, 5, 6]], torch.zeros((6, 40), device="cuda"))
    assert torch.equal(out[7], dy[1])
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert torch.equal(echo.embed_grad(none, dy[:0], 3), torch.zeros((3, 40), device="cuda"))
    before = out.clone()
    assert torch.equal(echo.embed_grad(none, dy[:0], 8, out=out, accumulate=True), before)
    assert torch.equal(echo.embed_grad(ids + 1000, dy, 8, out=out, accumulate=True), before)
    assert echo.embed_grad(ids, dy, 0).shape == (0, 40)


def test_embed_grad_strides(echo):
    ids = _ids(50, 0, 6, 10)
    wide = _randn((50, 90), 11, BF16)
    for h in (64, 33):
        dy = wide[:, 5:5 + h]
        out = torch.full((6, h + 3), 5.0, device="cuda")
        echo.embed_grad(ids, dy, 6, out=out[:, 2:2 + h])
        want, tol = _embed_grad_ref(ids, dy, 6, 1.0, 0)
        _close(out[:, 2:2 + h], want, tol, F32)
        assert (out[:, :2] == 5).all() and (out[:, 2 + h:] == 5).all()
    one = _randn((1, 64), 12, BF16).expand(50, 64)  # one gradient for every token
    want, tol = _embed_grad_ref(ids, one, 6, 1.0, 0)
    _close(echo.embed_grad(ids, one, 6), want, tol, F32)


def test_embed_grad_is_the_derivative(echo):
    # the lookup is linear: <dy, lookup(d)> = <gradient(dy), d> for every direction d of the table
    ids, dy, d = _ids(300, 0, 40, 13), _randn((300, 96), 14), _randn((32, 96), 15)
    left = (dy.double() * _embed_ref(ids, d, 1.25, 4)).sum()
    grad = echo.embed_grad(ids, dy, 32, scale=1.25, vocab_start=4)
    right = (grad.double() * d.double()).sum()
    size = (_embed_grad_ref(ids, dy.abs(), 32, 1.25, 4)[0] * d.double().abs()).sum()
    assert abs(float(left - right)) <= 304 * U * float(size)


# -- layer norm --------------------------------------------------------------------------------
def _ln_ref(x, w, b, eps):
    x = x.double()
    mean = x.mean(-1)
    d = x - mean[..., None]
    rstd = 1 / torch.sqrt((d * d).mean(-1) + float(np.float32(eps)))
    y = d * rstd[..., None]
    return (y if w is None else y * w.double()) + (0 if b is None else b.double()), mean, rstd


def _ln_tol(x, w, b, mean, rstd):
    x = x.double()
    peak = x.abs().amax(-1, keepdim=True)
    xh = (x - mean[..., None]).abs() * rstd[..., None]
    per = 128 * U * (peak * rstd[..., None] * (1 + 1 / math.sqrt(x.shape[-1])) + 2 * xh)
    return per * (1 if w is None else w.double().abs()) + (0 if b is None else 2 * U * b.double().abs())


LN_SHAPES = [(1, 1), (3, 2), (5, 31), (130, 257), (64, 1024), (37, 1537), (9, 2050), (6, 8200), (300, 2048), (5, 12288), (3, 32768), (2, 40002)]


@pytest.mark.parametrize("x_t,p_t", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (F32, BF16)])
@pytest.mark.parametrize("rows,h", LN_SHAPES)
def test_layer_norm(echo, x_t, p_t, rows, h):
    x = _randn((rows, h), 20, x_t, 2.0, 0.5)
    w, b = _randn((h,), 21, p_t, 0.2, 1.0), _randn((h,), 22, p_t)
    y, mean, rstd = echo.layer_norm(x, w, b, eps=1e-5)
    wy, wm, wr = _ln_ref(x, w, b, 1e-5)
    _close(mean, wm, 128 * U * x.double().abs().mean(-1), F32)
    peak = x.double().abs().amax(-1)
    _close(rstd, wr, wr * 128 * U * (1 + peak * wr), F32)
    _close(y, wy, _ln_tol(x, w, b, wm, wr), x_t)


def test_layer_norm_without_parameters_in_place_and_nd(echo):
    x = _randn((4, 5, 6, 96), 23, BF16)
    y, mean, rstd = echo.layer_norm(x)
    assert mean.shape == rstd.shape == (4, 5, 6)
    wy, wm, wr = _ln_ref(x, None, None, 1e-5)
    _close(y, wy, _ln_tol(x, None, None, wm, wr), BF16)
    w = _randn((96,), 24)
    only_w = echo.layer_norm(x, w)[0]
    wy, wm, wr = _ln_ref(x, w, None, 1e-5)
    _close(only_w, wy, _ln_tol(x, w, None, wm, wr), BF16)
    z = x.clone()
    assert echo.layer_norm(z, w, out=z)[0] is z and torch.equal(z, only_w)
    for h in (40000, 12288):
        x = _randn((3, h), 25)
        want = echo.layer_norm(x)[0]
        assert torch.equal(echo.layer_norm(x, out=x)[0], want)
    assert echo.layer_norm(x[:0])[0].shape == (0, 12288)


@pytest.mark.parametrize("h", [64, 65, 66, 1000])
def test_layer_norm_strides(echo, h):
    wide = _randn((20, h + 7), 26, F16)
    x = wide[:, 3:3 + h]
    out = torch.full((20, h + 6), 9.0, dtype=F16, device="cuda")
    y, mean, rstd = echo.layer_norm(x, out=out[:, 1:1 + h])
    want = echo.layer_norm(x.contiguous())
    assert torch.equal(y, want[0]) or _close(y, _ln_ref(x, None, None, 1e-5)[0], _ln_tol(x, None, None, want[1].double(), want[2].double()), F16) is None
    assert (out[:, 0] == 9).all() and (out[:, 1 + h:] == 9).all()
    one = x[:1].expand(20, h)
    assert torch.equal(echo.layer_norm(one)[0][7], echo.layer_norm(one)[0][0])
    t = _randn((h, 20), 27).t()  # columns of a row apart: taken as a copy
    wy, wm, wr = _ln_ref(t, None, None, 1e-5)
    _close(echo.layer_norm(t)[0], wy, _ln_tol(t, None, None, wm, wr), F32)


def test_layer_norm_special_rows(echo):
    x = _randn((6, 512), 28)
    x[1] = 3.0                      # no deviation
    x[2, 17] = float("nan")
    x[3, 5] = float("inf")
    x[4] = x[4] + 1e6               # a mean far above the deviation
    y, mean, rstd = echo.layer_norm(x, eps=1e-5)
    assert torch.equal(y[1], torch.zeros(512, device="cuda")) and abs(float(rstd[1]) - 1 / math.sqrt(1e-5)) < 1e-3
    assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all()
    keep = [0, 4, 5]
    wy, wm, wr = _ln_ref(x[keep], None, None, 1e-5)
    _close(y[keep], wy, _ln_tol(x[keep], None, None, wm, wr), F32)
    y = echo.layer_norm(torch.full((1, 64), 2.0, device="cuda"), eps=0.0)[0]
    assert torch.isnan(y).all()  # 0 / 0, as the formula has it


def _ln_grad_ref(dy, x, mean, rstd, w):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (x - mean) * rstd
    g = dy if w is None else dy * w.double()
    m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = rstd * (g - m1 - xh * m2)
    # errors: the sums within 128 u of the magnitudes summed, xh within 4 u of (|x| + |mean|) rstd
    exh = 4 * U * (x.abs() + mean.abs()) * rstd
    e1 = 128 * U * g.abs().mean(1, keepdim=True)
    e2 = 128 * U * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * exh).mean(1, keepdim=True)
    tx = rstd * (8 * U * (g.abs() + m1.abs() + (xh * m2).abs()) + e1 + xh.abs() * e2 + exh * m2.abs())
    n = dy.shape[0] + 4
    tw = n * U * (dy * xh).abs().sum(0) + (dy.abs() * exh).sum(0)
    return (dx, (dy * xh).sum(0), dy.sum(0)), (tx, tw, n * U * dy.abs().sum(0))


@pytest.mark.parametrize("x_t,p_t", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("rows,h", LN_SHAPES + [(2000, 96), (1201, 640), (700, 3000)])
def test_layer_norm_grad(echo, x_t, p_t, rows, h):
    x, dy = _randn((rows, h), 30, x_t, 2.0, 0.5), _randn((rows, h), 31, x_t)
    w = _randn((h,), 32, p_t, 0.2, 1.0)
    _, mean, rstd = echo.layer_norm(x, w)
    want, tol = _ln_grad_ref(dy, x, mean, rstd, w)
    got = echo.layer_norm_grad(dy, x, mean, rstd, w)
    for g, v, t, d in zip(got, want, tol, (x_t, p_t, p_t)):
        assert g.dtype == d
        _close(g, v, t, d)
    old = [_randn((h,), 33 + k, p_t) for k in range(2)]
    sums = [o.clone() for o in old]
    got2 = echo.layer_norm_grad(dy, x, mean, rstd, w, dweight=sums[0], dbias=sums[1], accumulate=True)
    assert got2[1] is sums[0] and got2[2] is sums[1] and torch.equal(got2[0], got[0])
    for g, v, t, o in zip(sums, want[1:], tol[1:], old):
        _close(g, v + o.double(), t + 2 * U * (v + o.double()).abs(), p_t)
    again = echo.layer_norm_grad(dy, x, mean, rstd, w)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_layer_norm_grad_forms(echo):
    x, dy = _randn((50, 200), 40), _randn((50, 200), 41)
    _, mean, rstd = echo.layer_norm(x)
    want, tol = _ln_grad_ref(dy, x, mean, rstd, None)
    got = echo.layer_norm_grad(dy, x, mean, rstd)
    for g, v, t in zip(got, want, tol):
        _close(g, v, t, F32)
    for target in ("dy", "x"):  # dx in place of an input
        a, b = dy.clone(), x.clone()
        g2 = echo.layer_norm_grad(a, b, mean, rstd, dx=a if target == "dy" else b)
        assert all(torch.equal(p, q) for p, q in zip(got, g2))
    wide = _randn((50, 211), 42)
    xs, one = wide[:, 3:203], dy[:1].expand(50, 200)  # apart rows; a broadcast gradient
    _, mean, rstd = echo.layer_norm(xs)
    want, tol = _ln_grad_ref(one, xs, mean, rstd, None)
    out = torch.full((50, 207), 4.0, device="cuda")
    got = echo.layer_norm_grad(one, xs, mean, rstd, dx=out[:, 5:205])
    for g, v, t in zip(got, want, tol):
        _close(g, v, t, F32)
    assert (out[:, :5] == 4).all() and (out[:, 205:] == 4).all()
    x = _randn((2, 3, 4, 32), 43, BF16)  # more dimensions
    _, mean, rstd = echo.layer_norm(x)
    got = echo.layer_norm_grad(x, x, mean, rstd)
    assert got[0].shape == x.shape
    none = torch.empty((0, 200), device="cuda")
    dx, dw, db = echo.layer_norm_grad(none, none, none[:, 0].contiguous(), none[:, 0].contiguous())
    assert dx.shape == (0, 200) and torch.equal(dw, torch.zeros(200, device="cuda")) and torch.equal(db, dw)
    keep = torch.ones(200, device="cuda")
    echo.layer_norm_grad(none, none, none[:, 0].contiguous(), none[:, 0].contiguous(), dweight=keep, dbias=keep.clone(), accumulate=True)
    assert (keep == 1).all()


@pytest.mark.parametrize("h", [200, 40002])
def test_layer_norm_grad_parts_alone(echo, h):
    """The C entry point computes only the gradients that are asked for."""
    x, dy = _randn((20, h), 44), _randn((20, h), 45)
    _, mean, rstd = echo.layer_norm(x)
    full = echo.layer_norm_grad(dy, x, mean, rstd)
    for ask in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 0, 1), (0, 0, 0)):
        outs = [torch.full_like(f, 3.0) for f in full]
        d = E.LayerNormGradDesc(20, h, dy.data_ptr(), x.data_ptr(), None, mean.data_ptr(), rstd.data_ptr(),
                                *[o.data_ptr() if a else None for o, a in zip(outs, ask)], h, h, h, 0, 0, 0)
        assert echo.lib.echo_layer_norm_grad(echo.h, C.byref(d)) == 0
        for o, f, a in zip(outs, full, ask):
            assert torch.equal(o, f if a else torch.full_like(f, 3.0))


def test_layer_norm_grad_is_the_derivative(echo):
    """Central differences of the 64-bit forward pass along a direction of each input."""
    rows, h = 7, 300
    x, w, b, dy = _randn((rows, h), 50), _randn((h,), 51), _randn((h,), 52), _randn((rows, h), 53)
    _, mean, rstd = echo.layer_norm(x, w, b)
    dx, dw, db = echo.layer_norm_grad(dy, x, mean, rstd, w)

    def loss(x, w, b):
        return float((_ln_ref(x, w, b, 1e-5)[0] * dy.double()).sum())

    step = 1e-5
    for k, (g, at) in enumerate(zip((dx, dw, db), (x, w, b))):
        v = _randn(at.shape, 54 + k).double()
        args = [x.double(), w.double(), b.double()]
        up, down = list(args), list(args)
        up[k] = args[k] + step * v
        down[k] = args[k] - step * v
        slope = (loss(*up) - loss(*down)) / (2 * step)
        # third derivatives times step^2, and the gradient's own rounding
        size = float((g.double().abs() * v.abs()).sum()) + 1
        assert abs(slope - float((g.double() * v).sum())) <= 1e-5 * size


# -- orthogonalised updates --------------------------------------------------------------------
def _ortho_ref(g, steps, coef, eps, scale):
    a, b, c = (float(np.float32(v)) for v in coef)
    x = g.double()
    x = x / (x.flatten(-2).norm(dim=-1)[..., None, None] + float(np.float32(eps)))
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    for _ in range(steps):
        q = x @ x.mT
        x = a * x + (b * q + c * q @ q) @ x
    return scale * (x.mT if tall else x)


QUINTIC = (3.4445, -4.7750, 2.0315)


def _ortho_close(got, want, dtype, gain=100):
    e = 2.0 ** -22 if dtype == F32 else 2.0 ** -11
    for g, w in zip(got.double().flatten(0, -3) if got.dim() > 2 else got.double()[None], want.flatten(0, -3) if want.dim() > 2 else want[None]):
        assert torch.isfinite(g).all()
        assert float((g - w).norm()) <= (gain * e + UO[dtype]) * float(w.norm())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(1, 1), (1, 9), (9, 1), (16, 16), (2, 33), (100, 257), (257, 100), (3, 64, 130), (128, 128), (129, 127), (2, 3, 40, 70),
                                   (300, 1000), (513, 512), (5, 384, 256)])
def test_orthogonalize(echo, dtype, shape):
    g = _randn(shape, 60, dtype, 1e-2)
    got = echo.orthogonalize(g)
    assert got.shape == g.shape and got.dtype == dtype
    _ortho_close(got, _ortho_ref(g, 5, QUINTIC, 1e-7, 1.0), dtype)
    assert torch.equal(got, echo.orthogonalize(g))


@pytest.mark.parametrize("steps,coef,scale", [(0, QUINTIC, 1.0), (1, QUINTIC, 0.5), (12, (1.875, -1.25, 0.375), 1.0), (3, (1.5, -0.5, 0.0), 2.0)])
def test_orthogonalize_steps_and_coefficients(echo, steps, coef, scale):
    g = _randn((60, 200), 61)
    got = echo.orthogonalize(g, steps=steps, coefficients=coef, scale=scale)
    want = _ortho_ref(g, steps, coef, 1e-7, scale)
    _ortho_close(got, want, F32)
    if steps == 12:  # converged: orthonormal rows
        assert float((got.double() @ got.double().mT - torch.eye(60, device="cuda", dtype=torch.float64)).abs().max()) < 1e-4


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_orthogonalize_sizes_of_values(echo, dtype):
    """The result does not depend on the matrix's scale, nor on its neighbours in the batch."""
    g = _randn((5, 48, 80), 62, dtype)
    want = _ortho_ref(g, 5, QUINTIC, 0.0, 1.0)
    sized = g.clone()
    for i, k in enumerate((0, 100, -100, 40, -60)):
        sized[i] = (g[i].double() * 2.0 ** k).to(dtype)
    _ortho_close(echo.orthogonalize(sized, eps=0.0), want, dtype)
    g[1] = 0
    g[2, 3, 4] = float("nan")
    g[3, 0, 0] = float("inf")
    got = echo.orthogonalize(g)
    assert torch.equal(got[1], torch.zeros_like(got[1]))
    assert torch.isnan(got[2]).any() and torch.isnan(got[3]).any()
    for i in (0, 4):
        _ortho_close(got[i], want[i], dtype)


def test_orthogonalize_low_rank_and_spiky(echo):
    g = torch.outer(_randn((70,), 63), _randn((300,), 64))
    _ortho_close(echo.orthogonalize(g), _ortho_ref(g, 5, QUINTIC, 1e-7, 1.0), F32, gain=1210)
    g = torch.zeros((70, 300), device="cuda")
    g[5, 7] = -3.0
    _ortho_close(echo.orthogonalize(g), _ortho_ref(g, 5, QUINTIC, 1e-7, 1.0), F32, gain=1210)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_orthogonalize_strides(echo, dtype):
    wide = _randn((3, 50, 91), 65, dtype)
    g = wide[:, 2:42, 3:73]
    out = torch.full((3, 44, 75), 6.0, dtype=dtype, device="cuda")
    view = out[:, 1:41, 2:72]
    want = echo.orthogonalize(g.contiguous())
    assert echo.orthogonalize(g, out=view) is view
    assert torch.equal(view, want)
    assert (out[:, 0] == 6).all() and (out[:, 41:] == 6).all() and (out[:, :, :2] == 6).all() and (out[:, :, 72:] == 6).all()
    assert torch.equal(echo.orthogonalize(g.mT), echo.orthogonalize(g.mT.contiguous()))
    z = g.contiguous()
    assert torch.equal(echo.orthogonalize(z, out=z), want)
    assert echo.orthogonalize(z[:0]).shape == (0, 40, 70)


# -- contexts, streams, refusals ---------------------------------------------------------------
def test_long_offsets(echo):
    """Arrays of more than 2^31 elements."""
    v, h = 180_000, 12288
    table = torch.zeros((v, h), dtype=BF16, device="cuda")
    table[-1] = 3
    ids = torch.tensor([v - 1, 0, v - 1], device="cuda")
    out = echo.embed(ids, table, scale=2.0)
    assert (out[0] == 6).all() and (out[1] == 0).all() and (out[2] == 6).all()
    echo.embed_grad(ids, out, v, out=table, accumulate=True)
    assert (table[-1] == 15).all() and (table[-2] == 0).all() and (table[0] == 0).all()
    table[-1] = _randn((h,), 70, BF16)
    y, mean, rstd = echo.layer_norm(table, out=table)
    del y
    wy, _, _ = _ln_ref(table[-1:], None, None, 1e-5)  # a normalised row stays, up to rounding
    assert float((wy - table[-1:].double()).abs().max()) < 0.05 and float(table[-1].double().std()) > 0.9
    dx, dw, db = echo.layer_norm_grad(table, table, mean, rstd, dx=table)
    assert torch.isfinite(dw).all() and float(db.abs().max()) > 0


@pytest.mark.parametrize("stream", ["own", "side"])
def test_other_streams(stream):
    """The order of torch's current stream holds whatever stream the context has."""
    side = torch.cuda.Stream()
    with Echo(0, stream=0 if stream == "own" else side) as e:
        for k in range(3):
            x = _randn((4000, 4096), 80 + k)
            x = x * 2 + 1  # pending work on the current stream
            y, mean, rstd = e.layer_norm(x)
            z = y.clone()  # reads the result in the current stream's order
            wy, wm, wr = _ln_ref(x[-3:], None, None, 1e-5)
            _close(z[-3:], wy, _ln_tol(x[-3:], None, None, wm, wr), F32)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            g = _randn((64, 64), 90)
            o = e.orthogonalize(g).clone()
        torch.cuda.current_stream().wait_stream(other)
        _ortho_close(o, _ortho_ref(g, 5, QUINTIC, 1e-7, 1.0), F32)


def test_operators_leave_the_composition_as_it_is(echo):
    c = W.config("tiny")
    g = W.build_gpt_graph(c)
    sc = W.make_scenarios(g, c, n_scen=4)
    with Echo(0) as e:
        e.load_graph(g)
        e.load_scenarios(sc)
        e.estimate_collectives()
        e.compose()
        want = e.read_makespan().copy()
        st, fn = e.read_times()
        e.layer_norm(_randn((64, 1024), 91))
        e.embed_grad(_ids(100, 0, 50, 92), _randn((100, 64), 93), 50)
        e.orthogonalize(_randn((64, 64), 94))
        st2, fn2 = e.read_times()
        assert np.array_equal(st, st2) and np.array_equal(fn, fn2) and np.array_equal(want, e.read_makespan())


def test_profile_names_the_operators(echo):
    with Echo(0) as e:
        e.set_profiling(True)
        x = _randn((8, 64), 95)
        _, mean, rstd = e.layer_norm(x)
        e.layer_norm_grad(x, x, mean, rstd)
        ids = _ids(8, 0, 4, 96)
        e.embed_grad(ids, e.embed(ids, x[:4]), 4)
        e.orthogonalize(x)
        p = e.read_profile()
        for prefix in ("embed", "embed_", "layer_norm", "layer_norm_grad", "ortho"):
            assert any(k.startswith(prefix) and n > 0 and ms > 0 for k, (n, ms) in p.items()), (prefix, p)


def test_refusals_in_python(echo):
    x = torch.zeros((4, 8), device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    s = torch.zeros(4, device="cuda")
    bad = [
        lambda: echo.embed(ids.float(), x),
        lambda: echo.embed(ids, x[0]),
        lambda: echo.embed(ids, x.double()),
        lambda: echo.embed(ids, x, out=torch.zeros((4, 7), device="cuda")),
        lambda: echo.embed(ids, x, out=torch.zeros((8, 4), device="cuda").t()),
        lambda: echo.embed(ids, x.cpu()),
        lambda: echo.embed(ids.cpu(), x),
        lambda: echo.embed(ids, x, vocab_start=-1),
        lambda: echo.embed_grad(ids, x[:3], 4),
        lambda: echo.embed_grad(ids, x, 4, accumulate=True),
        lambda: echo.embed_grad(ids, x, 4, out=torch.zeros((5, 8), device="cuda")),
        lambda: echo.embed_grad(ids, x, -1),
        lambda: echo.layer_norm(x, torch.zeros(7, device="cuda")),
        lambda: echo.layer_norm(x, torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda", dtype=BF16)),
        lambda: echo.layer_norm(x, eps=-1.0),
        lambda: echo.layer_norm(x, eps=float("nan")),
        lambda: echo.layer_norm(x.long()),
        lambda: echo.layer_norm(x[:, :0]),
        lambda: echo.layer_norm(x, out=x.to(BF16)),
        lambda: echo.layer_norm_grad(x, x[:3], s[:3], s[:3]),
        lambda: echo.layer_norm_grad(x, x, s[:3], s),
        lambda: echo.layer_norm_grad(x, x, s, s.double()),
        lambda: echo.layer_norm_grad(x, x, s, s, accumulate=True),
        lambda: echo.orthogonalize(x[0]),
        lambda: echo.orthogonalize(x, steps=-1),
        lambda: echo.orthogonalize(x, steps=65),
        lambda: echo.orthogonalize(x, coefficients=(float("nan"), 0, 0)),
        lambda: echo.orthogonalize(x[:, :0]),
        lambda: echo.orthogonalize(x, out=x.to(F16)),
    ]
    for k, f in enumerate(bad):
        with pytest.raises(EchoError) as err:
            f()
        assert err.value.code == 1, k
    # the context still works
    assert torch.equal(echo.embed(ids, x), x[ids])


def test_refusals_at_the_c_boundary(echo):
    lib, h = echo.lib, echo.h
    x = torch.zeros((4, 8), device="cuda")
    y = torch.full((4, 8), 2.0, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    px, py, pi = x.data_ptr(), y.data_ptr(), ids.data_ptr()
    host = np.zeros(64, np.float32).ctypes.data

    def code(fn, d):
        return getattr(lib, fn)(h, C.byref(d))

    for fn in ("echo_embed", "echo_embed_grad", "echo_layer_norm", "echo_layer_norm_grad", "echo_orthogonalize"):
        assert getattr(lib, fn)(h, None) == 1
    ok = (4, 8, 4, 0, pi, px, py, 8, 8, 64, 0, 0, 1.0)

    def embed(**kw):
        d = E.EmbedDesc(*ok)
        for k, v in kw.items():
            setattr(d, k, v)
        return code("echo_embed", d)

    assert embed(ids=None) == embed(table=None) == embed(out=None) == 1
    assert embed(n_tokens=-1) == embed(vocab_rows=-1) == embed(hidden=0) == embed(vocab_start=-5) == 1
    assert embed(hidden=(1 << 30) + 1) == 9
    assert embed(id_bits=16) == embed(table_type=3) == embed(out_type=-1) == 1
    assert embed(out_stride=7) == embed(table_stride=-1) == embed(out=py + 2) == embed(ids=pi + 4) == 1
    assert embed(table=host) == embed(out_stride=1 << 60) == 1
    d = E.EmbedGradDesc(4, 8, 4, 0, pi, px, py, 8, 8, 64, 0, 0, 0, 1.0)
    d.n_tokens = 1 << 31
    assert code("echo_embed_grad", d) == 9
    d.n_tokens, d.vocab_rows = 4, (1 << 31) - 1
    assert code("echo_embed_grad", d) == 9
    d.vocab_rows, d.dy = 4, None
    assert code("echo_embed_grad", d) == 1
    d = E.LayerNormDesc(4, 8, px, py, None, None, None, None, 8, 7, 0, 0, 1e-5)
    assert code("echo_layer_norm", d) == 1
    d = E.LayerNormDesc(4, 8, px, py, px + 1, None, None, None, 8, 8, 0, 0, 1e-5)
    assert code("echo_layer_norm", d) == 1
    d = E.LayerNormGradDesc(4, 8, px, px, None, None, px, py, None, None, 8, 8, 8, 0, 0, 0)
    assert code("echo_layer_norm_grad", d) == 1
    d = E.OrthogonalizeDesc(1, 70000, 8, px, py, 8, 0, 8, 0, 0, 5, 1.0, 0.0, 0.0, 0.0, 1.0)
    assert code("echo_orthogonalize", d) == 9
    d = E.OrthogonalizeDesc(2, 2, 8, px, py, 8, 16, 8, 15, 0, 5, 1.0, 0.0, 0.0, 0.0, 1.0)
    assert code("echo_orthogonalize", d) == 1
    torch.cuda.synchronize()
    assert (y == 2).all()  # nothing was enqueued
    buf = C.create_string_buffer(256)
    assert lib.echo_last_error(h, buf, 256) == 0 and buf.value
    assert embed() == 0


# -- sizes at which the kernels change their ways ----------------------------------------------
@pytest.mark.parametrize("n,v", [(5120, 51200), (5121, 51200), (32768, 300), (33000, 70000), (70001, 17), (40000, 1)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad_many_tokens(echo, n, v, accumulate):
    """Around the number of tokens that are sorted by counting, and that a sort's threads hold."""
    ids = _ids(n, -1, v + 2, 100)
    dy = _randn((n, 24), 101, BF16)
    old = _randn((v, 24), 102)
    got = echo.embed_grad(ids, dy, v, out=old.clone(), accumulate=accumulate)
    want, tol = _embed_grad_ref(ids, dy, v, 1.0, 0, old if accumulate else None)
    _close(got, want, tol, F32)
    assert torch.equal(got, echo.embed_grad(ids, dy, v, out=old.clone(), accumulate=accumulate))


@pytest.mark.parametrize("h", [8, 256, 257, 2048, 2049, 4096, 4097, 12288, 12289, 12296])
@pytest.mark.parametrize("x_t", [F32, BF16])
def test_layer_norm_row_lengths(echo, h, x_t):
    """Around the lengths at which a row's threads, or the kernel, change."""
    rows = 700 if h < 5000 else 170
    x, dy = _randn((rows, h), 110, x_t, 2.0, 0.5), _randn((rows, h), 111, x_t)
    w, b = _randn((h,), 112, F32, 0.2, 1.0), _randn((h,), 113)
    y, mean, rstd = echo.layer_norm(x, w, b)
    wy, wm, wr = _ln_ref(x, w, b, 1e-5)
    _close(y, wy, _ln_tol(x, w, b, wm, wr), x_t)
    want, tol = _ln_grad_ref(dy, x, mean, rstd, w)
    for g, v, t, d in zip(echo.layer_norm_grad(dy, x, mean, rstd, w), want, tol, (x_t, F32, F32)):
        _close(g, v, t, d)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(40, 3000), (3000, 40), (300, 5000), (2, 130, 4001), (1100, 1300), (7, 256, 512), (2500, 2600)])
def test_orthogonalize_split_sums(echo, dtype, shape):
    """Few tiles with long sums, which go in parts, and more tiles than one round takes."""
    g = _randn(shape, 120, dtype, 1e-2)
    got = echo.orthogonalize(g)
    _ortho_close(got, _ortho_ref(g, 5, QUINTIC, 1e-7, 1.0), dtype)
    assert torch.equal(got, echo.orthogonalize(g))


def test_orthogonalize_one_context_many_shapes(echo):
    """Calls of different sizes share scratch memory: none sees what another left there."""
    for k, (shape, dtype) in enumerate([((700, 900), F32), ((33, 2000), BF16), ((64, 64), F16), ((2000, 33), F32), ((3, 128, 300), BF16), ((700, 900), F32)]):
        g = _randn(shape, 130 + k, dtype)
        _ortho_close(echo.orthogonalize(g), _ortho_ref(g, 5, QUINTIC, 1e-7, 1.0), dtype)


def test_capture_in_a_graph():
    """After a first call of each size the operators can be captured and replayed."""
    side = torch.cuda.Stream()
    x, g, ids = _randn((64, 512), 140), _randn((96, 200), 141), _ids(64, 0, 50, 142)
    with Echo(0, stream=side) as e, torch.cuda.stream(side):
        def step():
            y, mean, rstd = e.layer_norm(x)
            dx, dw, db = e.layer_norm_grad(y, x, mean, rstd)
            return y, dx, dw, e.embed_grad(ids, dx, 50), e.orthogonalize(g)

        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step()
        x.mul_(1.5)
        g.add_(0.25)
        graph.replay()
        want = step()
        side.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("h", [200, 201, 2500, 13000])
def test_layer_norm_grad_far_from_zero(echo, h):
    """Rows that differ by 1 around 3000: x - mean comes before the product with rstd, so that
    (x - mean) rstd is within 3 u of itself, and not of |mean| rstd."""
    rows = 300
    x, dy, w = _randn((rows, h), 120, F32, 1.0, 3000.0), _randn((rows, h), 121), _randn((h,), 122, F32, 0.2, 1.0)
    _, mean, rstd = echo.layer_norm(x, w)
    g, xh, r = dy.double() * w.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None], rstd.double()[:, None]
    m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    e1, e2 = (132 * U * t.abs().mean(1, keepdim=True) for t in (g, g * xh))
    dx, dw, db = echo.layer_norm_grad(dy, x, mean, rstd, w)
    _close(dx, r * (g - m1 - xh * m2), r * (12 * U * (g.abs() + m1.abs() + (xh * m2).abs()) + e1 + xh.abs() * e2), F32)
    _close(dw, (dy * xh).sum(0), (rows + 8) * U * (dy * xh).abs().sum(0), F32)
    _close(db, dy.double().sum(0), (rows + 4) * U * dy.double().abs().sum(0), F32)


def test_captured_lengths_stay_launchable():
    """A shorter row's call between a longer one's capture and the graph's start takes none of
    the shared memory that the longer one asked for."""
    side = torch.cuda.Stream()
    xs = [_randn((400, h), 150 + h) for h in (12288, 5000)]  # slots of 48 KB and of 20 KB
    with Echo(0, stream=side) as e, torch.cuda.stream(side):
        def step():
            outs = [e.layer_norm(x) for x in xs]
            return [o[0] for o in outs] + [e.layer_norm_grad(o[0], x, o[1], o[2])[0] for o, x in zip(outs, xs)]

        want = step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step()
        graph.replay()
        side.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
