"""Losses of a head at the ends of what they take: padding of any content, rows of very different sizes, signs, types and
layouts that go together, matrices beyond 2^31 elements, two contexts at a time.

Tolerances as in test_gpu_head.py; where a call has to give another call's bits, equality."""
import math

import pytest

from paper_2412_12487_gb300 import Echo

from .test_gpu_head import BF16, F16, F32, U, Ref, _case, _check_ce, _close, _randint, _randn, _teacher, _teacher_ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def echo():
    with Echo(0) as e:
        yield e


@pytest.mark.parametrize("dtype,dw_type", [(F32, F32), (BF16, F32), (F16, F16)])
def test_padding_of_any_size(echo, dtype, dw_type):
    n, h, v = 50, 72, 400
    x, w = _case(n, h, v, 0, dtype, 1)
    labels, dloss = _randint(0, v, (n,), 2), _randn((n,), 3)
    labels[1::4] = -1
    live = labels >= 0
    clean = echo.cross_entropy(x, w, labels)
    grads = echo.cross_entropy_grad(dloss, x, w, labels, clean[1], dtype=dw_type)
    y = x.clone()
    y[~live] = torch.finfo(dtype).max  # what memory may hold
    got = echo.cross_entropy(y, w, labels)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1][live], clean[1][live]) and torch.equal(got[2], clean[2])
    g2 = echo.cross_entropy_grad(dloss, y, w, labels, clean[1], dtype=dw_type)
    assert torch.equal(g2[0], grads[0]) and torch.equal(g2[1], grads[1])


def test_rows_of_different_sizes(echo):
    """fp32 tokens from 2^-60 to 2^40 times the others, each with the digits of its own size."""
    n, h, v = 40, 130, 300
    x, w = _case(n, h, v, 0, F32, 4)
    by = 2.0 ** torch.linspace(-60, 40, n, device="cuda").round()
    z = torch.cat([x * by[:, None], torch.zeros((1, h), device="cuda")])
    labels = _randint(0, v, (n + 1,), 5)
    loss, lse, target = echo.cross_entropy(z, w, labels, scale=2.0 ** -38)
    X, W = z.double(), w.double()
    size = X.abs() @ W.abs().T
    far = 2.0 ** -37 * (X.abs().amax(1, keepdim=True) * W.abs().sum(1)[None] + W.abs().max() * X.abs().sum(1)[:, None])
    units = (64 + h / 256) * U + 3 * 2.0 ** -22
    want = (X @ W.T).gather(1, labels[:, None])[:, 0] * 2.0 ** -38
    tol = ((units * size + far).gather(1, labels[:, None])[:, 0] + 4 * U * want.abs()) * 2.0 ** -38
    _close(target, want, tol)
    assert torch.isfinite(loss).all() and float(lse[n]) == pytest.approx(math.log(v), rel=1e-6)
    # and rows of the weight
    by = 2.0 ** torch.linspace(-60, 40, v, device="cuda").round()
    big = w * by[:, None]
    target = echo.cross_entropy(x, big, labels[:n], scale=2.0 ** -38)[2]
    X, W = x.double(), big.double()
    want = (X @ W.T).gather(1, labels[:n, None])[:, 0] * 2.0 ** -38
    far = 2.0 ** -37 * (X.abs().amax(1, keepdim=True) * W.abs().sum(1)[None] + W.abs().amax(1)[None] * X.abs().sum(1)[:, None])
    tol = ((units * (X.abs() @ W.abs().T) + far).gather(1, labels[:n, None])[:, 0] * 2.0 ** -38 + 4 * U * want.abs())
    _close(target, want, tol)


@pytest.mark.parametrize("scale", [-0.5, 0.0])
def test_signs_and_zero(echo, scale):
    n, h, v = 90, 40, 333
    for dtype, dw_type in ((BF16, F32), (F32, F32), (F16, F16)):
        x, w = _case(n, h, v, 0, dtype, 6)
        labels, dloss, dlse = _randint(-1, v, (n,), 7), _randn((n,), 8), _randn((n,), 9)
        lse = _check_ce(echo, x, w, labels, 0, scale)
        ref = Ref(x, w, scale)
        dx, dw = echo.cross_entropy_grad(dloss, x, w, labels, lse, scale=scale, dlse=dlse, dtype=dw_type)
        valid = labels >= 0
        g = torch.where(valid, dloss.double() * scale, 0.0)
        coef = g + dlse.double() * scale
        want = ref.targets(torch.where(valid, labels, -1)[:, None], g[:, None], 0)
        a, b, ta, tb = ref.grads(coef, g.abs(), want, lse.double(), 1.0, dw_type)
        more = (4 * U * (g.abs() + (dlse.double() * scale).abs()))[:, None] * torch.exp(ref.z - lse.double()[:, None])  # (the coefficient's sum)
        _close(dx, a, ta + more @ ref.W.abs())
        _close(dw, b, tb + more.T @ ref.X.abs())


def test_types_that_go_together(echo):
    """32-bit ids, teachers of another type than the student, a broadcast gradient, one token."""
    n, h, v, k = 33, 64, 500, 9
    x, w = _case(n, h, v, 0, BF16, 10)
    ids, logits = _teacher(n, k, v, 0, F32, 11)
    want = echo.distill(x, w, ids, logits.to(F16).float(), temperature=1.5)
    for t in (F32, F16):
        got = echo.distill(x, w, ids.int(), logits.to(F16).to(t), temperature=1.5)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    one = torch.full((1,), 0.25, device="cuda").expand(n)
    grads = echo.distill_grad(one.contiguous(), x, w, ids, logits, want[1], temperature=1.5)
    assert all(torch.equal(a, b) for a, b in zip(grads, echo.distill_grad(one, x, w, ids.int(), logits, want[1], temperature=1.5)))
    loss, lse, cross = echo.distill(x[0], w, ids[0], logits[0].to(F16), temperature=1.5)
    assert loss.shape == () and torch.equal(loss, want[0][0]) and torch.equal(lse, want[1][0])
    dx, dw = echo.distill_grad(one[0], x[0], w, ids[0], logits[0], lse, temperature=1.5)
    assert dx.shape == (h,) and dw.shape == (v, h)
    # the same entry many times is one of their summed weight; a missing one in between changes nothing
    rep = torch.tensor([[7, 7, -1, 7, 7]], device="cuda")
    same = echo.distill(x[:1], w, rep, torch.zeros((1, 5), device="cuda"))
    single = echo.cross_entropy(x[:1], w, torch.tensor([7], device="cuda"))
    assert torch.equal(same[1], single[1])
    assert abs(float(same[2] - single[2])) <= 8 * U * abs(float(single[2]))
    assert abs(float(same[0] - (single[0] - math.log(4)))) <= 64 * U * (abs(float(single[1])) + abs(float(single[2])) + 2)


@pytest.mark.parametrize("dw_type", [F32, BF16])
@pytest.mark.parametrize("left", [0, 4, 1])
def test_sums_into_parts_of_a_matrix(echo, dw_type, left):
    n, h, v = 70, 96, 300
    x, w = _case(n, h, v, 0, BF16, 12)
    labels, dloss = _randint(-1, v, (n,), 13), _randn((n,), 14)
    lse = echo.cross_entropy(x, w, labels)[1]
    whole = _randn((v, h + 8), 15, dw_type)
    old = whole.clone()
    view = whole[:, left:left + h]
    tight = view.clone()
    echo.cross_entropy_grad(dloss, x, w, labels, lse, dweight=tight, accumulate=True)
    got = echo.cross_entropy_grad(dloss, x, w, labels, lse, dweight=view, accumulate=True)
    assert got[1] is view
    assert torch.equal(view, tight) and torch.equal(whole[:, :left], old[:, :left]) and torch.equal(whole[:, left + h:], old[:, left + h:])


def test_only_one_of_the_gradients(echo):
    """dx or dweight alone (NULL for the other, through the C call) are those of both."""
    import ctypes as C

    from paper_2412_12487_gb300 import echo as E
    n, h, v = 100, 64, 700
    for dtype, kind in ((BF16, 1), (F16, 2), (F32, 0)):
        x, w = _case(n, h, v, 0, dtype, 16)
        labels, dloss = _randint(-1, v, (n,), 17), _randn((n,), 18)
        lse = echo.cross_entropy(x, w, labels)[1]
        dx, dw = echo.cross_entropy_grad(dloss, x, w, labels, lse)
        for which in (0, 1):
            a, b = torch.zeros_like(dx), torch.zeros_like(dw)
            d = E.CrossEntropyGradDesc(n, h, v, 0, dloss.data_ptr(), None, x.data_ptr(), w.data_ptr(), labels.data_ptr(), lse.data_ptr(),
                                       a.data_ptr() if which == 0 else None, b.data_ptr() if which else None, h, h, h, h, kind, 0, 64, 0, 1.0)
            assert echo.lib.echo_cross_entropy_grad(echo.h, C.byref(d)) == 0
            torch.cuda.synchronize()
            if which:
                assert torch.equal(b, dw) and not a.any()
            else:
                assert not b.any()
                if dtype == F32:
                    assert torch.equal(a, dx)
                else:  # (P is one number then, as in both; tiles are shared out otherwise, and sums of parts rounded otherwise)
                    assert float((a.double() - dx.double()).abs().max()) <= 2.0 ** -7 * float(dx.double().abs().max())


def test_matrices_beyond_32_bits_of_elements(echo):
    n, h, v = 3, 16384, 135000
    g = torch.Generator(device="cuda").manual_seed(19)
    w = torch.randn((v, h), generator=g, device="cuda", dtype=BF16)
    x = _randn((n, h), 20, BF16, 0.01)
    labels = torch.tensor([v - 1, 131072, 5], device="cuda")
    loss, lse, target = echo.cross_entropy(x, w, labels)
    z = torch.cat([x.double() @ w[i:i + 15000].double().T for i in range(0, v, 15000)], 1)
    size = torch.cat([x.double().abs() @ w[i:i + 15000].double().abs().T for i in range(0, v, 15000)], 1)
    tol = (64 + h / 256) * U * size + 4 * U * z.abs()
    _close(lse, torch.logsumexp(z, 1), tol.amax(1) + 300 * U + 200 * U)
    _close(target, z.gather(1, labels[:, None])[:, 0], tol.gather(1, labels[:, None])[:, 0])
    one = torch.ones(n, device="cuda")
    dx, dw = echo.cross_entropy_grad(one, x, w, labels, lse)
    p = torch.exp(z - lse.double()[:, None])
    p[torch.arange(n), labels] -= 1
    rows = torch.tensor([0, 5, 131071, 131072, v - 2, v - 1], device="cuda")
    want = p[:, rows].T @ x.double()
    near = p[:, rows].abs().T @ x.double().abs()
    _close(dw[rows], want, near * (float(torch.expm1(tol.max() + 600 * U)) + 2.0 ** -19))
    dx_want = sum(p[:, i:i + 15000] @ w[i:i + 15000].double() for i in range(0, v, 15000))
    dx_size = sum(p[:, i:i + 15000].abs() @ w[i:i + 15000].double().abs() for i in range(0, v, 15000))
    _close(dx, dx_want, dx_size * (float(torch.expm1(tol.max() + 600 * U)) + 2.0 ** -8 + 2.0 ** -16))


def test_two_contexts_at_a_time():
    """Calls of two contexts on two streams, without waiting for one another."""
    x, w = _case(500, 256, 3000, 0, BF16, 21)
    labels, dloss = _randint(-1, 3000, (500,), 22), _randn((500,), 23)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    contexts = [Echo(0, stream=s) for s in streams]
    results = [[], []]
    for _ in range(4):
        for i, (e, s) in enumerate(zip(contexts, streams)):
            with torch.cuda.stream(s):
                out = e.cross_entropy(x, w, labels)
                results[i].append((*out, *e.cross_entropy_grad(dloss, x, w, labels, out[1])))
    torch.cuda.synchronize()
    first = results[0][0]
    for r in results[0] + results[1]:
        assert all(torch.equal(a, b) for a, b in zip(r, first))
    for e in contexts:
        e.wait()
        e.close()


def test_teacher_without_weight(echo):
    """Rows whose entries are all missing, have no weight, or an infinite one."""
    x, w = _case(4, 32, 60, 0, BF16, 24)
    ids = torch.tensor([[1, 2], [-1, -1], [3, 4], [5, 6]], device="cuda")
    t = torch.tensor([[0.0, -math.inf], [0.0, 0.0], [-math.inf, -math.inf], [math.nan, 0.0]], device="cuda")
    loss, lse, cross = echo.distill(x, w, ids, t)
    label = echo.cross_entropy(x, w, torch.tensor([1, -1, -1, 5], device="cuda"))
    assert abs(float(loss[0] - label[0][0])) <= 16 * U * float(lse[0].abs() + cross[0].abs()) and torch.equal(lse, label[1])
    assert loss[1] == 0 and loss[2] == 0 and cross[1] == 0 and cross[2] == 0 and torch.isnan(loss[3])
    g = torch.tensor([1.0, math.nan, math.inf, 0.0], device="cuda")
    t[3] = 0
    dx, dw = echo.distill_grad(g, x, w, ids, t, lse)
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all() and not dx[1:].any()


@pytest.mark.parametrize("n", [2, 7, 8, 9, 16, 17])
@pytest.mark.parametrize("h,left", [(516, 0), (517, 0), (1030, 3), (2052, 4)])
def test_few_tokens_in_full_precision(echo, n, h, left):
    """Up to 16 fp32 tokens take kernels of their own; one more does not.  Sums of up to 20 terms a lane and a tree: within
    the bounds of the others."""
    v, v0 = 333 if n != 7 else 40000, 11  # (many rows: more of them a block)
    x = _randn((n, h), 30)
    w = _randn((v, h + 8), 31, F32, 2.0 / math.sqrt(h))[:, left:left + h]
    labels, dloss = _randint(-1, v0 + v + 20, (n,), 32), _randn((n,), 33)
    lse = _check_ce(echo, x, w, labels, v0, 0.75)
    ids, logits = _teacher(n, 12, v, v0, F32, 34)
    ids[0, :3] = v0 + 5
    q, _, eq = _teacher_ref(ids, logits, 2.0)
    loss, lse2, cross = echo.distill(x, w, ids, logits, temperature=2.0, vocab_start=v0)
    ref = Ref(x, w, 1.0, 2.0)
    mine = (ids >= v0) & (ids < v0 + v)
    row = torch.where(mine, ids - v0, 0)
    zk, ek = torch.where(mine, ref.z.gather(1, row), 0.0), torch.where(mine, ref.ez.gather(1, row), 0.0)
    _close(lse2, ref.lse, ref.elast)
    _close(cross, (q * zk).sum(1), (q * ek + eq * zk.abs()).sum(1) + 20 * U * (q * zk).abs().sum(1))
    for dw_type in (F32, BF16):
        up = dloss.double()[:, None] * 2.0
        a, b, ta, tb = ref.grads((up * q).sum(1), (up * q).abs().sum(1), ref.targets(ids, up * q, v0), lse2.double(), 1.0, dw_type)
        eP = ref.targets(ids, (up * eq).abs(), v0) + ((up * eq).abs().sum(1) + 16 * U * (up * q).abs().sum(1))[:, None] * torch.exp(ref.z - lse2.double()[:, None])
        old = _randn((v, h + 8), 35, dw_type)
        out = old.clone()
        dx, dw = echo.distill_grad(dloss, x, w, ids, logits, lse2, temperature=2.0, vocab_start=v0, dweight=out[:, left:left + h], accumulate=True)
        _close(dx, a, ta + eP @ ref.W.abs())
        total = b + old[:, left:left + h].double()
        _close(dw, total, tb + eP.T @ ref.X.abs() + 2 * U * total.abs())
        assert torch.equal(out[:, :left], old[:, :left]) and torch.equal(out[:, left + h:], old[:, left + h:])
    y, m = x.clone(), labels.clone()
    m[0] = -1
    clean = echo.cross_entropy_grad(dloss, y, w, m, lse, scale=0.75, vocab_start=v0)
    y[0] = math.nan
    got = echo.cross_entropy_grad(dloss, y, w, m, lse, scale=0.75, vocab_start=v0)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1]) and not got[0][0].any()


@pytest.mark.parametrize("h", [1024, 1032, 1033, 4096, 4104, 12296])
def test_long_rows_of_full_precision(echo, h):
    """Rows that a warp, a block's registers, and neither can hold; more of them than blocks; each of its own size, which its
    last column may set alone."""
    n, v = 20, 2500
    x, w = _randn((n, h), 40), _randn((v, h), 41, F32, 1.0 / math.sqrt(h))
    x *= torch.pow(2.0, (torch.arange(n, device="cuda") % 5 - 2).float())[:, None]
    w *= torch.pow(2.0, -(torch.arange(v, device="cuda") % 13).float())[:, None]
    w[::3, -1] *= 64.0
    x[1::4, -1] *= 64.0
    labels = _randint(0, v, (n,), 42)
    labels[4] = v - 1
    first = echo.cross_entropy(x, w, labels)
    _check_ce(echo, x, w, labels, 0, 1.0, first)
    assert all(torch.equal(a, b) for a, b in zip(first, echo.cross_entropy(x, w, labels)))


@pytest.mark.parametrize("dtype,dw_type", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("n,h,v", [(17, 512, 9000), (200, 1024, 5000)])
def test_gradients_of_few_tokens_and_many_tiles(echo, dtype, dw_type, n, h, v):
    """Tiles of dW of a few stages, taken early by the pairs that have less of dx."""
    x, w = _case(n, h, v, 0, dtype, 43)
    labels, dloss = _randint(-1, v, (n,), 44), _randn((n,), 45, F32, 0.1)
    ref = Ref(x, w, 1.0)
    lse = echo.cross_entropy(x, w, labels)[1]
    up = torch.where(labels >= 0, dloss.double(), 0.0)
    a, b, ta, tb = ref.grads(up, up.abs(), ref.targets(labels[:, None], up[:, None], 0), lse.double(), 1.0, dw_type)
    old = _randn((v, h), 46, dw_type)
    for accumulate in (False, True):
        out = old.clone()
        dx, dw = echo.cross_entropy_grad(dloss, x, w, labels, lse, dweight=out, accumulate=accumulate)
        _close(dx, a, ta)
        total = b + old.double() if accumulate else b
        _close(dw, total, tb + 2 * U * total.abs())
