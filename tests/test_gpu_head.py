"""Losses of a head (cross entropy, distillation) and their gradients against plain 64-bit implementations.

Tolerances are bounds on rounding, written down before the first run.  U = 2^-24 is fp32's unit roundoff, uo the 16-bit
types'.

* logits: products of 16-bit numbers are exact; the tensor core adds up a set of stages with truncation (four additions of 16
  products a stage, each off by less than 2 U of the sum so far), then the sets' sums are rounded, fewer than H / 256 of
  them.  A set has up to 32 stages, 128 additions to sums that grow from nothing: 128 U of the magnitudes if all products had
  one sign; here signs are mixed and sums stay below half of that: (64 + H / 256) U of the sum of the products' magnitudes.  fp32 elements are sums of two fp16 numbers: 2^-22 of each, the product of the two low parts is left
  out (2^-22), or 2^-37 of the matrix's largest element where that is more.
* lse: the largest error of a logit, and sums of at most 128 exponentials (each within 2^-21) by four and a tree: 300 U, and
  U of its size a few times.
* an element of dz: the exponential of a logit's and lse's errors, 2^-20 for the exponential and the products; then its
  rounding: uo for one 16-bit number, 2^-21 for two, in fp16 (scaled by the largest token's size, of which a sum of K + 1
  weights is the bound) at least 2^-40 of that size.
* dx and dweight: those errors times the magnitudes of the other operand, and sums in fp32 as for logits.
"""
import math

import numpy as np
import pytest

from paper_2412_12487_gb300 import Echo, EchoError

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


def _randn(shape, seed, dtype=F32, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _randint(lo, hi, shape, seed, dtype=torch.int64):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(lo, hi, shape, generator=g, device="cuda").to(dtype)


def _close(got, want, tol):
    """|got - want| <= tol + one rounding of the output, element by element; NaN and infinities alike."""
    dtype = got.dtype
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    off = (got - want).abs() - (tol + UO[dtype] * (want.abs() + tol) + TINY[dtype])
    assert not fine.any() or float(torch.where(fine, off, torch.full_like(off, -1.0)).max()) <= 0, float(off[fine].max())


class Ref:
    """The definitions in 64 bits, with the errors that the kernels may have."""

    def __init__(self, x, w, scale=1.0, tau=1.0):
        self.x, self.w, self.alpha, self.tau = x, w, scale / tau, tau
        X, W = x.double().reshape(-1, x.shape[-1]), w.double()
        self.X, self.W, h = X, W, x.shape[-1]
        size = X.abs() @ W.abs().T
        self.units = (64 + h / 256) * U
        if x.dtype == F32:
            self.units += 3 * 2.0 ** -22
            size_far = 2.0 ** -37 * (X.abs().max() * W.abs().sum(1)[None] + W.abs().max() * X.abs().sum(1)[:, None]) if X.numel() and W.numel() else 0.0
        else:
            size_far = 0.0
        self.z = X @ W.T * self.alpha
        self.ez = (self.units * size + size_far) * abs(self.alpha) + 4 * U * self.z.abs()
        self.lse = torch.logsumexp(self.z, 1) if W.shape[0] else torch.full((X.shape[0],), -math.inf, device="cuda", dtype=torch.float64)
        self.elast = (self.ez.amax(1) if W.shape[0] else 0.0) + 300 * U + 8 * U * self.lse.abs()

    def targets(self, ids, q, v0):
        """The wanted probabilities of the shard's rows, from ids and weights [tokens, K]."""
        want = torch.zeros_like(self.z)
        at, k = torch.nonzero((ids >= v0) & (ids < v0 + self.W.shape[0]), as_tuple=True)
        return want.index_put_((at, ids[at, k].long() - v0), q[at, k], accumulate=True)

    def grads(self, coef, weight_sum, want, lse, alpha_tau, dw_type):
        """dx, dweight and their errors: P = coef p - want times the weights already in them."""
        e = self.ez + (300 + 8 * lse.abs()[:, None]) * U
        soft = torch.where(coef[:, None] == 0, 0.0, coef[:, None] * torch.exp(self.z - lse[:, None]))
        P = soft - want
        eP = soft.abs() * (torch.expm1(e) + 2.0 ** -20) + 4 * U * want.abs()
        largest = (coef.abs() + weight_sum).max() if coef.numel() else 0.0
        half = 2.0 ** -40 * largest
        two = 2.0 ** -21
        bf = self.x.dtype == BF16
        r_dx = two if self.x.dtype == F32 else UO[self.x.dtype]
        r_dw = two if F32 in (self.x.dtype, dw_type) else UO[self.x.dtype]
        abs_x = 0.0 if bf else half
        abs_w = 0.0 if bf and dw_type != F32 else half
        ex, ew = eP * 1.01 + r_dx * P.abs() + abs_x, eP * 1.01 + r_dw * P.abs() + abs_w
        units = lambda n: (64 + n / 256) * U + (3 * 2.0 ** -22 if self.x.dtype == F32 else 0.0)  # noqa: E731
        live = ((coef != 0) | (weight_sum != 0))[:, None]
        X = torch.where(live, self.X, 0.0)
        tx = ex @ self.W.abs() + units(P.shape[1]) * (P.abs() @ self.W.abs())
        tw = ew.T @ X.abs() + units(P.shape[0]) * (P.abs().T @ X.abs())
        if self.x.dtype == F32 and P.numel():
            tx = tx + 2.0 ** -37 * self.W.abs().max() * P.abs().sum(1)[:, None]
            tw = tw + 2.0 ** -37 * X.abs().max() * P.abs().sum(0)[:, None]
        elif self.x.dtype == BF16 and dw_type == F32 and P.numel():
            tw = tw + 2.0 ** -40 * X.abs().max() * P.abs().sum(0)[:, None]  # (x as fp16)
        return P @ self.W, P.T @ X, tx, tw


SIZES = [(1, 1, 1, 0), (1, 8, 300, 0), (3, 64, 257, 5), (257, 72, 129, 100), (130, 517, 1003, 0), (64, 2056, 700, 50), (600, 256, 2000, 7), (255, 1, 40, 3)]


def _case(n, h, v, v0, dtype, seed=1):
    x, w = _randn((n, h), seed, dtype), _randn((v, h), seed + 1, dtype, 2.0 / math.sqrt(h))
    return x, w


def _check_ce(echo, x, w, labels, v0, scale, got=None):
    ref = Ref(x, w, float(np.float32(scale)))
    loss, lse, target = got or echo.cross_entropy(x, w, labels, scale=scale, vocab_start=v0)
    lab = labels.reshape(-1).long()
    mine = (lab >= v0) & (lab < v0 + w.shape[0]) & (lab >= 0)
    row = torch.where(mine, lab - v0, 0)
    at = ref.z.gather(1, row[:, None])[:, 0] if w.shape[0] else torch.zeros_like(ref.lse)
    want = torch.where(mine, at, 0.0)
    et = torch.where(mine, ref.ez.gather(1, row[:, None])[:, 0], 0.0) if w.shape[0] else 0.0
    _close(lse.reshape(-1), ref.lse, ref.elast)
    _close(target.reshape(-1), want, et)
    _close(loss.reshape(-1), torch.where(lab >= 0, ref.lse - want, 0.0), torch.where(lab >= 0, ref.elast + et, 0.0))
    assert loss.shape == lse.shape == target.shape == labels.shape and loss.dtype == F32
    return lse


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n,h,v,v0", SIZES)
def test_cross_entropy(echo, dtype, n, h, v, v0):
    x, w = _case(n, h, v, v0, dtype)
    for bits, scale in ((torch.int64, 1.0), (torch.int32, -0.75)):
        labels = _randint(-2, v0 + v + 3, (n,), 3, bits)
        _check_ce(echo, x, w, labels, v0, scale)
        again = echo.cross_entropy(x, w, labels, scale=scale, vocab_start=v0)
        assert all(torch.equal(a, b) for a, b in zip(again, echo.cross_entropy(x, w, labels, scale=scale, vocab_start=v0)))


@pytest.mark.parametrize("dtype,dw_type", [(BF16, F32), (BF16, BF16), (BF16, F16), (F16, F32), (F16, F16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("n,h,v,v0", SIZES)
def test_cross_entropy_grad(echo, dtype, dw_type, n, h, v, v0):
    x, w = _case(n, h, v, v0, dtype, 4)
    labels = _randint(-2, v0 + v + 3, (n,), 5)
    dloss = _randn((n,), 6, F32, 0.01)
    scale = 1.25
    ref = Ref(x, w, scale)
    lse = (ref.lse + 0.5).float()  # as if other shards had something
    got = echo.cross_entropy_grad(dloss, x, w, labels, lse, scale=scale, vocab_start=v0, dtype=dw_type)
    valid = labels >= 0
    coef = torch.where(valid, dloss.double() * scale, 0.0)
    want = ref.targets(torch.where(valid, labels, -1)[:, None], coef[:, None], v0)
    dx, dw, tx, tw = ref.grads(coef, coef.abs(), want, lse.double(), 1.0, dw_type)
    assert got[0].dtype == dtype and got[1].dtype == dw_type
    _close(got[0], dx, tx)
    _close(got[1], dw, tw)
    old = _randn((v, h), 7, dw_type, 0.01)
    total = old.clone()
    got2 = echo.cross_entropy_grad(dloss, x, w, labels, lse, scale=scale, vocab_start=v0, dweight=total, accumulate=True)
    assert got2[1] is total and torch.equal(got2[0], got[0])
    _close(total, dw + old.double(), tw + 2 * U * (dw + old.double()).abs())
    again = echo.cross_entropy_grad(dloss, x, w, labels, lse, scale=scale, vocab_start=v0, dtype=dw_type)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def _teacher(n, k, v, v0, dtype, seed):
    """Ids with repeats, some of other shards and missing, and logits."""
    ids = _randint(-3, v0 + v + 5, (n, k), seed)
    logits = _randn((n, k), seed + 1, dtype, 3.0)
    return ids, logits


def _teacher_ref(ids, logits, tau, teacher_lse=None):
    t = (logits.double() / float(np.float32(tau))).masked_fill(ids < 0, -math.inf)
    l = torch.logsumexp(t, 1) if teacher_lse is None else teacher_lse.double()
    log_q = torch.where(t == -math.inf, 0.0, t - torch.where(l == -math.inf, 0.0, l)[:, None])
    q = torch.where(t == -math.inf, 0.0, torch.exp(log_q))
    # q's relative error: the subtraction's rounding, and sums of 256 exponentials
    eq = (64 + 8 * t.masked_fill(t == -math.inf, 0).abs().amax(1, keepdim=True) + (0 if teacher_lse is None else 8 * l.abs()[:, None])) * U
    return q, log_q, q * eq


@pytest.mark.parametrize("dtype,k", [(BF16, 1), (BF16, 33), (F16, 7), (F32, 64), (BF16, 256)])
@pytest.mark.parametrize("n,h,v,v0", SIZES)
def test_distill(echo, dtype, k, n, h, v, v0):
    x, w = _case(n, h, v, v0, dtype, 8)
    for tau, own in ((1.0, False), (2.5, True)):
        ids, logits = _teacher(n, k, v, v0, dtype, 9)
        if n > 2:
            ids[1] = -1  # nothing from the teacher
            logits[2, : k // 2] = -math.inf
        lt = None
        if own:
            lt = (torch.logsumexp((logits.double() / tau).masked_fill(ids < 0, -math.inf), 1).clamp_min(-50) + 0.3).float()
        ref = Ref(x, w, 1.0, float(np.float32(tau)))
        q, log_q, eq = _teacher_ref(ids, logits, tau, lt)
        loss, lse, cross = echo.distill(x, w, ids, logits, temperature=tau, teacher_lse=lt, vocab_start=v0)
        mine = (ids >= v0) & (ids < v0 + v) & (ids >= 0)
        row = torch.where(mine, ids - v0, 0)
        zk, ek = torch.where(mine, ref.z.gather(1, row), 0.0), torch.where(mine, ref.ez.gather(1, row), 0.0)
        want, ec = (q * zk).sum(1), (q * ek + eq * zk.abs()).sum(1) + (k + 8) * U * (q * zk).abs().sum(1)
        _close(lse, ref.lse, ref.elast)
        _close(cross, want, ec)
        mass, em = q.sum(1), eq.sum(1) + 16 * U * q.sum(1)
        entropy = (q * log_q).sum(1)
        ee = (eq * (log_q.abs() + 1)).sum(1) + 16 * U * (q * log_q).abs().sum(1) + (k + 8) * U
        total = tau * tau * (entropy + mass * ref.lse - want)
        tol = tau * tau * (ee + mass * ref.elast + em * ref.lse.abs() + ec + 4 * U * (entropy.abs() + (mass * ref.lse).abs() + want.abs()))
        empty = (mass == 0)
        _close(loss, torch.where(empty, 0.0, total), torch.where(empty, 0.0, tol))


@pytest.mark.parametrize("dtype,dw_type,k", [(BF16, F32, 5), (BF16, BF16, 40), (F16, F16, 7), (F16, F32, 64), (F32, F32, 9)])
@pytest.mark.parametrize("n,h,v,v0", SIZES)
def test_distill_grad(echo, dtype, dw_type, k, n, h, v, v0):
    tau, scale = 1.5, 0.5
    x, w = _case(n, h, v, v0, dtype, 11)
    ids, logits = _teacher(n, k, v, v0, dtype, 12)
    if n > 2:
        ids[1] = -1
    dloss, dlse = _randn((n,), 13, F32, 0.01), _randn((n,), 14, F32, 0.003)
    for extra in (None, dlse):
        ref = Ref(x, w, scale, tau)
        lse = (ref.lse + 0.25).float()
        got = echo.distill_grad(dloss, x, w, ids, logits, lse, temperature=tau, scale=scale, vocab_start=v0, dlse=extra, dtype=dw_type)
        q, _, eq = _teacher_ref(ids, logits, tau)
        up = dloss.double()[:, None] * tau * scale
        coef = (up * q).sum(1) + (0 if extra is None else extra.double() * scale / tau)
        want = ref.targets(ids, up * q, v0)
        ew = ref.targets(ids, (up * eq).abs(), v0)
        dx, dw, tx, tw = ref.grads(coef, (up * q).abs().sum(1), want, lse.double(), 1.0, dw_type)
        # the weights' and the coefficient's own errors
        ecoef = (up * eq).abs().sum(1) + 16 * U * ((up * q).abs().sum(1) + coef.abs())
        eP = ew + torch.where(coef[:, None] == 0, 0.0, ecoef[:, None] * torch.exp(ref.z - lse.double()[:, None])) * 1.01
        _close(got[0], dx, tx + eP @ ref.W.abs())
        _close(got[1], dw, tw + eP.T @ ref.X.abs())


def test_pieces_of_the_vocabulary(monkeypatch):
    """A piece of 256 rows at a time gives what one piece gives, but for the order of dx's sums."""
    n, h, v = 300, 200, 1300
    monkeypatch.setenv("ECHO_TEST_HEAD_PIECE", "1")
    with Echo(0) as small:
        for dtype, dw_type in ((BF16, F32), (BF16, BF16), (F16, F32), (F32, F32)):
            x, w = _case(n, h, v, 0, dtype, 15)
            labels, dloss = _randint(-1, v + 200, (n,), 16), _randn((n,), 17)
            ref = Ref(x, w)
            lse = ref.lse.float()
            coef = torch.where(labels >= 0, dloss.double(), 0.0)
            want = ref.targets(labels[:, None], coef[:, None], 0)
            dx, dw, tx, tw = ref.grads(coef, coef.abs(), want, lse.double(), 1.0, dw_type)
            got = small.cross_entropy_grad(dloss, x, w, labels, lse, dtype=dw_type)
            _close(got[0], dx, tx + 8 * U * (want.abs() @ ref.W.abs()))
            _close(got[1], dw, tw)
            only = small.cross_entropy_grad(dloss, x, w, labels, lse, dtype=dw_type)
            assert torch.equal(only[0], got[0]) and torch.equal(only[1], got[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masked_tokens_reach_nothing(echo, dtype):
    n, h, v = 40, 96, 300
    x, w = _case(n, h, v, 0, dtype, 18)
    labels = _randint(0, v, (n,), 19)
    labels[::3] = -100
    dloss = _randn((n,), 20)
    lse = echo.cross_entropy(x, w, labels)[1]
    clean = echo.cross_entropy_grad(dloss, x, w, labels, lse)
    for bad in (math.nan, math.inf):
        y, g = x.clone(), dloss.clone()
        y[::3] = bad  # padding holds anything
        g[::3] = bad
        l2 = lse.clone()
        l2[::3] = bad
        got = echo.cross_entropy_grad(g, y, w, labels, l2)
        assert (got[0][::3] == 0).all() and torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
        if dtype == BF16:
            loss = echo.cross_entropy(y, w, labels)[0]
            assert (loss[::3] == 0).all() and torch.isfinite(loss).all()
    all_masked = torch.full_like(labels, -1)
    dx, dw = echo.cross_entropy_grad(dloss, x, w, all_masked, lse)
    assert not dx.any() and not dw.any()
    loss = echo.cross_entropy(x, w, all_masked)[0]
    assert not loss.any()


def test_empty_calls(echo):
    x, w = _case(5, 32, 20, 0, BF16, 21)
    labels = _randint(0, 20, (5,), 22)
    none, dn = labels[:0], torch.empty(0, device="cuda")
    assert [t.shape for t in echo.cross_entropy(x[:0], w, none)] == [(0,)] * 3
    dx, dw = echo.cross_entropy_grad(dn, x[:0], w, none, dn)
    assert dx.shape == (0, 32) and not dw.any() and dw.shape == (20, 32)
    keep = torch.full((20, 40), 3.0, device="cuda")
    echo.cross_entropy_grad(dn, x[:0], w, none, dn, dweight=keep[:, 1:33], accumulate=True)
    assert (keep == 3).all()
    echo.cross_entropy_grad(dn, x[:0], w, none, dn, dweight=keep[:, 1:33])
    assert (keep[:, 1:33] == 0).all() and (keep[:, 0] == 3).all() and (keep[:, 33:] == 3).all()
    loss, lse, target = echo.cross_entropy(x, w[:0], labels)
    assert (lse == -math.inf).all() and not target.any()
    dx, dw = echo.cross_entropy_grad(torch.ones(5, device="cuda"), x, w[:0], labels, torch.zeros(5, device="cuda"))
    assert not dx.any() and dw.shape == (0, 32)
    ids = labels[:, None].repeat(1, 3)
    t = torch.zeros((5, 3), device="cuda")
    assert [s.shape for s in echo.distill(x[:0], w, ids[:0], t[:0])] == [(0,)] * 3


@pytest.mark.parametrize("h", [64, 65, 72])
def test_strides(echo, h):
    wide_x, wide_w = _randn((50, h + 9), 23, BF16), _randn((90, h + 16), 24, BF16)
    labels, dloss = _randint(0, 90, (50,), 25), _randn((50,), 26)
    for x, w in ((wide_x[:, 3:3 + h], wide_w[:, 8:8 + h]), (wide_x[:, :h], wide_w[:, 1:1 + h]), (wide_x[:1, :h].expand(50, h), wide_w[:, :h])):
        want = echo.cross_entropy(x.contiguous(), w.contiguous(), labels)
        got = echo.cross_entropy(x, w, labels)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        out_x, out_w = torch.full((50, h + 5), 7.0, dtype=BF16, device="cuda"), torch.full((90, h + 3), 7.0, device="cuda")
        grads = echo.cross_entropy_grad(dloss, x.contiguous(), w.contiguous(), labels, want[1])
        echo.cross_entropy_grad(dloss, x, w, labels, want[1], dx=out_x[:, 2:2 + h], dweight=out_w[:, 1:1 + h])
        assert torch.equal(out_x[:, 2:2 + h], grads[0]) and torch.equal(out_w[:, 1:1 + h], grads[1])
        assert (out_x[:, :2] == 7).all() and (out_x[:, 2 + h:] == 7).all() and (out_w[:, :1] == 7).all() and (out_w[:, 1 + h:] == 7).all()
    nd = _randn((2, 5, 5, h), 27, BF16)
    loss = echo.cross_entropy(nd, wide_w[:, :h], labels.view(2, 5, 5))[0]
    assert loss.shape == (2, 5, 5)
    assert torch.equal(loss.view(-1), echo.cross_entropy(nd.view(50, h), wide_w[:, :h], labels)[0])


def test_gradients_are_the_derivatives(echo):
    """Against differences of the loss itself, in fp32: both sides, along a direction of x and of weight.

    A step s moves the mean loss by s g + s^2 c / 2 + ...; the central difference is off by s^2 times a third derivative
    (logits of size 2 times the direction's, at most 8 here) and by the losses' own errors over s."""
    n, h, v = 60, 40, 200
    x, w = _randn((n, h), 28), _randn((v, h), 29, F32, 0.3)
    labels = _randint(-1, v, (n,), 30)
    ids, teacher = _teacher(n, 6, v, 0, F32, 31)
    tau = 2.0
    up = _randn((n,), 32)
    u, d = _randn((n, h), 33, F32, 1 / math.sqrt(h)), _randn((v, h), 34, F32, 0.3 / math.sqrt(h))
    s = 2.0 ** -6
    for loss_of, grad_of in ((lambda a, b: echo.cross_entropy(a, b, labels), lambda l: echo.cross_entropy_grad(up, x, w, labels, l)),
                             (lambda a, b: echo.distill(a, b, ids, teacher, temperature=tau), lambda l: echo.distill_grad(up, x, w, ids, teacher, l, temperature=tau))):
        loss, lse, _ = loss_of(x, w)
        dx, dw = grad_of(lse)
        for grad, hi, lo in ((float((dx.double() * u.double()).sum()), loss_of(x + s * u, w), loss_of(x - s * u, w)),
                             (float((dw.double() * d.double()).sum()), loss_of(x, w + s * d), loss_of(x, w - s * d))):
            slope = float((up.double() * (hi[0].double() - lo[0].double())).sum()) / (2 * s)
            size = float(up.double().abs().sum())
            # logits move by at most 4 s here: third derivatives of lse are at most 64 / 4 a token; losses are within 2000 U
            assert abs(slope - grad) <= size * (16 * s * s + 4 * 2000 * U / s * 4)


def test_weights_of_a_peaked_softmax_and_far_logits(echo):
    """Logits to +-60000 and tokens that are sure of themselves: exponentials that vanish, and none that overflows."""
    n, h, v = 20, 64, 500
    for dtype, size in ((BF16, 30.0), (F32, 30.0)):
        x, w = _randn((n, h), 35, dtype, size), _randn((v, h), 36, dtype, size)
        labels = _randint(0, v, (n,), 37)
        _check_ce(echo, x, w, labels, 0, 1.0)
        loss, lse, _ = echo.cross_entropy(x, w, labels)
        dx, dw = echo.cross_entropy_grad(torch.ones(n, device="cuda"), x, w, labels, lse)
        assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
    huge = torch.full((3, 8), 2.0 ** 60, device="cuda")
    tiny = torch.full((5, 8), 2.0 ** -62, device="cuda")
    lab = torch.tensor([0, 4, 2], device="cuda")
    loss, lse, target = echo.cross_entropy(huge, tiny, lab)
    assert torch.allclose(target, torch.full_like(target, 2.0), rtol=1e-6) and torch.allclose(loss, torch.full_like(loss, math.log(5)), rtol=1e-6)


def test_infinite_and_nan_elements(echo):
    x, w = _case(6, 32, 40, 0, BF16, 38)
    x[2, 3], x[4, 5] = math.nan, math.inf
    labels = _randint(0, 40, (6,), 39)
    loss, lse, _ = echo.cross_entropy(x, w, labels)
    keep = [0, 1, 3, 5]
    assert torch.isnan(lse[2]) and not torch.isfinite(loss[4])
    want = echo.cross_entropy(x[keep], w, labels[keep])
    assert torch.equal(loss[keep], want[0]) and torch.equal(lse[keep], want[1])


def test_labels_at_the_ends(echo):
    x, w = _case(6, 32, 40, 0, F16, 40)
    far = torch.tensor([0, 39, 40, 2 ** 62, -2 ** 63, 2 ** 63 - 1], device="cuda")
    _check_ce(echo, x, w, far, 0, 1.0)
    start = 2 ** 40
    near = torch.tensor([start, start + 39, start + 40, start - 1, -1, 0], device="cuda")
    got = echo.cross_entropy(x, w, near, vocab_start=start)
    assert got[2][2:].eq(0).all() and got[0][4] == 0
    ref = echo.cross_entropy(x, w, torch.tensor([0, 39, 40, 41, -1, 41], device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_shards_make_the_whole(echo):
    n, h, v, parts = 70, 128, 1200, 4
    x, w = _case(n, h, v, 0, BF16, 41)
    labels, dloss = _randint(-1, v, (n,), 42), _randn((n,), 43)
    loss, lse, _ = echo.cross_entropy(x, w, labels)
    got = [echo.cross_entropy(x, w[p * 300:p * 300 + 300], labels, vocab_start=p * 300) for p in range(parts)]
    total = torch.logsumexp(torch.stack([g[1] for g in got]).double(), 0)
    whole = torch.where(labels >= 0, total - torch.stack([g[2] for g in got]).double().sum(0), 0.0)
    ref = Ref(x, w)
    _close(loss, whole, 2 * ref.elast)
    dx, dw = echo.cross_entropy_grad(dloss, x, w, labels, lse)
    for p in range(parts):
        s = echo.cross_entropy_grad(dloss, x, w[p * 300:p * 300 + 300], labels, lse, vocab_start=p * 300)
        assert torch.equal(s[1], dw[p * 300:p * 300 + 300])


def test_other_streams_graphs_and_contexts(echo):
    n, h, v = 200, 96, 700
    x, w = _case(n, h, v, 0, BF16, 44)
    labels, dloss = _randint(-1, v, (n,), 45), _randn((n,), 46)
    want = echo.cross_entropy(x, w, labels)
    grads = echo.cross_entropy_grad(dloss, x, w, labels, want[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = echo.cross_entropy(x, w, labels)
        g = echo.cross_entropy_grad(dloss, x, w, labels, got[1])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got, *g), (*want, *grads)))
    with torch.cuda.stream(side), Echo(0, stream=side) as own:
        dw = torch.zeros((v, h), device="cuda")
        own.cross_entropy(x, w, labels)
        own.cross_entropy_grad(dloss, x, w, labels, want[1], dweight=dw, accumulate=True)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = own.cross_entropy(x, w, labels)
            gx, _ = own.cross_entropy_grad(dloss, x, w, labels, out[1], dweight=dw, accumulate=True)
        big = _randn((3 * n, h), 47, BF16)
        own.cross_entropy_grad(dloss.repeat(3), big, w, labels.repeat(3), want[1].repeat(3))  # outgrows the scratch that the graph has
        dw.zero_()
        graph.replay()
        graph.replay()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(gx, grads[0])
        _close(dw, 2 * grads[1].double(), 4 * U * grads[1].double().abs())
        own.wait()


def test_refusals(echo):
    x, w = _case(4, 16, 10, 0, BF16, 48)
    labels, g = _randint(0, 10, (4,), 49), torch.ones(4, device="cuda")
    ids, t = labels[:, None].repeat(1, 2), torch.zeros((4, 2), device="cuda")
    for call in (lambda: echo.cross_entropy(x, w.float(), labels),
                 lambda: echo.cross_entropy(x, w[:, :8], labels),
                 lambda: echo.cross_entropy(x, w, labels[:3]),
                 lambda: echo.cross_entropy(x, w, labels.float()),
                 lambda: echo.cross_entropy(x.double(), w.double(), labels),
                 lambda: echo.cross_entropy(x, w, labels, vocab_start=-1),
                 lambda: echo.cross_entropy(x, w, labels, scale=math.inf),
                 lambda: echo.cross_entropy(x.cpu(), w, labels),
                 lambda: echo.cross_entropy_grad(g, x, w, labels, None),
                 lambda: echo.cross_entropy_grad(g.double(), x, w, labels, g),
                 lambda: echo.cross_entropy_grad(g, x, w, labels, g, accumulate=True),
                 lambda: echo.cross_entropy_grad(g, x, w, labels, g, dweight=torch.zeros((10, 8), device="cuda")),
                 lambda: echo.cross_entropy_grad(g, x, w, labels, g, dx=torch.zeros((4, 16), device="cuda")),
                 lambda: echo.cross_entropy_grad(g, x, w, labels, g, dweight=torch.zeros((16, 10), device="cuda").t()),
                 lambda: echo.distill(x, w, ids, t[:, :1]),
                 lambda: echo.distill(x, w, ids, t, temperature=0.0),
                 lambda: echo.distill(x, w, ids, t, temperature=math.nan),
                 lambda: echo.distill(x, w, ids[:, :0], t[:, :0]),
                 lambda: echo.distill(x, w, ids, t, teacher_lse=g[:3])):
        with pytest.raises(EchoError) as err:
            call()
        assert err.value.code == 1, err.value
    with pytest.raises(EchoError) as err:
        echo.distill(x, w, ids.repeat(1, 200), t.repeat(1, 200))
    assert err.value.code == 9
    side = torch.cuda.Stream()
    with torch.cuda.stream(side), Echo(0, stream=side) as own:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            with pytest.raises(EchoError) as err:  # would have to allocate
                own.cross_entropy(x, w, labels)
        assert err.value.code == 4
    assert echo.cross_entropy(x, w, labels)[0].isfinite().all()


def test_a_wait_that_runs_out_is_reported(monkeypatch):
    x, w = _case(300, 256, 600, 0, BF16, 50)
    labels = _randint(0, 600, (300,), 51)
    monkeypatch.setenv("ECHO_TEST_SKIP_LEVEL", "1")
    monkeypatch.setenv("ECHO_TEST_WAIT_LIMIT_MS", "20")
    with Echo(0) as e:
        e.cross_entropy(x, w, labels)
        with pytest.raises(EchoError) as err:
            e.wait()
        assert err.value.code == 7
        e.wait()


def test_many_tiles(echo):
    """More tiles than pairs of blocks, in both directions of the grid's order, and a long sum."""
    n, h, v = 2100, 320, 9000
    x, w = _case(n, h, v, 0, BF16, 52)
    labels, dloss = _randint(-1, v, (n,), 53), _randn((n,), 54, F32, 1e-3)
    lse = _check_ce(echo, x, w, labels, 0, 1.0)
    ref = Ref(x, w)
    coef = torch.where(labels >= 0, dloss.double(), 0.0)
    want = ref.targets(labels[:, None], coef[:, None], 0)
    dx, dw, tx, tw = ref.grads(coef, coef.abs(), want, lse.double(), 1.0, F32)
    got = echo.cross_entropy_grad(dloss, x, w, labels, lse)
    _close(got[0], dx, tx)
    _close(got[1], dw, tw)
