"""Distillation over shards of the vocabulary: the whole loss from the shards' results, and the gradients."""
import math

import pytest

from paper_2412_12487_gb300 import Echo

from .test_gpu_head import BF16, F16, F32, U, Ref, _case, _close, _randn, _teacher, _teacher_ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def echo():
    with Echo(0) as e:
        yield e


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n", [9, 70])
def test_shards_make_the_whole(echo, dtype, own, n):
    """loss + T^2 (Q (l - lse) + cross - c) of any shard, with l of all rows and c the sum of all shards' cross; each of the
    shards' results within test_gpu_head.py's bounds."""
    h, v, k, tau, rows = 128, 1200, 9, 2.0, 300
    x, w = _case(n, h, v, 0, dtype, 1)
    ids, logits = _teacher(n, k, v, 0, F32, 2)
    ids[1] = -1                      # nothing from the teacher
    ids[2] = torch.arange(k) + rows  # all of another shard than the first
    lt = (torch.logsumexp((logits.double() / tau).masked_fill(ids < 0, -math.inf), 1).clamp_min(-50) + 0.3).float() if own else None
    q, log_q, eq = _teacher_ref(ids, logits, tau, lt)
    mass = q.sum(1)
    got = [echo.distill(x, w[p:p + rows], ids, logits, temperature=tau, teacher_lse=lt, vocab_start=p) for p in range(0, v, rows)]
    l = torch.logsumexp(torch.stack([g[1] for g in got]).double(), 0)
    c = torch.stack([g[2] for g in got]).double().sum(0)

    ref = Ref(x, w, 1.0, tau)
    mine = ids >= 0
    row = torch.where(mine & (ids < v), ids, 0)
    mine &= ids < v
    zk, ek = torch.where(mine, ref.z.gather(1, row), 0.0), torch.where(mine, ref.ez.gather(1, row), 0.0)
    cross, entropy = (q * zk).sum(1), (q * log_q).sum(1)
    want = torch.where(mass == 0, 0.0, tau * tau * (entropy + mass * ref.lse - cross))
    size = (q * zk).abs().sum(1)
    ec = (q * ek + eq * zk.abs()).sum(1) + (k + 8) * U * size
    ee = (eq * (log_q.abs() + 1)).sum(1) + 16 * U * (q * log_q).abs().sum(1) + (k + 8) * U
    em = eq.sum(1) + 16 * U * mass
    elast = ref.elast + 8 * U * 20  # (a shard's lse is within 20 of zero, as the whole one is)
    tol = tau * tau * (ee + 3 * mass * elast + 20 * em + 3 * ec + 4 * U * (entropy.abs() + 20 * mass + size))
    for loss, lse, part in got:
        whole = torch.where(mass == 0, 0.0, loss.double() + tau * tau * (mass * (l - lse.double()) + part.double() - c))
        assert float(lse.abs().max()) < 20
        assert float(((whole - want).abs() - tol).max()) <= 0
    _close(echo.distill(x, w, ids, logits, temperature=tau, teacher_lse=lt)[0], want, tol)

    dloss, dlse = _randn((n,), 4), _randn((n,), 5)
    lse = l.float()
    up = dloss.double()[:, None] * tau
    coef = (up * q).sum(1) + dlse.double() / tau
    a, b, ta, tb = ref.grads(coef, (up * q).abs().sum(1), ref.targets(ids, up * q, 0), lse.double(), 1.0, F32)
    ecoef = (up * eq).abs().sum(1) + 16 * U * ((up * q).abs().sum(1) + coef.abs())
    eP = ref.targets(ids, (up * eq).abs(), 0) + ecoef[:, None] * torch.exp(ref.z - lse.double()[:, None]) * 1.01
    dx = torch.zeros((n, h), dtype=torch.float64, device="cuda")
    rounding = torch.zeros_like(dx)
    for p in range(0, v, rows):
        part, dw = echo.distill_grad(dloss, x, w[p:p + rows], ids, logits, lse, temperature=tau, teacher_lse=lt, vocab_start=p, dlse=dlse)
        _close(dw, b[p:p + rows], tb[p:p + rows] + (eP.T @ ref.X.abs())[p:p + rows])
        dx += part.double()
        rounding += {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}[dtype] * part.double().abs() + 2.0 ** -24
    assert float(((dx - a).abs() - (ta + eP @ ref.W.abs() + rounding * 1.01)).max()) <= 0
