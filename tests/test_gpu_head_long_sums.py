"""Long sums of few rows, whose tiles are shared by many blocks: what the tensor core's truncation takes from them.

A sum of numbers of one sign shows it as a bias, the same for all results, which the mean over them leaves and other errors
do not.  Bounds, written down before the first run (U = 2^-24):

* a set of S stages is 4 S additions to a sum that grows from nothing; each loses less than 2 U of the sum so far, U in the
  mean, which is half of the set's end in the mean over the set: 2 S U of the result.  S is the mean of the lengths of a
  tile's sets, weighted by them: 11/8 of a usual set (3 stages for fp32 matrices, 2 of them up to 256 tokens).
* the exponential: 2^-22, as if it erred to one side; fp32's other steps of a factor of all results (the factor that turns a
  sum into a logit in base 2 and back, P's scale, the result's rounding): 2 U.
* all else has mixed signs: roundings to the nearest of P (2^-22), of the operands (2^-22), of the sums of sets; over at
  least 2e4 results of 5000 terms each it leaves less than U / 8.
"""
import pytest

from paper_2412_12487_gb300 import Echo

from .test_gpu_head import F32, U, _randn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def echo():
    with Echo(0) as e:
        yield e


def _positive(shape, seed, size):
    """Around ``size``, from 0.2 to 1.8 of it."""
    return _randn(shape, seed).mul_(0.25).clamp_(-0.8, 0.8).add_(1).mul_(size)


def _bias(got, want):
    return float(((got.double() - want) / want).mean())


@pytest.mark.parametrize("n,h,v,usual", [(200, 256, 51200, 2), (48, 1024, 51200, 2), (300, 256, 51200, 3), (1003, 517, 5003, 3)])
def test_gradients_over_many_rows(echo, n, h, v, usual):
    """The gradient of lse alone: dx is a mean of the weight's rows."""
    x, w = _randn((n, h), 1, F32, 0.1), _positive((v, h), 2, 0.02)
    labels, zero, one = torch.full((n,), -1, device="cuda"), torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    z = x.double() @ w.double().T
    lse = torch.logsumexp(z, 1).float()
    dx = echo.cross_entropy_grad(zero, x, w, labels, lse, dlse=one)[0]
    want = torch.exp(z - lse.double()[:, None]) @ w.double()
    assert abs(_bias(dx, want)) <= 2 * (11 / 8 * usual) * U + 2.0 ** -22 + 2 * U


@pytest.mark.parametrize("n,h,v,usual", [(300, 8192, 1000, 3), (2048, 2048, 512, 3), (64, 4096, 51200, 2)])
def test_logits_of_long_rows(echo, n, h, v, usual):
    """The label's logit, a sum over one row, where tiles are split and where some are.  (Up to 256 tokens and more than 76
    tiles: the tiles left over.)"""
    x, w = _positive((n, h), 3, 1.0), _positive((v, h), 4, 1.0 / h)
    labels = torch.arange(n, device="cuda") * (v // n if v > n else 1) % v
    if v > 40000:
        labels = v - 1 - torch.arange(n, device="cuda") * 8  # (the last tiles)
    target = echo.cross_entropy(x, w, labels)[2]
    want = (x.double() * w.double()[labels]).sum(1)
    # n results only: a rounding of the sums of sets (at most 300 to the nearest, U / 2 in the mean square each, of half the
    # sum) leaves 9 U of one and 9 U / sqrt(n) of the mean, four times which is allowed
    assert abs(_bias(target, want)) <= 2 * (11 / 8 * usual) * U + 2 * U + 36 * U / n ** 0.5
