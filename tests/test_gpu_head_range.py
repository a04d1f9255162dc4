"""Losses of a head at fp32 elements near the ends of fp32, whose products are ordinary numbers.  Tolerances as in
test_gpu_head.py."""
import pytest

from paper_2412_12487_gb300 import Echo

from .test_gpu_head import F32, Ref, _check_ce, _close, _randint, _randn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def echo():
    with Echo(0) as e:
        yield e


@pytest.mark.parametrize("h", [64, 65])
@pytest.mark.parametrize("far", [60, 100, 110, 125])
@pytest.mark.parametrize("n", [5, 40])
def test_tokens_and_weights_far_from_one(echo, n, far, h):
    """Tokens of 2^far and rows of the weight as much below one (2^-108 at the least: a row's largest element is 2^-112 or
    more, below which digits are lost), and the other way round; times what takes logits back to some units."""
    v = 300
    low = min(far, 108)
    for a, b in ((far, -low), (-low, far)):
        x, w = _randn((n, h), 1).clamp_(-6, 6) * 2.0 ** a, _randn((v, h), 2, F32, 0.125).clamp_(-0.75, 0.75) * 2.0 ** b
        scale = 2.0 ** -(a + b)
        labels, dloss = _randint(-1, v, (n,), 3), _randn((n,), 4)
        lse = _check_ce(echo, x, w, labels, 0, scale)
        ref = Ref(x, w, scale)
        up = torch.where(labels >= 0, dloss.double() * scale, 0.0)
        dx, dw, tx, tw = ref.grads(up, up.abs(), ref.targets(labels[:, None], up[:, None], 0), lse.double(), 1.0, F32)
        got = echo.cross_entropy_grad(dloss, x, w, labels, lse, scale=scale)
        # (dx is 2^-128 where the weight is 2^-108: below 2^-126 numbers are multiples of 2^-149, so each of a sum's v or n
        # additions is off by up to 2^-150 whatever its size, which the other bounds, in parts of magnitudes, do not count)
        _close(got[0], dx, tx + v * 2.0 ** -150)
        _close(got[1], dw, tw + n * 2.0 ** -150)


def test_equal_elements_far_from_one(echo):
    """Sums of 64 products of 2^110 and 2^-95 are 2^21, of all tokens and rows."""
    x, w = torch.full((17, 64), 2.0 ** 110, device="cuda"), torch.full((30, 64), 2.0 ** -95, device="cuda")
    for a, b in ((x, w), (torch.full_like(x, 2.0 ** -95), torch.full_like(w, 2.0 ** 110))):
        loss, lse, target = echo.cross_entropy(a, b, torch.arange(17, device="cuda"))
        assert ((target - 2.0 ** 21).abs() <= 0.25).all() and torch.isfinite(loss).all()  # (two roundings: 2^21 over ln 2, and back)
        assert ((lse - 2.0 ** 21).abs() <= 4.5).all()  # (ln 30 = 3.4, and lse's rounding in fp32)
