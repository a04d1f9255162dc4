"""Gradients of the logits that are small beside the largest: of tokens that hardly anything speaks for, which no norm of a
whole matrix shows.

Tokens are rows of the identity, so dweight is the transpose of dz and the logits are the weight's elements (exact in 16
bits; of two fp16 numbers in fp32, 2^-22 of an element, or 2^-37 of the largest).  With p the softmax's part of an element times the token's weight, dz = p minus that weight at its label,
and m the bound of dz over all tokens (twice the weight), an element is off by
  2^-19 of p for the exponential and the products (2^-20), the token's coefficient, lse's product with log2 e and the sums
        (U of one element, as the other tokens' are products with zero), and 2 U of the weight at the label;
  and, as one number of 16 bits, half a step of the type: 2^-8 in bf16 whatever its size, 2^-11 in fp16 and 2^-40 of m;
      as two fp16 numbers 2^-22 of it and 2^-40 of m;
and then rounded to dweight's type."""
import pytest

from paper_2412_12487_gb300 import Echo

from .test_gpu_head import BF16, F16, F32, TINY, UO, U, _randint, _randn

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dw_type", [(BF16, F32), (BF16, BF16), (F16, F32), (F16, F16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("weight", [1.0, 0.7, 1 / 1984])
def test_elements_of_all_sizes(dtype, dw_type, weight):
    n, v = 64, 3000
    x = torch.eye(n, device="cuda").to(dtype)
    w = _randn((v, n), 1, F32, 8.0).clamp_(-30, 30).to(dtype)
    labels = _randint(0, v, (n,), 2)
    labels[::9] = -1
    dloss = torch.full((n,), weight, device="cuda")
    z = w.double().T
    lse = torch.logsumexp(z, 1).float()
    dz = torch.exp(z - lse.double()[:, None])
    dz[torch.arange(n, device="cuda"), labels.clamp_min(0)] -= 1
    dz *= torch.where(labels >= 0, dloss.double(), 0.0)[:, None]
    with Echo(0) as e:
        _, dw = e.cross_entropy_grad(dloss, x, w, labels, lse, dtype=dw_type)
    m = 2 * float(dloss[0])
    label = dz < 0
    p = dz + label * m / 2
    tol = 2.0 ** -19 * p + 2 * U * label * m / 2
    if dtype == F32:
        tol = tol + 1.01 * p * (2.0 ** -22 * z.abs() + 2.0 ** -37 * float(w.abs().max()))
    if F32 in (dtype, dw_type):
        tol = tol + 2.0 ** -22 * dz.abs() + 2.0 ** -40 * m
    else:
        tol = tol + UO[dtype] * dz.abs() + (2.0 ** -40 * m if dtype == F16 else 0.0)
    off = (dw.double().T - dz).abs() - (tol + UO[dw_type] * (dz.abs() + tol) + TINY[dw_type])
    assert float(off.max()) <= 0
    assert float(dz.abs()[labels >= 0].min()) < 1e-18  # (sizes over all of the range)
