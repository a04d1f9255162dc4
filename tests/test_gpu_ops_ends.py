"""Operators of a training step at the ends of what their interface promises.

Tolerances are written down before the first run.  u = 2^-24 is fp32's unit roundoff, uo the output type's.

* Newton-Schulz: an iterate's elements are sums of two fp16 numbers whatever the matrix's type, so e = 2^-22; a step
  multiplies an error by at most 3.9 while the iterate grows by up to 3.44, and five steps stay within 100 e of the result's
  norm (1210 e for an iterate of rank one, which starts at its final norm: the sum of 3.9^k).  A row's or a column's error is
  part of the matrix's.  Rounding the output adds uo of each element.
* A 16-bit result is the rounded exact one but where an error d moves an element across a boundary between two roundings.
  Boundaries lie at least uo |w| apart, so that happens to a share min(1, d / (uo |w|)) of elements w; for d = 100 e times their
  root mean square and normally distributed w the mean of it is 0.8 r (1 - log r), r = 100 e / uo: 3% for bf16 and 16% for fp16.
"""

import ctypes as C
import importlib.util
import math
import os
import time

import pytest

from paper_2412_12487_gb300 import Echo, EchoError
from paper_2412_12487_gb300 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
UO = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
QUINTIC = (3.4445, -4.7750, 2.0315)
TIMEOUT = 7  # ECHO_E_TIMEOUT


@pytest.fixture(scope="module")
def echo():
    with Echo(0) as e:
        yield e


def _randn(shape, seed, dtype=F32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def _ortho_ref(g, steps=5, coef=QUINTIC, eps=0.0):
    a, b, c = (torch.tensor(v, dtype=F32).double().item() for v in coef)
    x = g.double()
    x = x / (x.flatten(-2).norm(dim=-1)[..., None, None] + torch.tensor(eps, dtype=F32).double().item())
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    for _ in range(steps):
        q = x @ x.mT
        x = a * x + (b * q + c * q @ q) @ x
    return x.mT if tall else x


def _ortho_close(got, want, gain=100.0):
    """Every row and column of every matrix, by norm."""
    uo = UO[got.dtype]
    got, want = (t.double().reshape(-1, *t.shape[-2:]) for t in (got, want))
    assert torch.isfinite(got).all()
    tol = gain * 2.0 ** -22 * want.flatten(1).norm(dim=1)[:, None]
    for dim in (1, 2):
        off = (got - want).norm(dim=dim) - (uo * want.norm(dim=dim) + tol * (1 + uo))
        assert float(off.max()) <= 0, float(off.max())
    assert ((got - want).flatten(1).norm(dim=1) <= uo * want.flatten(1).norm(dim=1) + tol[:, 0] * (1 + uo)).all()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape", [(513, 512), (300, 1000), (1000, 300), (5, 384, 256), (129, 127), (2, 2048, 1024), (40, 3000), (1003, 517)])
def test_orthogonalize_16_bit_results_are_the_rounded_ones(echo, dtype, shape):
    g = _randn(shape, 1, dtype)
    got, want = echo.orthogonalize(g, eps=0.0), _ortho_ref(g)
    _ortho_close(got, want)
    moved = float((got != want.to(dtype)).double().mean())
    assert moved <= {BF16: 0.05, F16: 0.25}[dtype], moved


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_orthogonalize_rows_and_columns(echo, dtype):
    """Matrices at the edges of tiles, split sums, one row or column: nothing missing at an edge."""
    for k, shape in enumerate([(1, 7), (2, 33), (33, 2000), (255, 257), (256, 256), (257, 255), (3, 128, 300), (300, 5000), (2500, 2600), (700, 64)]):
        g = _randn(shape, 10 + k, dtype)
        _ortho_close(echo.orthogonalize(g, eps=0.0), _ortho_ref(g), 1210 if shape[0] <= 2 else 100)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_orthogonalize_low_rank(echo, dtype):
    g = torch.outer(_randn((70,), 30), _randn((300,), 31)).to(dtype)
    _ortho_close(echo.orthogonalize(g, eps=0.0), _ortho_ref(g), gain=1210)


def test_orthogonalize_elements_far_below_the_largest(echo):
    """Elements over thirty powers of two: those below 2^-14 of the norm have fewer bits, at no cost to the result's norm
    (their absolute error stays at 2^-37: 450 * 2^-37 of the norm for 200 x 1000)."""
    g = _randn((200, 1000), 32) * torch.exp2(-30 * torch.rand((200, 1000), generator=torch.Generator(device="cuda").manual_seed(33), device="cuda"))
    _ortho_close(echo.orthogonalize(g, eps=0.0), _ortho_ref(g), gain=101)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_orthogonalize_ends_of_the_range(echo, dtype):
    """Norms beyond fp32's largest number, and elements below its smallest normal one."""
    g = _randn((6, 48, 80), 34).double()
    g = g / g.abs().amax(dim=(1, 2), keepdim=True)
    sized = torch.stack([g[i] * 2.0 ** k for i, k in enumerate((127, 126, 100, -110, -124, -126))]).to(dtype)
    assert torch.isfinite(sized).all()
    _ortho_close(echo.orthogonalize(sized, eps=0.0), _ortho_ref(sized))
    tiny = (g * 2.0 ** -130).to(dtype)  # a few bits of each are left: the result is that matrix's own
    _ortho_close(echo.orthogonalize(tiny, eps=0.0), _ortho_ref(tiny))


@pytest.mark.parametrize("h", [64, 256, 1024])
def test_layer_norm_rstd_is_the_rounded_one(echo, h):
    """Rows of +a and -a: every sum is exact, so nothing but the last rounding is left of 1 / sqrt(a^2)."""
    a = torch.arange(1, 1024, device="cuda", dtype=F32)
    sign = torch.tensor([1.0, -1.0], device="cuda").repeat(h // 2)
    _, mean, rstd = echo.layer_norm(a[:, None] * sign, eps=0.0)
    assert not mean.any()
    assert torch.equal(rstd, (1 / a.double()).float())


def _gives_up(monkeypatch, limit_ms="20"):
    monkeypatch.setenv("ECHO_TEST_SKIP_LEVEL", "1")
    monkeypatch.setenv("ECHO_TEST_WAIT_LIMIT_MS", limit_ms)


def _code(call):
    with pytest.raises(EchoError) as err:
        call()
    return err.value.code


def test_the_stream_is_no_operator(monkeypatch):
    """Asking for the stream leaves the report of a wait that ran out to the next operator."""
    g = _randn((300, 280), 40)
    _gives_up(monkeypatch)
    with Echo(0) as e:
        e.orthogonalize(g, steps=1)
        torch.cuda.synchronize()
        s = C.c_void_p()
        assert e.lib.echo_stream_get(e.h, C.byref(s)) == 0 and s.value == e._stream
        assert _code(lambda: e.layer_norm(g)) == TIMEOUT
        e.layer_norm(g)


def test_a_wait_is_reported_once_while_the_rest_still_runs(monkeypatch):
    """The first products have given up, the others of the same call will: one report for all of them."""
    g = _randn((300, 280), 41)
    _gives_up(monkeypatch, "40")
    with Echo(0) as e:
        e.orthogonalize(g, steps=5)
        time.sleep(0.15)
        assert _code(lambda: e.layer_norm(g)) == TIMEOUT
        torch.cuda.synchronize()
        assert torch.isfinite(e.layer_norm(g)[0]).all()


def test_a_last_operator_is_waited_for(monkeypatch):
    g = _randn((300, 280), 42)
    with Echo(0) as e:
        e.wait()
        e.orthogonalize(g)
        e.wait()
    _gives_up(monkeypatch)
    with Echo(0) as e:
        e.orthogonalize(g, steps=1)
        assert _code(e.wait) == TIMEOUT
        e.wait()
        e.layer_norm(g)


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "measured_step.py")
    spec = importlib.util.spec_from_file_location("measured_step", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_measured_times_are_the_kernels_own():
    """A layer norm that is measured for a timeline takes what it takes in a row of kernels, not what it takes between events."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "measured_step.py")
    spec = importlib.util.spec_from_file_location("measured_step", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    c = W.config("tiny")
    with Echo(0) as e:
        ns = m.measure(e, c)
        x, w, b = _randn((c.seq, c.hidden), 50, BF16), _randn((c.hidden,), 51), _randn((c.hidden,), 52)
        for _ in range(5):
            e.layer_norm(x, w, b)
        e.read_profile()
        e.set_profiling(True)
        for _ in range(20):
            e.layer_norm(x, w, b)
        between_events = min(1e6 * ms / n for n, ms in e.read_profile().values())
        e.set_profiling(False)
    assert ns["norm"] <= 0.75 * between_events, (ns, between_events)


def test_a_larger_call_leaves_a_captured_graph_its_scratch():
    """A graph keeps the address of the scratch that it was captured with.  Larger calls come after the capture, then
    arrays that would take the place of memory given back: the graph's results stay right, and the arrays as they were."""
    side = torch.cuda.Stream()
    x, g, ids = _randn((64, 512), 60), _randn((96, 200), 61), torch.arange(64, device="cuda") % 50
    with Echo(0, stream=side) as e, torch.cuda.stream(side):
        def step(x, g, ids):
            y, mean, rstd = e.layer_norm(x)
            return *e.layer_norm_grad(y, x, mean, rstd), e.embed_grad(ids, y, 50), e.orthogonalize(g)

        want = step(x, g, ids)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step(x, g, ids)
        large = [step(_randn((r, 2048), 62), _randn((m, 2 * m), 63), torch.arange(r, device="cuda") % 50) for r, m in ((3000, 400), (9000, 1200))]
        side.synchronize()
        arrays = [torch.full((n,), 7.0, device="cuda") for n in (1 << 10, 1 << 16, 1 << 20, 1 << 21, 1 << 22, 1 << 24) for _ in range(4)]
        for _ in range(3):
            for o in out:
                o.zero_()
            graph.replay()
            for a, b in zip(out, want):
                assert torch.equal(a, b)
        assert all((a == 7).all() for a in arrays)
        for k, (r, m) in enumerate(((3000, 400), (9000, 1200))):
            again = step(_randn((r, 2048), 62), _randn((m, 2 * m), 63), torch.arange(r, device="cuda") % 50)
            assert all(torch.equal(a, b) for a, b in zip(large[k], again))
        side.synchronize()


def test_a_call_that_would_allocate_in_a_capture_is_refused():
    """... and the capture goes on without it."""
    side = torch.cuda.Stream()
    x, g = _randn((64, 512), 64), _randn((96, 200), 65)
    with Echo(0, stream=side) as e, torch.cuda.stream(side):
        y, mean, rstd = e.layer_norm(x)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            assert _code(lambda: e.orthogonalize(g)) == 4  # ECHO_E_STATE
            assert _code(lambda: e.layer_norm_grad(x, x, mean, rstd)) == 4
            z = e.layer_norm(x)[0]
        graph.replay()
        side.synchronize()
        assert torch.equal(z, y)
        e.orthogonalize(g)
        e.layer_norm_grad(x, x, mean, rstd)
        side.synchronize()


def test_the_measured_optimizer_step_is_a_whole_one(echo):
    """Momentum, orthogonalised update and weights: what the workload's optimizer ops stand for."""
    m = _example()
    w, v, g = (_randn((2, 96, 40), 70 + k) for k in range(3))
    w2, v2 = w.clone(), v.clone()
    m.update(echo, w2, v2, g, rate=0.125, decay=0.5)
    assert torch.equal(v2, v * 0.5 + g)
    want = math.sqrt(96 / 40) * _ortho_ref(v2, eps=1e-7)
    got = (w.double() - w2.double()) / 0.125
    # the update's own error, and a rounding of the weights in fp32, eight times as large in it
    assert float((got - want).norm()) <= 102 * 2.0 ** -22 * float(want.norm()) + 8 * 2.0 ** -24 * float(w2.double().norm())


def test_captured_calls_are_not_profiled():
    """A capture runs nothing, so it has no times: the profile holds what ran between its events, and no error is left behind."""
    side = torch.cuda.Stream()
    x = _randn((64, 512), 80)
    with Echo(0, stream=side) as e, torch.cuda.stream(side):
        want = e.layer_norm(x)[0]
        e.set_profiling(True)
        e.layer_norm(x)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = e.layer_norm(x)[0]
        graph.replay()
        (name, (launches, ms)), = e.read_profile().items()
        assert launches == 1 and ms > 0
        assert torch.equal(y, want)
        e.layer_norm(x)
        assert e.read_profile()[name][0] == 1
        torch.cuda.current_stream().synchronize()
