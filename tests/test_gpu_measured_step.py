"""The operators in the path they are for: measured durations composed into a step's timeline."""
import importlib.util
import os

import numpy as np
import pytest

import oracle
from paper_2412_12487_gb300 import Echo, EchoError
from paper_2412_12487_gb300 import workloads as W

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("measured_step", os.path.join(ROOT, "examples", "measured_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_measured_times_go_to_their_ops():
    m = _example()
    c = W.config("tiny")
    g = W.build_gpt_graph(c)
    sc = W.make_scenarios(g, c, n_scen=2)
    ns = {"embed": 1e4, "embed_grad": 2e4, "norm": 3e4, "norm_grad": 4e4, "optimizer": 15e4}
    dur = m.put(g, c, sc.dur, ns)
    comp = g.kind == W.KIND_COMPUTE
    count = {v: int((dur[:, 0] == v).sum()) for v in (10_000, 20_000, 30_000, 40_000, 50_000)}
    per_stage = c.dp * c.tp * c.microbatches
    assert count[10_000] == count[20_000] == per_stage                          # the first stage's lookups and gradients
    assert count[30_000] == count[40_000] == per_stage * (2 * c.layers + 1)     # two a layer, and the last stage's
    assert count[50_000] == 3 * c.dp * c.tp * c.pp
    other = ~(comp & np.isin(g.kclass, (W.KC_EMB, W.KC_NORM, W.KC_OPT)))
    assert np.array_equal(dur[other], sc.dur[other]) and np.array_equal(dur[:, 0][~other], dur[:, 1][~other])


@pytest.mark.gpu
def test_step_with_measured_durations_matches_the_oracle():
    m = _example()
    c = W.config("tiny")
    g = W.build_gpt_graph(c)
    sc = W.make_scenarios(g, c, n_scen=2)
    with Echo(0) as e:
        ns = m.measure(e, c, reps=2)
        assert set(ns) == {"embed", "embed_grad", "norm", "norm_grad", "optimizer"} and min(ns.values()) > 500
        sc.dur = m.put(g, c, sc.dur, ns)
        e.load_graph(g)
        e.load_scenarios(sc)
        e.estimate_collectives()
        e.compose()
        start, finish = e.read_times()
    want = oracle.compose(g, sc, refine_passes=1)
    assert np.array_equal(finish, want.finish) and np.array_equal(start, want.start)


@pytest.mark.gpu
def test_a_wait_that_runs_out_is_reported(monkeypatch):
    """A step's tiles that never arrive: the kernels give up, and the context's next operator says so, once."""
    g = torch.randn((300, 280), device="cuda")
    monkeypatch.setenv("ECHO_TEST_SKIP_LEVEL", "1")
    monkeypatch.setenv("ECHO_TEST_WAIT_LIMIT_MS", "20")
    with Echo(0) as e:
        e.orthogonalize(g, steps=1)
        torch.cuda.synchronize()
        with pytest.raises(EchoError) as err:
            e.layer_norm(g)
        assert err.value.code == 7  # ECHO_E_TIMEOUT
        x = e.layer_norm(g)[0]
        assert torch.isfinite(x).all()
    monkeypatch.delenv("ECHO_TEST_SKIP_LEVEL")
    with Echo(0) as e:
        assert torch.isfinite(e.orthogonalize(g)).all()
        e.layer_norm(g)
