"""The operators as a training step uses them: one after the other, forward and backward, against 64-bit differentiation;
and their measured times in a step's timeline."""
import importlib.util
import math
import os

import numpy as np
import pytest

import oracle
from paper_2412_12487_gb300 import Echo, rotary_frequencies
from paper_2412_12487_gb300 import workloads as W

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("measured_step", os.path.join(ROOT, "examples", "measured_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


NS = {"embed": 1e4, "embed_grad": 2e4, "norm": 3e4, "norm_grad": 4e4, "optimizer": 15e4, "rotary": 7_000_003_003, "rotary_grad": 8_000_009_003,
      "loss": 2 * 9_000_011_003, "loss_grad": 3 * 11_000_017_003}  # (times that no generated op has)


@pytest.mark.parametrize("name", ["tiny", "gpt1.3b"])
def test_measured_times_go_to_their_ops(name):
    m = _example()
    c = W.config(name)
    g = W.build_gpt_graph(c)
    sc = W.make_scenarios(g, c, n_scen=1)
    dur = m.put(g, c, sc.dur, NS)[:, 0]
    comp = g.kind == W.KIND_COMPUTE
    count = {v: int((comp & (dur == v)).sum()) for v in (7_000_003_003, 8_000_009_003, 9_000_011_003, 11_000_017_003)}
    passes = c.dp * c.tp * c.microbatches
    assert count[7_000_003_003] == count[8_000_009_003] == passes * c.layers    # a rotation a layer, each way
    assert count[9_000_011_003] == 2 * passes                            # the last stage's product and loss
    assert count[11_000_017_003] == 3 * passes                           # its loss and two products, backward
    loss = comp & (g.kclass == W.KC_LOSS)
    assert int(loss.sum()) == 2 * passes and set(dur[loss]) == {9_000_011_003, 11_000_017_003}
    assert set(g.kclass[comp & np.isin(dur, (7_000_003_003, 8_000_009_003))]) == {W.KC_ELEM}
    old = m.put(g, c, sc.dur, {k: v for k, v in NS.items() if k in ("embed", "embed_grad", "norm", "norm_grad", "optimizer")})[:, 0]
    changed = ~np.isin(dur, (7_000_003_003, 8_000_009_003, 9_000_011_003, 11_000_017_003))
    assert np.array_equal(dur[changed], old[changed])


@pytest.mark.gpu
def test_a_step_with_all_measured_durations_matches_the_oracle():
    m = _example()
    c = W.config("tiny")
    g = W.build_gpt_graph(c)
    sc = W.make_scenarios(g, c, n_scen=2)
    with Echo(0) as e:
        more = m.measure_layers_and_loss(e, c, reps=2)
        assert set(more) == {"rotary", "rotary_grad", "loss", "loss_grad"} and min(more.values()) > 500
        sc.dur = m.put(g, c, sc.dur, {**m.measure(e, c, reps=2), **more})
        e.load_graph(g)
        e.load_scenarios(sc)
        e.estimate_collectives()
        e.compose()
        start, finish = e.read_times()
    want = oracle.compose(g, sc, refine_passes=1)
    assert np.array_equal(finish, want.finish) and np.array_equal(start, want.start)


@pytest.mark.gpu
@pytest.mark.parametrize("captured", [False, True])
def test_a_layer_from_tokens_to_gradients(captured):
    """Embedding, norm, projections, rotation, scores, norm, loss of labels and of a teacher: gradients of every weight
    against automatic differentiation in 64 bits.  All matrices are fp32.

    Tolerance: every operator is within 2^-18 of its own size here (sums of up to 300 terms, 22-bit operands), and the
    products between them, by torch in fp32, within 2^-16; ten of them in a row, whose slopes are at most 2 (norms of rows near
    unit deviation): 10 * 2 * 2^-16 of the gradient's largest element, 2^-11."""
    tokens, hidden, vocab, heads, dim, top = 96, 64, 300, 4, 16, 5
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    labels = torch.where(torch.arange(tokens, device="cuda") % 7 == 0, -100, torch.roll(ids, -1))
    top_ids, top_logits = torch.randint(-1, vocab, (tokens, top), generator=gen, device="cuda"), rand(tokens, top)
    at = torch.arange(tokens, device="cuda") % 40
    table, ln, wq, wk, head = rand(vocab, hidden), 1 + 0.1 * rand(hidden), rand(hidden, hidden) / 8, rand(hidden, hidden) / 8, rand(vocab, hidden) / 8
    bias = 0.1 * rand(hidden)
    f, tau, scale = rotary_frequencies(dim), 2.0, 1 / math.sqrt(dim)
    g_ce, g_kd = torch.full((tokens,), 1 / tokens, device="cuda"), torch.full((tokens,), 0.5 / tokens, device="cuda")

    def ours(e):
        x = e.embed(ids, table)
        y, mean, rstd = e.layer_norm(x, ln, bias)
        q, k = (y @ wq).view(tokens, heads, dim), (y @ wk).view(tokens, heads, dim)
        qr, kr = e.rotary(q, k, at, f)
        # scores of neighbouring tokens weigh the token before
        s = (qr * torch.roll(kr, 1, 0)).sum(-1, keepdim=True) * scale
        z = (y.view(tokens, heads, dim) * (1 + s)).reshape(tokens, hidden)
        _, lse, _ = e.cross_entropy(z, head, labels)
        loss, _, _ = e.cross_entropy(z, head, labels)
        kd, lse_kd, _ = e.distill(z, head, top_ids, top_logits, temperature=tau)
        dz, dhead = e.cross_entropy_grad(g_ce, z, head, labels, lse)
        dz2, dhead = e.distill_grad(g_kd, z, head, top_ids, top_logits, lse_kd, temperature=tau, dweight=dhead, accumulate=True)
        dz = (dz + dz2).view(tokens, heads, dim)
        dy = dz * (1 + s)
        ds = (dz * y.view(tokens, heads, dim)).sum(-1, keepdim=True) * scale
        dq, dk = e.rotary_grad(ds * torch.roll(kr, 1, 0), torch.roll(ds * qr, -1, 0), at, f)
        dq, dk = dq.view(tokens, hidden), dk.view(tokens, hidden)
        dy = dy.reshape(tokens, hidden) + dq @ wq.T + dk @ wk.T
        dx, dln, dbias = e.layer_norm_grad(dy, x, mean, rstd, ln)
        return loss, kd, e.embed_grad(ids, dx, vocab), dln, dbias, y.T @ dq, y.T @ dk, dhead

    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), Echo(0, stream=side) as e:
            ours(e)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = ours(e)
            for _ in range(2):
                graph.replay()
            e.wait()
    else:
        with Echo(0) as e:
            got = ours(e)
    w = [t.double().requires_grad_() for t in (table, ln, bias, wq, wk, head)]
    x = w[0][ids]
    y = torch.nn.functional.layer_norm(x, (hidden,), w[1], w[2], 1e-5)
    angle = at.double()[:, None, None] * torch.tensor(f, device="cuda")
    c, s_ = torch.cos(angle), torch.sin(angle)

    def turn(t):
        a, b = t[..., :dim // 2], t[..., dim // 2:]
        return torch.cat((a * c - b * s_, a * s_ + b * c), -1)

    qr, kr = turn((y @ w[3]).view(tokens, heads, dim)), turn((y @ w[4]).view(tokens, heads, dim))
    s = (qr * torch.roll(kr, 1, 0)).sum(-1, keepdim=True) * scale
    logits = (y.view(tokens, heads, dim) * (1 + s)).reshape(tokens, hidden) @ w[5].T
    loss = torch.nn.functional.cross_entropy(logits, labels, reduction="none", ignore_index=-100)
    t = (top_logits.double() / tau).masked_fill(top_ids < 0, -math.inf)
    none = (top_ids < 0).all(1)
    t = torch.where(none[:, None], 0.0, t)
    q = torch.softmax(t, 1)
    log_p = torch.log_softmax(logits / tau, 1).gather(1, top_ids.clamp_min(0))
    kd = torch.where(none, 0.0, tau * tau * (torch.where(q > 0, q * (torch.log(q.clamp_min(1e-300)) - log_p), 0.0)).sum(1))
    ((g_ce.double() * loss).sum() + (g_kd.double() * kd).sum()).backward()
    for name, a, b in zip(("loss", "kd", "table", "ln", "bias", "wq", "wk", "head"), got, (loss, kd, w[0].grad, w[1].grad, w[2].grad, w[3].grad, w[4].grad, w[5].grad)):
        off = float((a.double() - b.detach()).abs().max() / b.detach().abs().max())
        assert off <= 2.0 ** -11, (name, off)
