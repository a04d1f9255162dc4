"""Durations of a training step's kernels, measured on this GPU and composed into the step's timeline.

A tracer runs each rank's kernels on one device and measures them (Sec. 4.1 of the paper).  This example does so for the
kernel classes that the library runs itself, at the shapes of one rank of a workload: the embedding lookup and its gradient
(first pipeline stage), the layer norms forward and backward, and the step of a matrix optimizer, whose updates the library
makes orthogonal.  Their times replace the generator's for those ops; the step is composed with both.  The optimizer is
another one than the generator's, which reads and writes 16 bytes a parameter in three ops: the measured step is the same
workload with a matrix optimizer, and the whole time of its step, momentum and weights included, is spread over the three.
Matrix products and attention keep the generator's durations.

    python examples/measured_step.py [tiny | gpt1.3b | gpt175b]
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2412_12487_gb300 import Echo  # noqa: E402
from paper_2412_12487_gb300 import workloads as W  # noqa: E402


def update(e: Echo, weight, momentum, grad, rate: float = 0.02, decay: float = 0.95):
    """A matrix optimizer's step for weights [..., rows, cols]: the momentum's orthogonalised update, scaled for tall ones."""
    momentum.mul_(decay).add_(grad)
    rows, cols = weight.shape[-2:]
    weight.add_(e.orthogonalize(momentum, scale=max(1.0, rows / cols) ** 0.5), alpha=-rate)


def measure(e: Echo, c: W.GPTConfig, reps: int = 5):
    """Nanoseconds of each operator on one rank: {"embed", "embed_grad", "norm", "norm_grad", "optimizer"}.

    A row of calls is captured in a graph, on a context of its own beside ``e``, and timed as a whole: what the kernels take
    in a stream, without the calls and without events between them.  Inputs that fit L2 stay there, as those do that the
    kernel before has just written."""
    tokens, hidden, rows = c.seq, c.hidden, W.VOCAB // c.tp
    bf16, dev = torch.bfloat16, torch.device("cuda", e.device)
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(side), Echo(e.device, stream=side) as own:
        gen = torch.Generator(device=dev).manual_seed(0)
        ids = torch.randint(0, W.VOCAB, (tokens,), generator=gen, device=dev)
        table = torch.randn((rows, hidden), generator=gen, device=dev).to(bf16)
        weight, bias = torch.ones(hidden, device=dev), torch.zeros(hidden, device=dev)
        main = {k: torch.zeros_like(v, dtype=torch.float32) for k, v in (("table", table), ("weight", weight), ("bias", bias))}
        layers, h, t = c.layers // c.pp, c.hidden, c.tp
        shapes = [(layers, *s) for s in ((3 * h // t, h), (h, h // t), (4 * h // t, h), (h, 4 * h // t))]  # of a stage's layers
        weights, momenta, grads = ([torch.randn(s, generator=gen, device=dev, dtype=bf16) for s in shapes] for _ in range(3))

        def time(call, n):
            result = call()  # scratch memory is allocated
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                for _ in range(n):
                    call()
            graph.replay()
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            graph.replay()
            end.record()
            end.synchronize()
            return result, begin.elapsed_time(end) * 1e6 / n

        def optimizer():
            for w, m, g in zip(weights, momenta, grads):
                update(own, w, m, g)

        ns, many = {}, 20 * reps
        x, ns["embed"] = time(lambda: own.embed(ids, table), many)
        (y, mean, rstd), ns["norm"] = time(lambda: own.layer_norm(x, weight, bias), many)
        (dx, _, _), ns["norm_grad"] = time(lambda: own.layer_norm_grad(y, x, mean, rstd, weight, dweight=main["weight"], dbias=main["bias"], accumulate=True), many)
        _, ns["embed_grad"] = time(lambda: own.embed_grad(ids, dx, rows, out=main["table"], accumulate=True), many)
        _, ns["optimizer"] = time(optimizer, reps)
        own.wait()
    return ns


def put(g: W.Graph, c: W.GPTConfig, dur: np.ndarray, ns) -> np.ndarray:
    """``dur`` [ops][scenarios] with the measured times in the place of the ops of their classes."""
    dur = dur.copy()
    comp = g.kind == W.KIND_COMPUTE
    norm = comp & (g.kclass == W.KC_NORM)
    forward = g.work < 5 * c.seq * c.hidden * W.MEM_FLOP_PER_BYTE  # (4 bytes an element; the backward norms have 6)
    dur[norm & forward] = round(ns["norm"])
    dur[norm & ~forward] = round(ns["norm_grad"])
    # a lookup waits for the copy of its tokens; a gradient does not
    first = np.minimum(g.pred_off[:-1], max(len(g.pred_idx) - 1, 0))
    after_copy = (np.diff(g.pred_off) > 0) & (g.kind[g.pred_idx[first]] == W.KIND_MEMCPY)
    emb = comp & (g.kclass == W.KC_EMB)
    dur[emb & after_copy] = round(ns["embed"])
    dur[emb & ~after_copy] = round(ns["embed_grad"])
    dur[comp & (g.kclass == W.KC_OPT)] = round(ns["optimizer"] / 3)  # (the step's three ops; every stage has as many layers)
    return dur


def main(name: str = "gpt1.3b"):
    c = W.config(name)
    g = W.build_gpt_graph(c)
    sc = W.make_scenarios(g, c, n_scen=4)
    with Echo(0) as e:
        ns = measure(e, c)
        for k, v in ns.items():
            print(f"{k:12s} {v * 1e-3:10.1f} us")
        e.load_graph(g)
        for label, dur in (("generated", sc.dur), ("measured", put(g, c, sc.dur, ns))):
            e.load_scenarios(sc, dur=dur)
            e.estimate_collectives()
            e.compose()
            print(f"step with {label} durations: " + ", ".join(f"{m * 1e-6:.2f}" for m in e.read_makespan()) + " ms")


if __name__ == "__main__":
    main(*sys.argv[1:2])
