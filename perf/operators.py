"""The operators of a rank's training step that the library runs itself, as cases to measure.

Each is a kernel class of the step's execution graph (``workloads``): the embedding lookup of the first pipeline stage and
its gradient, the layer norms of every layer forward and backward, and the orthogonalised update of a matrix optimiser.
Shapes are those of ``workloads.CONFIGS``: one micro-batch of ``seq`` tokens, the hidden size, a vocabulary of 51200 rows
split over the tensor-parallel ranks.

``run`` computes an operator in its plain form, from elementary operations in 32 bits, or, where ``own`` is true, through
the library's own entry points.
"""
import functools
import math

import torch

own = False

VOCAB = 51200
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
ORTHO_EPS = 1e-7
LN_EPS = 1e-5


def _embed(tokens, hidden, vocab_rows, vocab_start, table, out, ids=64):
    return {"op": "embed", "tokens": tokens, "hidden": hidden, "vocab_rows": vocab_rows, "vocab_start": vocab_start, "table": table, "out": out, "ids": ids}


def _embed_grad(tokens, hidden, vocab_rows, vocab_start, dy, table, accumulate, ids=64):
    return {"op": "embed_grad", "tokens": tokens, "hidden": hidden, "vocab_rows": vocab_rows, "vocab_start": vocab_start, "dy": dy, "table": table,
            "accumulate": accumulate, "ids": ids}


def _ln(rows, hidden, x, param):
    return {"op": "layer_norm", "rows": rows, "hidden": hidden, "x": x, "param": param}


def _ln_grad(rows, hidden, x, param, accumulate):
    return {"op": "layer_norm_grad", "rows": rows, "hidden": hidden, "x": x, "param": param, "accumulate": accumulate}


def _ortho(batch, rows, cols, x, steps=5):
    return {"op": "orthogonalize", "batch": batch, "rows": rows, "cols": cols, "x": x, "steps": steps}


def listed():
    return [
        # one micro-batch of the smallest workload on one of two tensor-parallel ranks: launches are all there is
        dict(_embed(512, 1024, VOCAB // 2, 0, "bf16", "bf16"), name="embed-tiny"),
        # a micro-batch of the 96-layer workload, looked up in one of eight shards of the fp32 master table: tokens of the
        # other shards give zero rows
        dict(_embed(2048, 12288, VOCAB // 8, 0, "f32", "bf16"), name="embed-gpt175b"),
        # one micro-batch's gradient added to the rank's fp32 main gradient: few of the shard's rows are touched
        dict(_embed_grad(2048, 2048, VOCAB // 2, 0, "bf16", "f32", True), name="embed-grad-gpt1.3b-add"),
        # eight micro-batches at once into a fresh 16-bit gradient of the whole table; the commonest token has a thousand rows
        dict(_embed_grad(16384, 2048, VOCAB, 0, "bf16", "bf16", False), name="embed-grad-gpt1.3b-8mb"),
        # one token, as a decoder's step has it
        dict(_ln(1, 2048, "bf16", "bf16"), name="ln-1-row"),
        # a norm of the 96-layer workload: one micro-batch
        dict(_ln(2048, 12288, "bf16", "f32"), name="ln-gpt175b"),
        # the backward pass of the smallest workload's norm
        dict(_ln_grad(512, 1024, "bf16", "bf16", False), name="ln-grad-tiny"),
        # a ragged batch of packed sequences and an odd hidden size, in full precision
        dict(_ln_grad(4999, 1537, "f32", "f32", False), name="ln-grad-odd"),
        # the backward pass of a norm of the 96-layer workload, its parameters' gradients added to fp32 main gradients
        dict(_ln_grad(2048, 12288, "bf16", "f32", True), name="ln-grad-gpt175b"),
        # the update of an odd-shaped weight in full precision
        dict(_ortho(1, 1003, 517, "f32"), name="ortho-odd"),
        # the attention projections of a pipeline stage's six layers, on one of two tensor-parallel ranks
        dict(_ortho(6, 2048, 1024, "bf16"), name="ortho-gpt1.3b-proj"),
        # the query, key and value weight of one layer of the 96-layer workload, on one of eight tensor-parallel ranks
        dict(_ortho(1, 4608, 12288, "f32"), name="ortho-gpt175b-qkv"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "layer_norm", "layer_norm_grad", "orthogonalize"])
    if op == "orthogonalize":
        while True:
            batch, rows, cols = rng.randint(1, 6), _log_int(rng, 16, 12288), _log_int(rng, 16, 12288)
            m, n = min(rows, cols), max(rows, cols)
            if batch * m * m * n <= 4608 * 4608 * 4096:
                break
        return _ortho(batch, rows, cols, rng.choice(["f32", "bf16", "f16"]), rng.choice([3, 5, 5, 6]))
    while True:
        tokens, hidden = _log_int(rng, 1, 16384), _log_int(rng, 64, 12288)
        if rng.random() < 0.5:
            hidden = max(64, hidden // 64 * 64)
        if tokens * hidden <= 4096 * 12288:
            break
    x = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op == "layer_norm":
        return _ln(tokens, hidden, x, rng.choice(["f32", x]))
    if op == "layer_norm_grad":
        return _ln_grad(tokens, hidden, x, rng.choice(["f32", x]), rng.random() < 0.5)
    tp = rng.choice([1, 2, 4, 8])
    rows = min(VOCAB // tp, (1 << 28) // hidden)
    start = rows * rng.randint(0, tp - 1)
    ids = rng.choice([32, 64])
    if op == "embed":
        return _embed(tokens, hidden, rows, start, rng.choice(["f32", x]), x, ids)
    return _embed_grad(tokens, hidden, rows, start, x, rng.choice(["f32", x]), rng.random() < 0.5, ids)


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _token_ids(n, bits, gen):
    """Token ids as text has them: four fifths fall off as one over their rank, the others are spread over the vocabulary."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    common = torch.exp(u * math.log(VOCAB)).long() - 1
    spread = torch.randint(0, VOCAB, (n,), generator=gen, device="cuda")
    pick = torch.rand(n, generator=gen, device="cuda") < 0.8
    return torch.where(pick, common, spread).clamp_(0, VOCAB - 1).to(torch.int32 if bits == 32 else torch.int64)


def _normal(shape, gen, std=1.0, mean=0.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).add_(mean)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    if op == "embed":
        ids = _token_ids(case["tokens"], case["ids"], gen)
        return {"case": case, "ids": ids, "table": _normal((case["vocab_rows"], case["hidden"]), gen, 0.02).to(TYPES[case["table"]]),
                "scale": math.sqrt(case["hidden"])}
    if op == "embed_grad":
        ids = _token_ids(case["tokens"], case["ids"], gen)
        state = {"case": case, "ids": ids, "dy": _normal((case["tokens"], case["hidden"]), gen, 1e-2).to(TYPES[case["dy"]]),
                 "scale": math.sqrt(case["hidden"]), "sum": None}
        if case["accumulate"]:
            state["sum"] = _normal((case["vocab_rows"], case["hidden"]), gen, 1e-2).to(TYPES[case["table"]])
        return state
    if op == "orthogonalize":
        # a gradient: some strong directions over a floor of noise
        b, r, c = case["batch"], case["rows"], case["cols"]
        k = max(1, min(r, c) // 16)
        strong = torch.bmm(_normal((b, r, k), gen), _normal((b, k, c), gen)).div_(math.sqrt(k))
        return {"case": case, "g": strong.add_(_normal((b, r, c), gen, 0.5)).mul_(1e-3).to(TYPES[case["x"]])}
    # activations of a residual stream: channels of different means and sizes, a few of them large
    rows, hidden = case["rows"], case["hidden"]
    size = torch.exp(_normal((hidden,), gen, 0.4))
    size[torch.randint(0, hidden, (max(1, hidden // 256),), generator=gen, device="cuda")] *= 8
    x = _normal((rows, hidden), gen).mul_(size).add_(_normal((hidden,), gen, 0.3, 0.2)).to(TYPES[case["x"]])
    w = _normal((hidden,), gen, 0.1, 1.0).to(TYPES[case["param"]])
    if op == "layer_norm":
        return {"case": case, "x": x, "w": w, "b": _normal((hidden,), gen, 0.1).to(TYPES[case["param"]])}
    x32 = x.float()
    mean = x32.mean(1)
    rstd = torch.rsqrt((x32 - mean[:, None]).square_().mean(1) + LN_EPS)
    state = {"case": case, "x": x, "w": w, "mean": mean, "rstd": rstd, "dy": _normal((rows, hidden), gen, 1e-2).to(x.dtype), "dw": None, "db": None}
    if case["accumulate"]:
        state["dw"], state["db"] = (_normal((hidden,), gen, 0.1).to(w.dtype) for _ in range(2))
    return state


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _context():
    """The context that a user's program keeps."""
    from paper_2412_12487_gb300 import Echo
    return Echo(0)


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    case, e = s["case"], _context()
    op = case["op"]
    if op == "embed":
        return {"out": e.embed(s["ids"], s["table"], scale=s["scale"], vocab_start=case["vocab_start"], dtype=TYPES[case["out"]])}
    if op == "embed_grad":
        return {"dtable": e.embed_grad(s["ids"], s["dy"], case["vocab_rows"], scale=s["scale"], vocab_start=case["vocab_start"],
                                       dtype=TYPES[case["table"]], out=s["sum"], accumulate=case["accumulate"])}
    if op == "layer_norm":
        y, mean, rstd = e.layer_norm(s["x"], s["w"], s["b"], eps=LN_EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "layer_norm_grad":
        dx, dw, db = e.layer_norm_grad(s["dy"], s["x"], s["mean"], s["rstd"], s["w"], dweight=s["dw"], dbias=s["db"], accumulate=case["accumulate"])
        return {"dx": dx, "dw": dw, "db": db}
    return {"o": e.orthogonalize(s["g"], steps=case["steps"], coefficients=COEFFICIENTS, eps=ORTHO_EPS)}


def _run_plain(s):
    case = s["case"]
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "layer_norm": _plain_ln, "layer_norm_grad": _plain_ln_grad,
            "orthogonalize": _plain_ortho}[case["op"]](case, s)


def _plain_embed(case, s):
    row = s["ids"].long() - case["vocab_start"]
    mine = (row >= 0) & (row < case["vocab_rows"])
    y = s["table"][row.clamp(0, case["vocab_rows"] - 1)].float() * s["scale"]
    return {"out": (y * mine[:, None]).to(TYPES[case["out"]])}


def _plain_embed_grad(case, s):
    row = s["ids"].long() - case["vocab_start"]
    mine = (row >= 0) & (row < case["vocab_rows"])
    dy = s["dy"].float() * (s["scale"] * mine[:, None])
    dtable = torch.zeros((case["vocab_rows"], case["hidden"]), device="cuda") if s["sum"] is None else s["sum"].float()
    dtable.index_add_(0, row.clamp(0, case["vocab_rows"] - 1), dy)
    if s["sum"] is None:
        return {"dtable": dtable.to(TYPES[case["table"]])}
    if s["sum"].dtype != torch.float32:
        s["sum"].copy_(dtable)
    return {"dtable": s["sum"]}


def _plain_ln(case, s):
    x = s["x"].float()
    mean = x.sum(1) / case["hidden"]
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).sum(1) / case["hidden"] + LN_EPS)
    y = d * rstd[:, None] * s["w"].float() + s["b"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_ln_grad(case, s):
    dy, w = s["dy"].float(), s["w"].float()
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * w
    m1 = g.sum(1, keepdim=True) / case["hidden"]
    m2 = (g * xh).sum(1, keepdim=True) / case["hidden"]
    dx = (g - m1 - xh * m2) * s["rstd"][:, None]
    dw, db = (dy * xh).sum(0), dy.sum(0)
    if s["dw"] is None:
        return {"dx": dx.to(s["x"].dtype), "dw": dw.to(s["w"].dtype), "db": db.to(s["w"].dtype)}
    s["dw"].copy_(dw + s["dw"].float())
    s["db"].copy_(db + s["db"].float())
    return {"dx": dx.to(s["x"].dtype), "dw": s["dw"], "db": s["db"]}


def _newton_schulz(x, _):
    a, b, c = COEFFICIENTS
    p = torch.bmm(x, x.transpose(1, 2))
    return a * x + torch.bmm(b * p + c * torch.bmm(p, p), x)


def _plain_ortho(case, s):
    x = s["g"].float()
    x = x / (torch.sqrt((x * x).sum((1, 2), keepdim=True)) + ORTHO_EPS)
    wide = case["rows"] <= case["cols"]  # the smaller square products
    x = functools.reduce(_newton_schulz, range(case["steps"]), x if wide else x.transpose(1, 2))
    return {"o": (x if wide else x.transpose(1, 2)).to(s["g"].dtype).contiguous()}


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def _expected_rows(case):
    """Expected (tokens of the shard, distinct rows of it that they touch), from the distribution of the ids."""
    v = torch.arange(VOCAB, dtype=torch.float64)
    p = 0.8 * torch.log((v + 2) / (v + 1)) / math.log(VOCAB) + 0.2 / VOCAB
    p = p[case["vocab_start"]:case["vocab_start"] + case["vocab_rows"]]
    return float(p.sum()) * case["tokens"], float((1 - (1 - p) ** case["tokens"]).sum())


def work(case):
    op = case["op"]
    if op == "orthogonalize":
        m, n = sorted((case["rows"], case["cols"]))
        # two of the three products of a step are symmetric: half of each is enough
        return {"bytes": 2 * SIZE[case["x"]] * case["batch"] * m * n, "flops": case["batch"] * (case["steps"] * (3 * m * m * n + m ** 3) + 3 * m * n)}
    if op in ("embed", "embed_grad"):
        t, h = case["tokens"], case["hidden"]
        hits, distinct = _expected_rows(case)
        if op == "embed":
            return {"bytes": t * case["ids"] // 8 + distinct * h * SIZE[case["table"]] + t * h * SIZE[case["out"]], "flops": hits * h}
        table = 2 * distinct if case["accumulate"] else case["vocab_rows"]
        return {"bytes": t * case["ids"] // 8 + hits * h * SIZE[case["dy"]] + table * h * SIZE[case["table"]], "flops": 2 * hits * h}
    r, h = case["rows"], case["hidden"]
    if op == "layer_norm":
        return {"bytes": 2 * r * h * SIZE[case["x"]] + 2 * h * SIZE[case["param"]] + 8 * r, "flops": 8 * r * h}
    return {"bytes": 3 * r * h * SIZE[case["x"]] + (5 if case["accumulate"] else 3) * h * SIZE[case["param"]] + 8 * r, "flops": 14 * r * h}


# ---------------------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        row = s["ids"].to(torch.int64) - case["vocab_start"]
        out = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device="cuda")
        at = torch.nonzero((row >= 0) & (row < case["vocab_rows"])).flatten()
        out[at] = s["table"][row[at]].double() * s["scale"]
        return {"out": out}
    if op == "embed_grad":
        # tokens in the order of their rows; a row's sum is the difference of two running sums
        row = s["ids"].to(torch.int64) - case["vocab_start"]
        at = torch.nonzero((row >= 0) & (row < case["vocab_rows"])).flatten()
        row, order = torch.sort(row[at], stable=True)
        total = torch.zeros((case["vocab_rows"], case["hidden"]), dtype=torch.float64, device="cuda")
        if at.numel():
            running = torch.cumsum(s["dy"][at[order]].double(), 0)
            last = torch.nonzero(torch.cat([row[1:] != row[:-1], torch.ones(1, dtype=torch.bool, device="cuda")])).flatten()
            upto = running[last]
            total[row[last]] = s["scale"] * torch.cat([upto[:1], upto[1:] - upto[:-1]])
        return {"dtable": total if s["sum"] is None else total + s["sum"].double()}
    if op == "orthogonalize":
        a, b, c = COEFFICIENTS
        x = s["g"].double()
        x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + ORTHO_EPS)
        tall = case["rows"] > case["cols"]
        for _ in range(case["steps"]):
            # x p(x'x) or p(xx') x, whichever square is the smaller
            q = x.mT @ x if tall else x @ x.mT
            q = b * q + c * (q @ q)
            x = a * x + (x @ q if tall else q @ x)
        return {"o": x}
    x = s["x"].double()
    if op == "layer_norm":
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + LN_EPS) ** -0.5
        return {"y": torch.addcmul(s["b"].double(), (x - mean[:, None]) * rstd[:, None], s["w"].double()), "mean": mean, "rstd": rstd}
    # the gradient as the product with the Jacobian: the part along the constant and along the normalised row taken out
    mean, rstd = s["mean"].double()[:, None], s["rstd"].double()[:, None]
    dy, unit = s["dy"].double(), (x - mean) * rstd
    g = dy * s["w"].double()
    along = torch.einsum("rh,rh->r", g, unit) / case["hidden"]
    dx = rstd * (g - g.mean(1, keepdim=True) - unit * along[:, None])
    dw, db = torch.einsum("rh,rh->h", dy, unit), dy.sum(0)
    if s["dw"] is not None:
        dw, db = dw + s["dw"].double(), db + s["db"].double()
    return {"dx": dx, "dw": dw, "db": db}
