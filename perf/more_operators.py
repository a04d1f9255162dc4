"""More operators of a rank's training step that the library runs itself, as cases to measure.

They are the last pipeline stage's loss and the rotary positions of every layer, forward and backward: softmax cross
entropy straight from hidden states and the head's weight, distillation from a teacher's top logits on the same head, and
the rotation of queries and keys.  Shapes are those of ``workloads.CONFIGS``: micro-batches of ``seq`` tokens, the hidden
size, a vocabulary of 51200 rows split over the tensor-parallel ranks, heads of 128 elements.

``run`` computes an operator in its plain form, from elementary operations in 32 bits (angles in 64), or, where ``own`` is
true, through the library's own entry points.
"""
import functools
import math

import torch

own = False

VOCAB = 51200
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MOST = 2048 * 12288 * 6400  # elements multiplied in the largest product


def _ce(tokens, hidden, vocab_rows, vocab_start, x, ids=64):
    return {"op": "cross_entropy", "tokens": tokens, "hidden": hidden, "vocab_rows": vocab_rows, "vocab_start": vocab_start, "x": x, "ids": ids}


def _ce_grad(tokens, hidden, vocab_rows, vocab_start, x, dw, accumulate, ids=64):
    return dict(_ce(tokens, hidden, vocab_rows, vocab_start, x, ids), op="cross_entropy_grad", dw=dw, accumulate=accumulate)


def _distill(tokens, hidden, vocab_rows, vocab_start, x, top, temperature, ids=64):
    return dict(_ce(tokens, hidden, vocab_rows, vocab_start, x, ids), op="distill", top=top, temperature=temperature)


def _distill_grad(tokens, hidden, vocab_rows, vocab_start, x, top, temperature, dw, accumulate, ids=64):
    return dict(_distill(tokens, hidden, vocab_rows, vocab_start, x, top, temperature, ids), op="distill_grad", dw=dw, accumulate=accumulate)


def _rotary(tokens, heads, kv_heads, dim, rot, x, interleaved, first, factor=1.0, grad=False, ids=64):
    return {"op": "rotary_grad" if grad else "rotary", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rot, "x": x,
            "interleaved": interleaved, "first": first, "factor": factor, "ids": ids}


def listed():
    return [
        # a small full-precision model with sizes that nothing divides
        dict(_ce(1003, 517, 5003, 0, "f32"), name="ce-odd"),
        # one micro-batch of the 96-layer workload on one of eight tensor-parallel ranks: labels of the other shards
        dict(_ce(2048, 12288, VOCAB // 8, 3 * (VOCAB // 8), "bf16"), name="ce-gpt175b"),
        # the backward pass of one micro-batch of the 24-layer workload, its weight's gradient added to the rank's fp32 main gradient
        dict(_ce_grad(2048, 2048, VOCAB // 2, 0, "bf16", "f32", True), name="ce-grad-gpt1.3b-add"),
        # the same of the 96-layer workload, into a fresh 16-bit gradient
        dict(_ce_grad(2048, 12288, VOCAB // 8, 0, "bf16", "bf16", False), name="ce-grad-gpt175b"),
        # the smallest workload taught by a teacher's sixteen best tokens
        dict(_distill(512, 1024, VOCAB // 2, 0, "bf16", 16, 1.0), name="distill-tiny"),
        # the 24-layer workload's micro-batch with the whole vocabulary on the rank and a softened teacher
        dict(_distill(2048, 2048, VOCAB, 0, "bf16", 64, 2.0), name="distill-gpt1.3b"),
        # a ragged batch of a small fp16 student
        dict(_distill_grad(777, 1000, 10007, 0, "f16", 7, 1.5, "f16", False), name="distill-grad-odd"),
        # the backward pass of the 24-layer workload's micro-batch, added to the fp32 main gradient
        dict(_distill_grad(2048, 2048, VOCAB // 2, 0, "bf16", 64, 2.0, "f32", True), name="distill-grad-gpt1.3b-add"),
        # one token far into its context, as a decoder's step has it
        dict(_rotary(1, 16, 16, 128, 128, "bf16", False, 70001), name="rotary-1-token"),
        # the queries and keys of one micro-batch of the 96-layer workload on one of eight tensor-parallel ranks
        dict(_rotary(2048, 12, 12, 128, 128, "bf16", False, 0), name="rotary-gpt175b"),
        # an odd number of heads in full precision, a quarter of each turned, in pairs of neighbours
        dict(_rotary(1999, 9, 3, 80, 20, "f32", True, 0, grad=True), name="rotary-grad-part"),
        # the gradients of a long context's queries and few keys, with frequencies scaled for eight times the length
        dict(_rotary(65536, 32, 8, 128, 128, "bf16", False, 0, 8.0, grad=True), name="rotary-grad-long"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["cross_entropy", "cross_entropy_grad", "distill", "distill_grad", "rotary", "rotary_grad"])
    x = rng.choice(["f32", "bf16", "bf16", "f16"])
    ids = rng.choice([32, 64])
    if op.startswith("rotary"):
        while True:
            tokens, heads = _log_int(rng, 1, 65536), _log_int(rng, 1, 96)
            kv = rng.choice([heads, max(1, heads // 4), 1])
            dim = rng.choice([32, 64, 80, 96, 128, 128, 256])
            if tokens * (heads + kv) * dim * SIZE[x] <= 65536 * 40 * 128 * 2:
                break
        rot = rng.choice([dim, dim, 2 * rng.randint(1, dim // 2)])
        return _rotary(tokens, heads, kv, dim, rot, x, rng.random() < 0.5, rng.choice([0, rng.randint(0, 1000000)]), rng.choice([1.0, 1.0, 4.0, 32.0]),
                       op == "rotary_grad", ids)
    while True:
        tokens, hidden = _log_int(rng, 1, 8192), _log_int(rng, 64, 12288)
        if rng.random() < 0.5:
            hidden = max(64, hidden // 64 * 64)
        tp = rng.choice([1, 2, 4, 8])
        rows = rng.choice([VOCAB // tp, rng.randint(1000, VOCAB // tp)])
        if tokens * hidden * rows <= MOST // (3 if x == "f32" else 1) and tokens * rows <= 2048 * VOCAB:
            break
    start = (VOCAB // tp) * rng.randint(0, tp - 1)
    top, temperature = _log_int(rng, 1, 128), rng.choice([1.0, 1.0, 2.0, 0.5])
    dw, accumulate = rng.choice(["f32", x]), rng.random() < 0.5
    if op == "cross_entropy":
        return _ce(tokens, hidden, rows, start, x, ids)
    if op == "cross_entropy_grad":
        return _ce_grad(tokens, hidden, rows, start, x, dw, accumulate, ids)
    if op == "distill":
        return _distill(tokens, hidden, rows, start, x, top, temperature, ids)
    return _distill_grad(tokens, hidden, rows, start, x, top, temperature, dw, accumulate, ids)


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _normal(shape, gen, std=1.0, mean=0.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).add_(mean)


def _int(t, bits):
    return t.to(torch.int32 if bits == 32 else torch.int64)


def _zipf(n, gen):
    """Token ids as text has them: four fifths fall off as one over their rank, the others are spread over the vocabulary."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    common = torch.exp(u * math.log(VOCAB)).long() - 1
    spread = torch.randint(0, VOCAB, (n,), generator=gen, device="cuda")
    pick = torch.rand(n, generator=gen, device="cuda") < 0.8
    return torch.where(pick, common, spread).clamp_(0, VOCAB - 1)


def _frequencies(case):
    """Radians a position of each pair; a factor above 1 slows the pairs that turn less than 32 times over 4096 positions."""
    half = case["rot"] // 2
    f = 10000.0 ** (-torch.arange(half, dtype=torch.float64) * 2 / case["rot"])
    turns = 4096 * f / (2 * math.pi)
    keep = ((turns - 1) / 31).clamp(0, 1)
    return f * (keep + (1 - keep) / case["factor"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    t = case["tokens"]
    if case["op"].startswith("rotary"):
        dtype = TYPES[case["x"]]
        f = _frequencies(case)
        # packed sequences: positions begin again a few times
        at = torch.arange(t, device="cuda")
        begin = torch.sort(torch.randint(0, t, (min(4, t),), generator=gen, device="cuda"))[0]
        begin[0] = 0
        which = torch.searchsorted(begin, at, right=True) - 1
        return {"case": case, "f": f.numpy(), "f_gpu": f.cuda(), "positions": _int(at - begin[which] + case["first"], case["ids"]),
                "scale": 0.1 * math.log(case["factor"]) + 1,
                "q": _normal((t, case["heads"], case["dim"]), gen).to(dtype), "k": _normal((t, case["kv_heads"], case["dim"]), gen).to(dtype)}
    h, v, v0, dtype = case["hidden"], case["vocab_rows"], case["vocab_start"], TYPES[case["x"]]
    w = _normal((v, h), gen, 0.02).to(dtype)
    labels = _zipf(t, gen)
    # a normalised residual stream that already leans towards the next token where the shard has it
    row = labels - v0
    mine = (row >= 0) & (row < v)
    to = w[row.clamp(0, v - 1)].float()
    lean = torch.rand(t, generator=gen, device="cuda").mul_(12) * mine
    x = _normal((t, h), gen).add_(to * (lean / (to * to).sum(1).clamp_min_(1e-6))[:, None]).to(dtype)
    state = {"case": case, "h": x, "w": w}
    tau = 1.0
    if case["op"].startswith("cross"):
        ignored = torch.rand(t, generator=gen, device="cuda") < 0.03  # padding
        state["labels"] = _int(torch.where(ignored, -100, labels), case["ids"])
        weight = (~ignored).float()
    else:
        # the teacher's best tokens, by their frequency and chance; the next token is the first, and some have fewer than all
        tau, top = case["temperature"], case["top"]
        rank = torch.arange(1, VOCAB + 1, device="cuda", dtype=torch.float32)
        score = -torch.log(rank) - torch.log(-torch.log(torch.rand((t, VOCAB), generator=gen, device="cuda").clamp_(1e-12, 1 - 1e-6)))
        score.scatter_(1, labels[:, None], 9.0)
        score, ids = torch.topk(score, top, dim=1)
        gone = torch.rand((t, top), generator=gen, device="cuda") < 0.05
        gone[:, 0] = False
        state["ids"] = _int(torch.where(gone, -1, ids), case["ids"])
        state["logits"] = (score + 10).to(dtype)
        weight = torch.ones(t, device="cuda")
    if case["op"].endswith("grad"):
        z = x.float() @ w.float().T / tau
        state["lse"] = torch.logsumexp(z, 1) + math.log(max(1, round(VOCAB / v)))  # with what the other shards have
        state["dloss"] = weight / weight.sum().clamp_min(1)
        state["sum"] = _normal((v, h), gen, 1e-4).to(TYPES[case["dw"]]) if case["accumulate"] else None
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
    if op.startswith("rotary"):
        call = e.rotary_grad if op == "rotary_grad" else e.rotary
        q, k = call(s["q"], s["k"], s["positions"], s["f"], interleaved=case["interleaved"], scale=s["scale"])
        return {"q": q, "k": k}
    v0 = case["vocab_start"]
    if op == "cross_entropy":
        loss, lse, target = e.cross_entropy(s["h"], s["w"], s["labels"], vocab_start=v0)
        return {"loss": loss, "lse": lse, "target": target}
    if op == "distill":
        loss, lse, cross = e.distill(s["h"], s["w"], s["ids"], s["logits"], temperature=case["temperature"], vocab_start=v0)
        return {"loss": loss, "lse": lse, "cross": cross}
    how = {"vocab_start": v0, "dtype": TYPES[case["dw"]], "dweight": s["sum"], "accumulate": case["accumulate"]}
    if op == "cross_entropy_grad":
        dh, dw = e.cross_entropy_grad(s["dloss"], s["h"], s["w"], s["labels"], s["lse"], **how)
    else:
        dh, dw = e.distill_grad(s["dloss"], s["h"], s["w"], s["ids"], s["logits"], s["lse"], temperature=case["temperature"], **how)
    return {"dh": dh, "dw": dw}


def _run_plain(s):
    case = s["case"]
    return {"cross_entropy": _plain_ce, "cross_entropy_grad": _plain_ce_grad, "distill": _plain_distill, "distill_grad": _plain_distill_grad,
            "rotary": _plain_rotary, "rotary_grad": _plain_rotary}[case["op"]](case, s)


def _plain_lse(z):
    most = z.amax(1)
    return most + torch.log(torch.exp(z - most[:, None]).sum(1))


def _plain_rows(ids, case):
    """Rows of the shard, and which ids are of it."""
    row = ids.long() - case["vocab_start"]
    mine = (ids >= 0) & (row >= 0) & (row < case["vocab_rows"])
    return row.clamp(0, case["vocab_rows"] - 1), mine


def _plain_ce(case, s):
    z = s["h"].float() @ s["w"].float().T
    row, mine = _plain_rows(s["labels"], case)
    lse = _plain_lse(z)
    target = z.gather(1, row[:, None])[:, 0] * mine
    return {"loss": (lse - target) * (s["labels"] >= 0), "lse": lse, "target": target}


def _plain_grads(case, s, h, w, dz):
    dh, dw = dz @ w, dz.T @ h
    if s["sum"] is None:
        return {"dh": dh.to(s["h"].dtype), "dw": dw.to(TYPES[case["dw"]])}
    s["sum"].copy_(dw + s["sum"].float())
    return {"dh": dh.to(s["h"].dtype), "dw": s["sum"]}


def _plain_ce_grad(case, s):
    h, w = s["h"].float(), s["w"].float()
    g = s["dloss"] * (s["labels"] >= 0)
    dz = torch.exp(h @ w.T - s["lse"][:, None]) * g[:, None]
    row, mine = _plain_rows(s["labels"], case)
    dz.scatter_add_(1, row[:, None], (-g * mine)[:, None])
    return _plain_grads(case, s, h, w, dz)


def _plain_teacher(case, s):
    t = s["logits"].float() / case["temperature"]
    t = torch.where(s["ids"] >= 0, t, torch.full_like(t, -math.inf))
    log_q = t - _plain_lse(t)[:, None]
    return torch.exp(log_q), torch.where(s["ids"] >= 0, log_q, torch.zeros_like(t))


def _plain_distill(case, s):
    tau = case["temperature"]
    z = s["h"].float() @ s["w"].float().T / tau
    q, log_q = _plain_teacher(case, s)
    row, mine = _plain_rows(s["ids"], case)
    lse = _plain_lse(z)
    cross = (q * mine * z.gather(1, row)).sum(1)
    return {"loss": tau * tau * ((q * log_q).sum(1) + q.sum(1) * lse - cross), "lse": lse, "cross": cross}


def _plain_distill_grad(case, s):
    tau = case["temperature"]
    h, w = s["h"].float(), s["w"].float()
    q, _ = _plain_teacher(case, s)
    g = s["dloss"] * tau
    dz = torch.exp(h @ w.T / tau - s["lse"][:, None]) * (g * q.sum(1))[:, None]
    row, mine = _plain_rows(s["ids"], case)
    dz.scatter_add_(1, row, -q * mine * g[:, None])
    return _plain_grads(case, s, h, w, dz)


def _plain_rotary(case, s):
    angle = s["positions"].double()[:, None] * s["f_gpu"]  # far positions lose their digits in 32 bits
    scale = s["scale"]
    cos, sin = (torch.cos(angle) * scale).float()[:, None], (torch.sin(angle) * scale).float()[:, None]
    if case["op"] == "rotary_grad":
        sin = -sin
    return {name: _plain_turn(case, s[name], cos, sin) for name in ("q", "k")}


def _plain_turn(case, x, cos, sin):
    rot = case["rot"]
    x32 = x.float()
    a, b = (x32[..., 0:rot:2], x32[..., 1:rot:2]) if case["interleaved"] else (x32[..., :rot // 2], x32[..., rot // 2:rot])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((a, b), -1).flatten(-2) if case["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((turned, x32[..., rot:]), -1).to(x.dtype)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    t, size = case["tokens"], SIZE[case["x"]]
    if case["op"].startswith("rotary"):
        n = t * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * n * case["dim"] * size + t * case["ids"] // 8, "flops": 3 * n * case["rot"]}
    h, v = case["hidden"], case["vocab_rows"]
    inputs = (t + v) * h * size
    per_token = case["top"] * (case["ids"] // 8 + size) if "top" in case else case["ids"] // 8
    if not case["op"].endswith("grad"):
        return {"bytes": inputs + t * (per_token + 12), "flops": 2 * t * h * v}
    dw = (2 if case["accumulate"] else 1) * v * h * SIZE[case["dw"]]
    return {"bytes": inputs + t * (per_token + 8) + t * h * size + dw, "flops": 6 * t * h * v}


# ---------------------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------------------
def _exact_turn(case, x, turn):
    """Pairs as complex numbers times ``turn`` [tokens, pairs]."""
    rot, t = case["rot"], case["tokens"]
    x = x.double()
    out = x.clone()
    pairs = x[..., :rot].reshape(t, -1, rot // 2, 2) if case["interleaved"] else x[..., :rot].reshape(t, -1, 2, rot // 2).transpose(2, 3)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
    out[..., :rot] = (turned if case["interleaved"] else turned.transpose(2, 3)).reshape(t, -1, rot)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("rotary"):
        angle = torch.outer(s["positions"].double(), s["f_gpu"])
        turn = torch.polar(torch.full_like(angle, s["scale"]), -angle if op == "rotary_grad" else angle)
        return {name: _exact_turn(case, s[name], turn) for name in ("q", "k")}
    h, w, v0 = s["h"].double(), s["w"].double(), case["vocab_start"]
    tau = case.get("temperature", 1.0)
    z = torch.einsum("th,vh->tv", h, w) / tau
    # the wanted distribution over the shard's rows, and its weight over the whole vocabulary
    want = torch.zeros_like(z)
    if "labels" in s:
        valid = s["labels"] >= 0
        mass, entropy = valid.double(), 0.0
        at = torch.nonzero(valid & (s["labels"] >= v0) & (s["labels"] < v0 + case["vocab_rows"])).flatten()
        want[at, s["labels"][at].long() - v0] = 1.0
    else:
        t = (s["logits"].double() / tau).masked_fill(s["ids"] < 0, -math.inf)
        q = torch.softmax(t, 1)
        mass, entropy = q.sum(1), torch.special.entr(q).sum(1)
        at, k = torch.nonzero((s["ids"] >= v0) & (s["ids"] < v0 + case["vocab_rows"]), as_tuple=True)
        want.index_put_((at, s["ids"][at, k].long() - v0), q[at, k], accumulate=True)
    if not op.endswith("grad"):
        lse = torch.logsumexp(z, 1)
        part = torch.linalg.vecdot(want, z)
        return {"loss": tau ** 2 * (mass * lse - part - entropy), "lse": lse, "target" if "labels" in s else "cross": part}
    dz = (mass[:, None] * torch.exp(z - s["lse"].double()[:, None]) - want) * (tau * s["dloss"].double())[:, None]
    dw = torch.einsum("tv,th->vh", dz, h)
    return {"dh": torch.einsum("tv,vh->th", dz, w), "dw": dw if s["sum"] is None else dw + s["sum"].double()}
