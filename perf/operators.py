"""Workloads of the operators around the optimizer step: the gradients' global norm and clipping, the
embedding and its gradient, the log probabilities of given tokens and their gradient.

`run` computes them in their plain form, in elementary torch operations in 32 bits with one rounding at the end,
or, where `own` is true, by the calls that a user makes of the library.

Fields of a case
  op        "norm":      norm of each tensor, of all, and the step's gradient scale
            "clip":      the same, and the clipped gradients in buffers of their own
            "lookup":    rows of an embedding table, scaled
            "embgrad":   the table's gradient (every row of it)
            "logprob":   log probability of a target per row, entropy, rank, `top` alternatives
            "lossgrad":  log probability, entropy and the gradient of their weighted sum
  dtype     type of what is large: "fp32" or "bf16"
norm, clip
  layout    "model": the tensors of a transformer with these `vocab`, `hidden`, `ff`, `layers`; `gated`: three
            MLP matrices, four attention ones and a head of its own, as LLaMA has them, else as GPT-2 has them.
            "split": `count` tensors of uneven sizes, `n` elements in all, one right behind the other
lookup, embgrad
  vocab, dim, n   rows and columns of the table, tokens;  tokens: "zipf" (a few are frequent) or "uniform"; one in 50
            is padding (-1);  out: type of the looked-up rows, or of the table's gradient;  scale
logprob, lossgrad
  rows, cols, stride    logits and the distance of two rows in elements;  scale: reciprocal temperature
  top       alternatives;  masked: share of the columns that are -inf;  ignored: share of the rows without a target
  call      lossgrad: "one" (weights known beforehand: one call) or "two" (forward, then gradient)
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
MAX_NORM = 1.0
LARGEST_NORM = 7_000_000_000     # bytes of the drawn gradients


def _norm(name, op, dtype, **sizes):
    return dict(name=name, op=op, dtype=dtype, **sizes)


def _model(vocab, hidden, ff, layers, gated):
    return dict(layout="model", vocab=vocab, hidden=hidden, ff=ff, layers=layers, gated=gated)


def listed():
    return [
        # one norm vector's gradient by itself: the smallest call, all latency
        _norm("norm_vector", "norm", "bf16", layout="split", n=4096, count=1),
        # LLaMA-7B shapes, 291 tensors: the norm before a step that takes the scale from device memory
        _norm("norm_llama7b", "norm", "bf16", **_model(32000, 4096, 11008, 32, True)),
        # GPT-2-125M shapes, 99 tensors, fp32 gradients, clipped for an optimizer that takes no scale
        _norm("clip_gpt2", "clip", "fp32", **_model(50257, 768, 3072, 12, False)),
        # 1.3B shapes, bf16 gradients, clipped
        _norm("clip_1p3b", "clip", "bf16", **_model(50304, 2048, 8192, 24, False)),
        # the embedding of one decoding step of a small batch
        dict(name="lookup_decode", op="lookup", dtype="fp32", vocab=50257, dim=768, n=3, tokens="zipf", out="fp32", scale=1.0),
        # the embedding of a training batch of 16384 tokens, 7B shapes
        dict(name="lookup_batch", op="lookup", dtype="bf16", vocab=32000, dim=4096, n=16384, tokens="zipf", out="bf16", scale=64.0),
        # the gradient of a short sequence: nearly all rows of the table are zero
        dict(name="embgrad_short", op="embgrad", dtype="fp32", vocab=50257, dim=768, n=96, tokens="zipf", out="fp32", scale=1.0),
        # the gradient of a training batch, 7B shapes: frequent tokens have hundreds of rows to add
        dict(name="embgrad_batch", op="embgrad", dtype="bf16", vocab=32000, dim=4096, n=16384, tokens="zipf", out="bf16", scale=64.0),
        # one decoded token of one sequence with five alternatives
        dict(name="logprob_decode", op="logprob", dtype="fp32", rows=1, cols=50257, stride=50257, scale=1.0, top=5, masked=0.0, ignored=0.0),
        # a prompt of 4096 tokens scored, twenty alternatives each, temperature 0.8
        dict(name="logprob_prompt", op="logprob", dtype="bf16", rows=4096, cols=50304, stride=50304, scale=1.25, top=20, masked=0.0, ignored=0.0),
        # the loss of a training batch and its gradient in one call
        dict(name="loss_batch", op="lossgrad", dtype="bf16", rows=8192, cols=32000, stride=32000, scale=1.0, masked=0.0, ignored=0.1, call="one"),
        # a policy-gradient batch: entropy bonus, masked vocabulary, padding rows, rows padded to 50304; the weights come after the forward pass
        dict(name="loss_policy", op="lossgrad", dtype="fp32", rows=1000, cols=50257, stride=50304, scale=1.25, masked=0.3, ignored=0.2, call="two"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "clip", "lookup", "embgrad", "logprob", "lossgrad"])
    dtype = rng.choice(["fp32", "bf16"])
    if op in ("norm", "clip"):
        if rng.random() < 0.5:
            n = _log(rng, 1000, 1_000_000_000)
            return dict(op=op, dtype=dtype, layout="split", n=n, count=min(n, _log(rng, 1, 2000)))
        hidden = rng.choice([256, 768, 1000, 2048])
        return dict(op=op, dtype=dtype, **_model(_log(rng, 1000, 60000), hidden, _log(rng, hidden, 4 * hidden), rng.randint(1, 24), rng.random() < 0.5))
    if op in ("lookup", "embgrad"):
        vocab, dim = _log(rng, 100, 60000), rng.choice([_log(rng, 16, 4096), 8 * _log(rng, 8, 512)])
        return dict(op=op, dtype=dtype, vocab=vocab, dim=dim, n=_log(rng, 1, 40000), tokens=rng.choice(["zipf", "uniform"]),
                    out=rng.choice(["fp32", "bf16"]), scale=rng.choice([1.0, math.sqrt(dim)]))
    cols = rng.choice([_log(rng, 100, 160000), 64 * _log(rng, 8, 2500)])
    rows = _log(rng, 1, 400_000_000 / cols)
    more = dict(op=op, dtype=dtype, rows=rows, cols=cols, stride=cols + rng.choice([0, 0, 1, 64]), scale=rng.choice([1.0, 1.25]),
                masked=rng.choice([0.0, 0.3]), ignored=rng.choice([0.0, 0.2]))
    return dict(more, top=rng.choice([0, 1, 5, 20])) if op == "logprob" else dict(more, call=rng.choice(["one", "two"]))


def _sizes(case):
    if case["layout"] == "model":
        v, h, f = case["vocab"], case["hidden"], case["ff"]
        layer = [h, h * h, h * h, h * h, h * h, h, h * f, h * f, h * f] if case["gated"] else [h, h, 3 * h * h, h * h, h, h, h * f, h * f]
        return [v * h] + case["layers"] * layer + ([h, v * h] if case["gated"] else [h, h])
    weight = [1 + (k * 2654435761 + case["n"]) % 997 for k in range(case["count"])]
    spare = case["n"] - case["count"]
    ends = [spare * sum_ // sum(weight) for sum_ in _running(weight)]
    return [1 + b - a for a, b in zip([0] + ends, ends)]


def _running(values):
    total = 0
    return [total := total + v for v in values]


def _places(case):
    """Where the tensors begin in one buffer, and its length: tensors of a model lie as an allocator aligns them."""
    sizes = _sizes(case)
    room = [-(-s // 128) * 128 for s in sizes] if case["layout"] == "model" else sizes
    ends = _running(room)
    return [0] + ends[:-1], sizes, ends[-1]


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, op = DTYPES[case["dtype"]], case["op"]
    state = dict(case=case)
    if op in ("norm", "clip"):
        begin, sizes, length = _places(case)
        flat = _randn(length, dtype, gen).mul_(1e-3)
        if case["layout"] == "model":      # nothing between the tensors
            for b, s, e in zip(begin, sizes, begin[1:] + [length]):
                flat[b + s:e] = 0
        state.update(flat=flat, grads=[flat[b:b + s] for b, s in zip(begin, sizes)])
        # the reciprocal of a loss scale, as a mixed-precision loop keeps it on the GPU
        state["unscale"] = torch.full((1,), 0.5 + 0.5 * (seed % 2), device="cuda")
        if op == "clip" and own:
            state["out"] = torch.zeros_like(flat)
    elif op in ("lookup", "embgrad"):
        v, d, n = case["vocab"], case["dim"], case["n"]
        u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * math.log(v + 1)) - 1).long() if case["tokens"] == "zipf" else (u * v).long()
        ids = ids.clamp_(0, v - 1)
        ids[torch.rand(n, generator=gen, device="cuda") < 0.02] = -1
        state["tokens"] = ids
        if op == "lookup":
            state["table"] = _randn((v, d), dtype, gen).mul_(0.02)
        else:
            state["grad_out"] = _randn((n, d), dtype, gen).mul_(1e-3)
        if own:
            state["out"] = torch.empty((n, d) if op == "lookup" else (v, d), dtype=DTYPES[case["out"]], device="cuda")
    else:
        r, c = case["rows"], case["cols"]
        x = _randn((r, case["stride"]), dtype, gen).mul_(3.0)[:, :c]
        t = torch.randint(0, c, (r,), generator=gen, device="cuda")
        if case["masked"]:
            gone = torch.rand(c, generator=gen, device="cuda") < case["masked"]
            x[:, gone] = -math.inf
            allowed = torch.nonzero(~gone).reshape(-1)
            if allowed.numel():
                t = allowed[t % allowed.numel()]
        if case["ignored"]:
            t[torch.rand(r, generator=gen, device="cuda") < case["ignored"]] = -100
        state.update(logits=x, targets=t)
        if op == "lossgrad":
            state["weight"] = -torch.rand(r, generator=gen, device="cuda") / r
            state["entropy_weight"] = torch.full((r,), 0.01 / r, device="cuda") if case["call"] == "two" else None
            if own:
                state["out"] = torch.empty_strided((r, c), (case["stride"], 1), dtype=dtype, device="cuda")
    if own:
        state["plan"] = _plan(case, state)
    return state


def _plan(case, state):
    """The handle that a user's program keeps: tables, workspaces and small outputs."""
    from paper_2505_00347_amd import solo
    if case["op"] == "norm":
        return solo.SoloGradNorm(state["grads"])
    if case["op"] == "clip":
        begin, sizes, _ = _places(case)
        return solo.SoloGradNorm(state["grads"], [state["out"][b:b + s] for b, s in zip(begin, sizes)])
    if case["op"] in ("lookup", "embgrad"):
        return solo.SoloEmbedding(case["vocab"], case["dim"], case["n"], scale=case["scale"])
    return solo.SoloLogprob(case["rows"], case["cols"], top=case.get("top", 0), rank=case["op"] == "logprob", scale=case["scale"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    op, plan = state["case"]["op"], state["plan"]
    if op == "norm":
        return plan.norm(MAX_NORM, state["unscale"])
    if op == "clip":
        return (*plan.clip(MAX_NORM, state["unscale"]), state["out"])
    if op == "lookup":
        return plan.lookup(state["table"], state["tokens"], state["out"])
    if op == "embgrad":
        return plan.grad(state["grad_out"], state["tokens"], state["out"])
    if op == "logprob":
        return plan.forward(state["logits"], state["targets"])
    if state["case"]["call"] == "one":
        return plan.forward_grad(state["logits"], state["targets"], state["weight"], state["entropy_weight"], state["out"])
    logprob, entropy = plan.forward(state["logits"], state["targets"])[:2]
    return logprob, entropy, plan.grad(state["logits"], state["targets"], state["weight"], state["entropy_weight"], state["out"])


def _run_plain(state):
    return {"norm": _plain_norm, "clip": _plain_norm, "lookup": _plain_lookup, "embgrad": _plain_embgrad,
            "logprob": _plain_logprob, "lossgrad": _plain_lossgrad}[state["case"]["op"]](state)


def _plain_norm(state):
    u = state["unscale"]
    if len(state["grads"]) == 1:
        square = state["flat"].float().square().sum().reshape(1)
    else:
        begin, sizes, length = _places(state["case"])
        room = [b - a for a, b in zip(begin, begin[1:] + [length])]
        square = torch.stack([s.sum() for s in state["flat"].float().square().split(room)])
    norm = square.sum().sqrt().reshape(1) * u.abs()
    scale = torch.where(torch.isfinite(norm), u * torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm)), torch.zeros_like(norm))
    result = norm, scale, square.sqrt() * u.abs()
    if state["case"]["op"] == "norm":
        return result
    clipped = torch.where(torch.isfinite(norm), state["flat"].float() * scale, torch.zeros_like(norm))
    return (*result, clipped.to(state["flat"].dtype))


def _plain_lookup(state):
    ids, table = state["tokens"], state["table"]
    known = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(known, ids, 0)].float() * state["case"]["scale"]
    return torch.where(known[:, None], rows, 0.0).to(DTYPES[state["case"]["out"]])


def _plain_embgrad(state):
    case, ids = state["case"], state["tokens"]
    known = (ids >= 0) & (ids < case["vocab"])
    g = torch.where(known[:, None], state["grad_out"].float(), 0.0)
    sums = torch.zeros((case["vocab"], case["dim"]), device="cuda").index_add_(0, torch.where(known, ids, 0), g)
    return (sums * case["scale"]).to(DTYPES[case["out"]])


def _softmax(state):
    """Logits and targets with nothing in the rows without a target, the maxima's distances' exponentials, their sum, and the rows that count."""
    t = state["targets"]
    row = (t >= 0) & (t < state["case"]["cols"])
    x = torch.where(row[:, None], state["logits"].float(), 0.0)
    z = x * state["case"]["scale"]
    m = z.amax(1, keepdim=True)
    z = torch.where(m > -math.inf, z - m, -math.inf)
    e = z.exp()
    return x, z, e, e.sum(1, keepdim=True), torch.where(row, t, 0)[:, None], row


def _logprob_entropy(z, e, s, t, row):
    logprob = (z.gather(1, t) - s.log()).reshape(-1)
    empty = s.reshape(-1) == 0
    logprob = torch.where(empty, -math.inf, logprob)
    entropy = (s.log() - torch.where(e > 0, e * z, 0.0).sum(1, keepdim=True) / s).reshape(-1)
    return torch.where(row, logprob, 0.0), torch.where(row & ~empty, entropy, 0.0)


def _plain_logprob(state):
    case = state["case"]
    x, z, e, s, t, row = _softmax(state)
    logprob, entropy = _logprob_entropy(z, e, s, t, row)
    rank = torch.where(row, (x > x.gather(1, t)).sum(1), -1).to(torch.int32)
    if not case["top"]:
        return logprob, entropy, rank
    # a whole number for each logit, in the logits' order, that no other column of the row has: ties go to the lowest column
    bits = (x + 0.0).view(torch.int32)
    order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long()
    key = order * (1 << 32) + (case["cols"] - torch.arange(case["cols"], device="cuda"))
    k = min(case["top"], case["cols"])
    column = key.topk(k, dim=1).indices
    value = torch.where(s > 0, z.gather(1, column) - s.log(), -math.inf)
    return (logprob, entropy, rank, torch.where(row[:, None], value, -math.inf), torch.where(row[:, None], column, -1).to(torch.int32))


def _plain_lossgrad(state):
    x, z, e, s, t, row = _softmax(state)
    logprob, entropy = _logprob_entropy(z, e, s, t, row)
    p = torch.where(s > 0, e / s, 0.0)
    grad = -p * state["weight"][:, None]
    if state["entropy_weight"] is not None:
        inner = torch.where(p > 0, z - s.log() + entropy[:, None], 0.0)
        grad = grad - p * inner * state["entropy_weight"][:, None]
    grad = grad.scatter_add_(1, t, state["weight"][:, None] * (s > 0))
    grad = torch.where(row[:, None], grad * state["case"]["scale"], 0.0)
    return logprob, entropy, grad.to(state["logits"].dtype)


def work(case):
    size, op = {"fp32": 4, "bf16": 2}, case["op"]
    big = size[case["dtype"]]
    if op in ("norm", "clip"):
        n = sum(_sizes(case))
        return {"bytes": n * big * (2 if op == "clip" else 1) + 4 * len(_sizes(case)), "flops": (3 if op == "clip" else 2) * n}
    if op == "lookup":
        n, d = case["n"], case["dim"]
        return {"bytes": min(n, case["vocab"]) * d * big + n * d * size[case["out"]] + 8 * n, "flops": n * d}
    if op == "embgrad":
        n, d = case["n"], case["dim"]
        return {"bytes": n * d * big + case["vocab"] * d * size[case["out"]] + 8 * n, "flops": n * d}
    r, c = case["rows"], case["cols"]
    live = int(r * (1 - case["ignored"]))
    if op == "logprob":
        return {"bytes": live * c * big + r * (8 + 12 + 8 * case["top"]), "flops": 6 * live * c}
    return {"bytes": live * c * big + r * c * big + r * 20, "flops": 10 * live * c}


def exact(case, seed):
    state = prepare(case, seed)
    return {"norm": _exact_norm, "clip": _exact_norm, "lookup": _exact_lookup, "embgrad": _exact_embgrad,
            "logprob": _exact_rows, "lossgrad": _exact_rows}[case["op"]](case, state)


def _exact_norm(case, state):
    u = float(state["unscale"])
    square = torch.zeros(len(state["grads"]), dtype=torch.float64, device="cuda")
    for k, g in enumerate(state["grads"]):
        for piece in g.split(1 << 28):
            d = piece.double()
            square[k] += torch.dot(d, d)
    norm = math.sqrt(float(square.sum())) * abs(u)
    scale = u * min(1.0, MAX_NORM / norm)
    result = [torch.tensor([norm], dtype=torch.float64), torch.tensor([scale], dtype=torch.float64), square.sqrt() * abs(u)]
    return result + [state["flat"].double() * scale] if case["op"] == "clip" else result


def _exact_lookup(case, state):
    ids = state["tokens"]
    out = torch.zeros((case["n"], case["dim"]), dtype=torch.float64, device="cuda")
    at = torch.nonzero(ids >= 0).reshape(-1)
    out[at] = state["table"].double()[ids[at]] * case["scale"]
    return out


def _exact_embgrad(case, state):
    ids = state["tokens"]
    order = ids.argsort(stable=True)
    ids, sums = ids[order], torch.zeros((case["vocab"], case["dim"]), dtype=torch.float64, device="cuda")
    values, counts = ids.unique_consecutive(return_counts=True)
    end = 0
    for v, n in zip(values.tolist(), counts.tolist()):
        if v >= 0:
            sums[v] = state["grad_out"][order[end:end + n]].double().sum(0)
        end += n
    return sums * case["scale"]


def _exact_rows(case, state):
    """Row blocks in 64 bits: log-softmax by its definition, and the gradient of weight * logprob + entropy_weight * entropy."""
    parts = []
    step = max(1, 50_000_000 // case["cols"])
    for a in range(0, case["rows"], step):
        x, t = state["logits"][a:a + step].double() * case["scale"], state["targets"][a:a + step]
        row = t >= 0
        logp = x - torch.logsumexp(x, 1, keepdim=True)
        p = logp.exp()
        plogp = torch.xlogy(p, p)
        h = -plogp.sum(1)
        lp = logp[torch.arange(len(t), device="cuda"), t.clamp(min=0)]
        some = [torch.where(row, lp, 0.0), torch.where(row, h, 0.0)]
        if case["op"] == "logprob":
            if case["top"]:
                some.append(torch.where(row[:, None], logp.topk(min(case["top"], case["cols"]), dim=1).values, -math.inf))
        else:
            w = state["weight"][a:a + step].double()[:, None]
            g = -w * p
            g[torch.arange(len(t), device="cuda"), t.clamp(min=0)] += w.reshape(-1)
            if state["entropy_weight"] is not None:
                g -= state["entropy_weight"][a:a + step].double()[:, None] * (plogp + p * h[:, None])
            some.append(torch.where(row[:, None], g * case["scale"], 0.0))
        parts.append([v.cpu() for v in some] if case["op"] == "lossgrad" else some)
    whole = [torch.cat(v) for v in zip(*parts)]
    if case["op"] == "lossgrad":
        return whole
    return whole[:2] + [None] + (whole[2:] + [None] if case["top"] else [])
