"""Workloads of the row operators of a language model: layer norm and its gradient, distillation from a teacher's top
alternatives and its gradient, sampling of tokens.

`run` computes them in their plain form, in elementary torch operations (32 bits; 64 where a token hangs on a comparison of
sums) with one rounding at the end, or, where `own` is true, by the calls that a user makes of the library.

Fields of a case
  op        "layernorm":  forward          "layernorm_train":  forward, then the gradients of input, weight and bias
            "distill":    loss per row     "distill_train":    loss and the gradient of the logits
            "sample":     one token per row and its log probability among what is kept
  dtype     type of what is large (layer norm: of the input and its gradient): "fp32" or "bf16"
  rows, cols
layernorm, layernorm_train
  out       type of the output and its gradient;  weights: type of weight and bias and of their gradients
  rms       root mean square only: nothing is subtracted, and there is no bias;  extra: elements between two rows of the input
distill, distill_train
  extra     elements between two rows of the logits;  top: alternatives of the teacher per row
  rest      what the teacher's alternatives leave of 1 counts as one more alternative; else they are brought to a sum of 1
  scale     reciprocal temperature, of the student and, without `rest`, of the teacher
  masked    share of the columns that are -inf;  ignored: share of the rows without a teacher
  call      distill_train: "one" (weights known beforehand: one call) or "two" (loss, then gradient)
sample
  extra     elements between two rows;  masked: share of the columns that are -inf
  temperature, top_k, top_p, min_p    for all rows (top_k 0, top_p 1, min_p 0: off), or, with `mixed`, of the rows' own:
            these in one row of four, others in the other three (greedy, plain, another nucleus)
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
NO_REST = 2.0 ** -20             # a rest of the teacher's probabilities below this is their rounding


def _layernorm(name, op, dtype, rows, cols, out=None, weights="fp32", rms=False, extra=0):
    return dict(name=name, op=op, dtype=dtype, rows=rows, cols=cols, out=out or dtype, weights=weights, rms=rms, extra=extra)


def _distill(name, op, dtype, rows, cols, top, rest, scale=1.0, extra=0, masked=0.0, ignored=0.0, call="one"):
    return dict(name=name, op=op, dtype=dtype, rows=rows, cols=cols, top=top, rest=rest, scale=scale, extra=extra, masked=masked,
                ignored=ignored, call=call)


def _sample(name, dtype, rows, cols, temperature, top_k=0, top_p=1.0, min_p=0.0, mixed=False, extra=0, masked=0.0):
    return dict(name=name, op="sample", dtype=dtype, rows=rows, cols=cols, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p,
                mixed=mixed, extra=extra, masked=masked)


def listed():
    return [
        # one decoding step of a small batch, GPT-2 width: all latency
        _layernorm("norm_decode", "layernorm", "fp32", 3, 768),
        # a training batch of 16384 tokens at 7B width, evaluated
        _layernorm("norm_batch", "layernorm", "bf16", 16384, 4096, weights="bf16", rms=True),
        # a short batch of odd length, trained: the reduction over the rows has little to read
        _layernorm("norm_train_short", "layernorm_train", "fp32", 1001, 768),
        # a training batch of 16384 tokens at 7B width
        _layernorm("norm_train_batch", "layernorm_train", "bf16", 16384, 4096, weights="bf16"),
        # a residual stream kept in 32 bits in front of bf16 products, 1.3B width
        _layernorm("norm_train_stream", "layernorm_train", "fp32", 8192, 2048, out="bf16"),
        # the loss of a validation batch against stored alternatives
        _distill("distill_eval", "distill", "bf16", 512, 50304, 20, True),
        # a training batch against a teacher's twenty best, temperature 2, weights of a mean over rows
        _distill("distill_batch", "distill_train", "bf16", 8192, 32000, 20, False, scale=0.5, ignored=0.1),
        # masked vocabulary, padding rows, rows padded to 50304; the weights come after the loss
        _distill("distill_masked", "distill_train", "fp32", 1000, 50257, 32, True, extra=47, masked=0.3, ignored=0.2, call="two"),
        # one token of one sequence, nucleus sampling
        _sample("sample_one", "fp32", 1, 50257, 0.8, top_p=0.95),
        # a serving batch whose requests have parameters of their own
        _sample("sample_mixed", "bf16", 250, 50304, 0.7, top_k=50, top_p=0.9, mixed=True),
        # a batch of rollouts, drawn from the whole distribution
        _sample("sample_rollouts", "fp32", 1024, 32000, 1.0),
        # the same with a floor relative to the likeliest token, bf16 logits, and the nucleus of what is left
        _sample("sample_floor", "bf16", 1024, 50257, 1.2, top_p=0.98, min_p=0.02, masked=0.3),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["layernorm", "layernorm_train", "distill", "distill_train", "sample", "sample"])
    dtype = rng.choice(["fp32", "bf16"])
    if op.startswith("layernorm"):
        cols = rng.choice([_log(rng, 16, 16384), 8 * _log(rng, 8, 2048)])
        rms = rng.random() < 0.3
        return dict(op=op, dtype=dtype, rows=_log(rng, 1, 30_000_000 / cols), cols=cols, out=rng.choice([dtype, dtype, "fp32", "bf16"]),
                    weights=rng.choice(["fp32", "bf16"]), rms=rms, extra=rng.choice([0, 0, 1, 64]))
    cols = rng.choice([_log(rng, 100, 160000), 64 * _log(rng, 8, 2500)])
    more = dict(op=op, dtype=dtype, cols=cols, extra=rng.choice([0, 0, 1, 64]), masked=rng.choice([0.0, 0.3]))
    if op == "sample":
        return dict(more, rows=_log(rng, 1, 30_000_000 / cols), temperature=rng.choice([0.0, 0.5, 0.8, 1.0, 1.3]), top_k=rng.choice([0, 0, 1, 40, 1000]),
                    top_p=rng.choice([1.0, 0.5, 0.9, 0.95]), min_p=rng.choice([0.0, 0.0, 0.001, 0.1]), mixed=rng.random() < 0.3)
    return dict(more, rows=_log(rng, 1, 130_000_000 / cols), top=rng.choice([1, 5, 20, 32, 64]), rest=rng.random() < 0.5, scale=rng.choice([1.0, 0.5, 1.25]),
                ignored=rng.choice([0.0, 0.2]), call=rng.choice(["one", "two"]))


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _rand(shape, gen):
    return torch.rand(shape, generator=gen, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case=case)
    {"layernorm": _prepare_layernorm, "distill": _prepare_distill, "sample": _prepare_sample}[case["op"].split("_")[0]](case, state, gen)
    if own:
        state["plan"] = _plan(case)
    return state


def _prepare_layernorm(case, state, gen):
    r, c, dtype, out, weights = case["rows"], case["cols"], DTYPES[case["dtype"]], DTYPES[case["out"]], DTYPES[case["weights"]]
    # rows of different magnitudes around means of their own, as the inner activations of a model are
    x = _randn((r, c + case["extra"]), dtype, gen)[:, :c]
    x.mul_(0.5 + 2 * _rand((r, 1), gen)).add_(_randn((r, 1), torch.float32, gen))
    state.update(x=x, weight=(1 + 0.1 * _randn(c, torch.float32, gen)).to(weights),
                 bias=None if case["rms"] else (0.1 * _randn(c, torch.float32, gen)).to(weights))
    if case["op"] == "layernorm_train":
        state["grad_out"] = _randn((r, c), out, gen).mul_(1e-3)
    if own:
        state["out"] = torch.empty((r, c), dtype=out, device="cuda")
        if case["op"] == "layernorm_train":
            state["grad_x"] = torch.empty((r, c), dtype=dtype, device="cuda")
            state["grad_weight"] = torch.empty(c, dtype=weights, device="cuda")
            state["grad_bias"] = None if case["rms"] else torch.empty(c, dtype=weights, device="cuda")


def _prepare_logits(case, gen, spread):
    """Logits, and the columns that are not masked."""
    r, c = case["rows"], case["cols"]
    x = _randn((r, c + case["extra"]), DTYPES[case["dtype"]], gen)[:, :c].mul_(spread)
    allowed = torch.arange(c, device="cuda")
    if case["masked"]:
        gone = _rand(c, gen) < case["masked"]
        gone[0] = False
        x[:, gone] = -math.inf
        allowed = torch.nonzero(~gone).reshape(-1)
    return x, allowed


def _prepare_distill(case, state, gen):
    r, top = case["rows"], case["top"]
    x, allowed = _prepare_logits(case, gen, 2.0)
    # one alternative from each of `top` parts of the columns, in any order of probability; what they leave of 1 differs by row
    n = allowed.numel()
    place = ((torch.arange(top, device="cuda") + _rand((r, top), gen)) * (n / top)).long().clamp_(max=n - 1)
    tokens = allowed[place]
    value = torch.log_softmax(2 * _randn((r, top), torch.float32, gen), 1) + torch.log1p(-0.01 - 0.3 * _rand((r, 1), gen))
    # a student that has learned something: it likes what the teacher likes
    x.scatter_(1, tokens, (value + 9 + _randn((r, top), torch.float32, gen)).to(x.dtype))
    tokens[_rand((r, top), gen) < 0.02] = -1
    if case["ignored"]:
        tokens[_rand(r, gen) < case["ignored"]] = -1
    state.update(logits=x, value=value, token=tokens)
    if case["op"] == "distill_train":
        state["weight"] = _rand(r, gen) / r
        if own:
            state["out"] = torch.empty_strided((r, case["cols"]), (case["cols"] + case["extra"], 1), dtype=x.dtype, device="cuda")


def _prepare_sample(case, state, gen):
    r = case["rows"]
    # rows between a sure model and an unsure one
    x, _ = _prepare_logits(case, gen, 2 + 2 * _rand((r, 1), gen))
    state.update(logits=x, uniform=_rand(r, gen))
    if case["mixed"]:
        kind = torch.arange(r, device="cuda") % 4
        choose = lambda *v: torch.tensor(v, device="cuda")[kind]    # noqa: E731
        state["rows_own"] = dict(temperature=choose(case["temperature"], 0.0, 1.0, 0.9), top_k=choose(case["top_k"], 0, 0, 200).int(),
                                 top_p=choose(case["top_p"], 1.0, 1.0, 0.8), min_p=choose(case["min_p"], 0.0, 0.0, 0.01))


def _plan(case):
    """The handle that a user's program keeps: workspaces and small outputs."""
    from paper_2505_00347_amd import solo
    r, c = case["rows"], case["cols"]
    if case["op"].startswith("layernorm"):
        return solo.SoloLayerNorm(r, c, eps=EPS, rms=case["rms"])
    if case["op"].startswith("distill"):
        return solo.SoloDistill(r, c, case["top"], rest=case["rest"], scale=case["scale"], teacher_scale=1.0 if case["rest"] else case["scale"])
    return solo.SoloSampler(r, c, temperature=case["temperature"], top_k=case["top_k"], top_p=case["top_p"], min_p=case["min_p"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    case, plan = state["case"], state["plan"]
    if case["op"].startswith("layernorm"):
        y = plan.forward(state["x"], state["weight"], state["bias"], state["out"])
        if case["op"] == "layernorm":
            return y
        return y, *plan.grad(state["grad_out"], state["x"], state["weight"], state["grad_x"], state["grad_weight"], state["grad_bias"])
    if case["op"] == "sample":
        return plan.sample(state["logits"], state["uniform"], **state.get("rows_own", {}))
    teacher = state["value"], state["token"]
    if case["op"] == "distill":
        return plan.forward(state["logits"], *teacher)
    if case["call"] == "one":
        return plan.forward_grad(state["logits"], *teacher, state["weight"], state["out"])
    return plan.forward(state["logits"], *teacher), plan.grad(state["logits"], *teacher, state["weight"], state["out"])


def _run_plain(state):
    return {"layernorm": _plain_layernorm, "distill": _plain_distill, "sample": _plain_sample}[state["case"]["op"].split("_")[0]](state)


def _plain_layernorm(state):
    case, x, w = state["case"], state["x"].float(), state["weight"].float()
    centred = x if case["rms"] else x - x.mean(1, keepdim=True)
    rstd = (centred.square().mean(1, keepdim=True) + EPS).rsqrt()
    xhat = centred * rstd
    y = xhat * w
    y = (y if case["rms"] else y + state["bias"].float()).to(DTYPES[case["out"]])
    if case["op"] == "layernorm":
        return y
    dy = state["grad_out"].float()
    g = dy * w
    dx = g - xhat * (g * xhat).mean(1, keepdim=True)
    if not case["rms"]:
        dx = dx - g.mean(1, keepdim=True)
    types = DTYPES[case["dtype"]], DTYPES[case["weights"]]
    return y, (dx * rstd).to(types[0]), (dy * xhat).sum(0).to(types[1]), None if case["rms"] else dy.sum(0).to(types[1])


def _plain_distill(state):
    case, token = state["case"], state["token"]
    value = state["value"].float()
    live = (token >= 0) & (token < case["cols"]) & (value > -math.inf)
    at = torch.where(live, token, 0)
    row = live.any(1, keepdim=True)
    if case["rest"]:
        log_p = torch.where(live, value, -math.inf)
    else:
        v = torch.where(live, value * case["scale"], -math.inf)
        v = v - torch.where(row, v.amax(1, keepdim=True), 0.0)
        log_p = v - v.exp().sum(1, keepdim=True).log()
    p = torch.where(live, log_p.exp(), 0.0)
    # the student's distribution; rows without a teacher hold anything
    z = torch.where(row, state["logits"].float(), 0.0) * case["scale"]
    m = z.amax(1, keepdim=True)
    d = torch.where(m > -math.inf, z - m, -math.inf)
    e = d.exp()
    s = e.sum(1, keepdim=True)
    log_q = d.gather(1, at) - s.log()
    loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1, keepdim=True)
    total, tail = p.sum(1, keepdim=True), 0.0
    if case["rest"]:
        # (1 - sum of p next to the border: in 64 bits)
        left = 1 - log_p.double().exp().sum(1, keepdim=True)
        left = torch.where(left >= NO_REST, left, 0.0).float()
        among = torch.zeros_like(e).scatter_add_(1, at, live.float()) > 0
        s_rest = torch.where(among, 0.0, e).sum(1, keepdim=True)
        loss = loss + torch.where(left > 0, left * (left.log() - (s_rest / s).log()), 0.0)
        total = total + left
        tail = torch.where(among, 0.0, torch.where(s_rest > 0, left / s_rest, 0.0))
    loss = torch.where(row, loss, 0.0).reshape(-1)
    if case["op"] == "distill":
        return loss
    grad = torch.where(s > 0, e * (total / s - tail), 0.0)
    grad = grad.scatter_add_(1, at, torch.where(s > 0, -p, 0.0))
    grad = torch.where(row, grad * (state["weight"][:, None] * case["scale"]), 0.0)
    return loss, grad.to(state["logits"].dtype)


def _plain_sample(state):
    """In 64 bits: which token it is hangs on comparisons of sums."""
    case, x = state["case"], state["logits"]
    r, c = case["rows"], case["cols"]
    whole = dict(temperature=case["temperature"], top_k=case["top_k"], top_p=case["top_p"], min_p=case["min_p"])
    own_ = state.get("rows_own") or {k: torch.full((r,), v, device="cuda") for k, v in whole.items()}
    temperature, top_k, top_p, min_p = (own_[k].double()[:, None] for k in ("temperature", "top_k", "top_p", "min_p"))
    x = x.double()
    m = x.amax(1, keepdim=True)
    w = ((x - m) / torch.where(temperature > 0, temperature, 1.0)).exp()
    w = torch.where(temperature > 0, w, (x == m).double())
    top_k = torch.where(temperature > 0, torch.where(top_k > 0, top_k, c), 1)
    # the columns in the order of the logits, ties by the lower column
    order = x.sort(dim=1, descending=True, stable=True).indices
    w = w.gather(1, order)
    first = (torch.arange(c, device="cuda")[None, :] < top_k) & (w >= min_p)
    first[:, 0] = True
    w = torch.where(first, w, 0.0)
    sums = w.cumsum(1)
    # a column stays if those before it do not have the nucleus's share yet
    before = torch.cat([torch.zeros_like(m), sums[:, :-1]], 1)
    first = first & ((top_p >= 1) | (before < top_p * sums[:, -1:]))
    first[:, 0] = True
    w = torch.where(first, w, 0.0)
    sums = w.cumsum(1)
    mass = sums[:, -1:]
    at = (sums > state["uniform"].double()[:, None] * mass).int().argmax(1, keepdim=True)
    return order.gather(1, at).reshape(-1), (w.gather(1, at) / mass).log().float().reshape(-1)


def work(case):
    size, r, c = {"fp32": 4, "bf16": 2}, case["rows"], case["cols"]
    big, op = size[case["dtype"]], case["op"]
    if op.startswith("layernorm"):
        out, weights = size[case["out"]], (1 if case["rms"] else 2) * c * size[case["weights"]]
        forward = {"bytes": r * c * (big + out) + weights, "flops": 7 * r * c}
        if op == "layernorm":
            return forward
        # each of input, output, the output's gradient and the input's gradient once
        return {"bytes": r * c * (2 * big + 2 * out) + 2 * weights, "flops": 20 * r * c}
    if op == "sample":
        return {"bytes": r * c * big + r * 16, "flops": 4 * r * c}
    live = int(r * (1 - case["ignored"]))
    teacher = r * case["top"] * 12 + 4 * r
    if op == "distill":
        return {"bytes": live * c * big + teacher, "flops": 5 * live * c}
    return {"bytes": live * c * big + r * c * big + teacher + 4 * r, "flops": 8 * live * c}


def exact(case, seed):
    if case["rows"] * case["cols"] > 300_000_000:
        return None
    state = prepare(case, seed)
    return {"layernorm": _exact_layernorm, "distill": _exact_distill, "sample": _exact_sample}[case["op"].split("_")[0]](case, state)


def _exact_layernorm(case, state):
    """From the normalised row's Jacobian: dx = rstd (g - projection of g on what the norm takes out)."""
    parts, dw, db = [], 0.0, 0.0
    w = state["weight"].double()
    for a in range(0, case["rows"], max(1, 20_000_000 // case["cols"])):
        x = state["x"][a:a + max(1, 20_000_000 // case["cols"])].double()
        n = x.shape[1]
        mean = torch.zeros_like(x[:, :1]) if case["rms"] else x.sum(1, keepdim=True) / n
        std = (((x - mean) ** 2).sum(1, keepdim=True) / n + EPS).sqrt()
        h = (x - mean) / std
        some = [h * w if case["rms"] else torch.addcmul(state["bias"].double(), h, w)]
        if case["op"] == "layernorm_train":
            dy = state["grad_out"][a:a + len(x)].double()
            g = dy * w
            shift = 0.0 if case["rms"] else g.sum(1, keepdim=True) / n
            some.append((g - shift - h * ((g * h).sum(1, keepdim=True) / n)) / std)
            dw, db = dw + (dy * h).sum(0), db + dy.sum(0)
        parts.append(some)
    whole = [torch.cat(v) for v in zip(*parts)]
    return whole[0] if case["op"] == "layernorm" else (*whole, dw, None if case["rms"] else db)


def _exact_distill(case, state):
    """Row blocks in 64 bits: Kullback-Leibler divergence of the two lists of probabilities, and the softmax's Jacobian on its slope."""
    c, scale, losses, grads = case["cols"], case["scale"], [], []
    step = max(1, 30_000_000 // c)
    for a in range(0, case["rows"], step):
        token, value = state["token"][a:a + step], state["value"][a:a + step].double()
        live = token >= 0
        has = live.any(1)
        x = torch.where(has[:, None], state["logits"][a:a + step].double(), 0.0)
        logq = torch.log_softmax(x * scale, 1)
        value = torch.where(live, value, -math.inf)
        logp = value if case["rest"] else torch.where(has[:, None], torch.log_softmax(value * scale, 1), -math.inf)
        p = logp.exp()
        at = token.clamp(min=0)
        some = torch.xlogy(p, p) - torch.where(live, p * logq.gather(1, at), 0.0)
        loss = some.sum(1)
        teacher = torch.zeros_like(logq).scatter_add_(1, at, torch.where(live, p, 0.0))
        if case["rest"]:
            left = 1 - p.sum(1)
            left = torch.where(left >= NO_REST, left, 0.0)
            outside = torch.ones_like(logq, dtype=torch.bool)
            rows = torch.arange(len(at), device=at.device)[:, None].expand_as(at)
            outside[rows[live], at[live]] = False
            logq_out = torch.where(outside, logq, -math.inf)
            log_tail = torch.logsumexp(logq_out, 1)
            loss = loss + torch.where(left > 0, torch.xlogy(left, left) - left * log_tail, 0.0)
            # the rest of the teacher, spread as the student spreads its own
            teacher = teacher + torch.where(outside, left[:, None] * (logq_out - log_tail[:, None]).exp(), 0.0)
        losses.append(torch.where(has, loss, 0.0))
        if case["op"] == "distill_train":
            g = logq.exp() * teacher.sum(1, keepdim=True) - teacher
            grads.append(torch.where(has[:, None], g * (scale * state["weight"][a:a + step].double())[:, None], 0.0).cpu())
    loss = torch.cat(losses)
    return loss if case["op"] == "distill" else (loss.cpu(), torch.cat(grads))


def _exact_sample(case, state):
    """Log probability of the token: of the sorted columns a prefix is kept; the rows one by one where they are few, else none."""
    if case["rows"] > 1024:
        return None
    found = []
    for r in range(case["rows"]):
        own_ = state.get("rows_own")
        # (as the call takes them: in 32 bits)
        t, k, p, m = (float(own_[n][r] if own_ else torch.tensor(float(case[n]))) for n in ("temperature", "top_k", "top_p", "min_p"))
        x = state["logits"][r].double()
        if t <= 0:
            found.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            continue
        v = x.sort(descending=True).values
        q = ((v - v[0]) / t).exp()
        q[int(k) if k > 0 else case["cols"]:] = 0
        q[1:][q[1:] < m] = 0
        q = q / q.sum()
        if p < 1:
            gone = q.cumsum(0) - q >= p
            gone[0] = False
            q[gone] = 0
            q = q / q.sum()
        found.append(q[(q.cumsum(0) > state["uniform"][r].double()).int().argmax()].log())
    return [None, torch.stack(found)]
