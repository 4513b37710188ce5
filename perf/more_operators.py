"""Routing, norms, log probabilities and distillation, over the range their users run.

The layer shapes are those of the models the paper evaluates (a Mixtral-8x7B-, a Qwen2-57B-A14B- and a
Qwen1.5-MoE-A2.7B-shaped layer); vocabularies and `draw`'s shapes are generic, odd ones too.

Operators (`case["op"]`):
  route       logits -> the chosen experts, their weights and the tables of rows grouped by expert
  route_grad  the weights' gradient -> the logits' gradient
  norm        root-mean-square norm after the residual's addition, as it is or in 8 bits with a scale for each row
  norm_grad   its input gradient (with that of the residual stream) and its weight gradient
  logprobs    log probabilities of given tokens, entropy, and the most likely alternatives
  distill     KL to a teacher's top log probabilities and cross entropy of labels; with grad, the logits' gradient too
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _route(name, op, T, E, k, score="softmax", norm=True, bias=False, groups=1, top_groups=1, best=1, scale=1.0, dtype="f32", pad=0.0):
    """best: the scores of a group that its own is the sum of; pad: the part of the batch that is padding."""
    c = dict(op=op, T=T, E=E, k=k, score=score, norm=norm, bias=bias, groups=groups, top_groups=top_groups, best=best, scale=scale,
             dtype=dtype, pad=pad)
    return dict(c, name=name) if name else c


def _norm(name, op, T, d, dtype="bf16", residual=True, out="same"):
    """out: "same" (the input's type) or "int8"; norm_grad: residual says that the residual stream has a gradient of its own."""
    c = dict(op=op, T=T, d=d, dtype=dtype, residual=residual, out=out)
    return dict(c, name=name) if name else c


def _logprobs(name, T, V, top, dtype="bf16", temperature=1.0):
    c = dict(op="logprobs", T=T, V=V, top=top, dtype=dtype, temperature=temperature)
    return dict(c, name=name) if name else c


def _distill(name, T, V, top, dtype="bf16", temperature=1.0, tail=False, ce=0.0, grad=True, pad=0.0):
    c = dict(op="distill", T=T, V=V, top=top, dtype=dtype, temperature=temperature, tail=tail, ce=ce, grad=grad, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's decode step through the routing of a layer with 64 experts: all latency
        _route("route_qwen2_T1", "route", 1, 64, 8, norm=False),
        # a long prompt where experts are chosen by balanced scores out of the best groups, with padding behind it
        _route("route_groups_T8191", "route", 8191, 256, 8, "sigmoid", bias=True, groups=8, top_groups=4, best=2, scale=2.5, pad=0.1),
        # a training batch's gradient back to the router
        _route("route_grad_qwen15", "route_grad", 4096, 60, 4, norm=False),
        # a server's step in front of 8-bit experts
        _norm("norm_int8_qwen2_T64", "norm", 64, 3584, out="int8"),
        # a long prompt's norm between a layer's parts
        _norm("norm_mixtral_T8192", "norm", 8192, 4096),
        # the backward of a training batch
        _norm("norm_grad_qwen15", "norm_grad", 4096 + 37, 2048),
        # one user's step that answers with alternatives
        _logprobs("logprobs_T1", 1, 131072, 20),
        # a server's batch, sampled at a temperature, logits in full precision
        _logprobs("logprobs_T64_f32", 64, 100003, 64, dtype="f32", temperature=0.7),
        # scoring a long prompt, and a teacher's pass over training text
        _logprobs("logprobs_prompt", 4096, 131072, 32),
        # an evaluation of a small batch
        _distill("distill_eval_T48", 48, 131072, 32, grad=False),
        # the recovery objective with labels, what the list leaves out as one more class, padded rows
        _distill("distill_tail_f32", 1021, 50001, 100, dtype="f32", temperature=2.0, tail=True, ce=0.5, pad=0.2),
        # a training step on a teacher's top log probabilities
        _distill("distill_T4096", 4096, 131072, 64),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["route", "route_grad", "norm", "norm_grad", "logprobs", "distill", "distill"])
    dtype = "f32" if rng.random() < 0.35 else "bf16"
    if op.startswith("route"):
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * max(2, log_int(2, 256) // groups)
        top_groups = rng.randint(1, groups)
        k = min(16, log_int(1, 16), E // groups * top_groups)
        score = rng.choice(["softmax", "sigmoid"])
        return _route("", op, log_int(1, 32768), E, k, score, rng.random() < 0.5, rng.random() < 0.5, groups, top_groups, rng.choice([1, 2]),
                      rng.choice([1.0, 2.5]), rng.choice(["f32", "f32", "bf16"]), rng.choice([0.0, 0.0, 0.3]))
    odd = rng.random() < 0.4
    if op.startswith("norm"):
        d = rng.choice([2048, 3584, 4096]) if rng.random() < 0.4 else log_int(33, 12000)
        return _norm("", op, log_int(1, 32768 if d < 5000 else 8192), d | 1 if odd and d not in (2048, 3584, 4096) else d, dtype, rng.random() < 0.6,
                     "int8" if op == "norm" and rng.random() < 0.5 else "same")
    V = log_int(1000, 250000)
    V = V | 1 if odd else V // 8 * 8
    T, top = min(log_int(1, 4096), (4096 * 131072) // (V * (2 if dtype == "f32" else 1))), log_int(1, 128)
    temperature = rng.choice([1.0, 1.0, 0.7, 2.0])
    if op == "logprobs":
        return _logprobs("", T, V, rng.choice([0, top]), dtype, temperature)
    return _distill("", T, V, top, dtype, temperature, rng.random() < 0.4, rng.choice([0.0, 0.5]), rng.random() < 0.75, rng.choice([0.0, 0.3]))


# ---- inputs -----------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1234567 + seed)
    return g


def _matrix(g, rows, cols, std, dtype):
    """rows x cols whose rows start on 16-byte boundaries: a view of wider rows where they must."""
    unit = 16 // dtype.itemsize
    return torch.empty((rows, -(-cols // unit) * unit), dtype=dtype, device="cuda").normal_(0.0, std, generator=g)[:, :cols]


def _route_inputs(c, g):
    T, E = c["T"], c["E"]
    # popular experts have larger logits
    logits = _matrix(g, T, E, 1.0, torch.float32)
    logits += torch.empty(E, device="cuda").normal_(0.0, 0.5, generator=g)
    logits[T - int(c["pad"] * T):] = -math.inf  # padding goes nowhere
    inp = dict(logits=logits if c["dtype"] == "f32" else _as(logits, torch.bfloat16), bias=None)
    if c["bias"]:
        inp["bias"] = torch.empty(E, device="cuda").normal_(0.0, 0.1, generator=g)
    if c["op"] == "route_grad":
        inp["dw"] = torch.empty((T, c["k"]), device="cuda").normal_(0.0, 1e-2, generator=g)
        inp["ids"] = _choose(inp["logits"], inp["bias"], c)
    return inp


def _as(t, dtype):
    """t in another type, rows on 16-byte boundaries."""
    unit = 16 // dtype.itemsize
    out = torch.zeros((t.shape[0], -(-t.shape[1] // unit) * unit), dtype=dtype, device="cuda")
    out[:, :t.shape[1]] = t
    return out[:, :t.shape[1]]


def _norm_inputs(c, g):
    td = TYPES[c["dtype"]]
    inp = dict(w=torch.empty(c["d"], device="cuda").normal_(1.0, 0.2, generator=g).to(td), x=_matrix(g, c["T"], c["d"], 1.0, td))
    # a few large channels, as hidden states have them
    inp["x"][:, torch.randint(0, c["d"], (max(1, c["d"] // 200),), generator=g, device="cuda")] *= 8.0
    if c["op"] == "norm":
        inp["residual"] = _matrix(g, c["T"], c["d"], 2.0, td) if c["residual"] else None
    else:
        inp["dy"] = _matrix(g, c["T"], c["d"], 1e-2, td)
        inp["dr"] = _matrix(g, c["T"], c["d"], 1e-2, td) if c["residual"] else None
        inp["rstd"] = torch.rsqrt(inp["x"].float().square().mean(1) + EPS)
    return inp


def _vocabulary_logits(g, T, V, dtype):
    """Most tokens unlikely, a few dozen of each row likely, the same ones for teacher and student."""
    logits = _matrix(g, T, V, 1.5, dtype)
    likely = torch.arange(48, device="cuda") * (V // 48) + torch.randint(0, V // 48, (T, 48), generator=g, device="cuda")
    lift = torch.empty((T, 48), device="cuda").exponential_(0.5, generator=g) + 4.0
    logits.scatter_(1, likely, (logits.gather(1, likely).float() + lift).to(dtype))
    return logits, likely


def _vocabulary_inputs(c, g):
    T, V, td = c["T"], c["V"], TYPES[c["dtype"]]
    logits, likely = _vocabulary_logits(g, T, V, td)
    tokens = likely.gather(1, torch.randint(0, 48, (T, 1), generator=g, device="cuda")).squeeze(1).int()
    inp = dict(logits=logits)
    if c["op"] == "logprobs":
        return dict(inp, tokens=tokens)
    # the teacher differs by some noise on the likely tokens, the others' are its own
    t = (logits.float() + 0.3).scatter_(1, likely, logits.gather(1, likely).float() + torch.empty((T, 48), device="cuda").normal_(0.0, 1.0, generator=g))
    t /= c["temperature"]
    values, ids = t.topk(c["top"], 1)
    inp.update(ids=ids.int(), lp=values - t.logsumexp(1, keepdim=True), labels=None, scale=torch.full((T,), 1.0 / T, device="cuda"))
    if c["ce"]:
        inp["labels"] = tokens
    inp["scale"][T - int(c["pad"] * T):] = 0.0  # padding has no loss
    return inp


def prepare(case, seed):
    g = _generator(seed)
    inputs = _route_inputs if case["op"].startswith("route") else _norm_inputs if case["op"].startswith("norm") else _vocabulary_inputs
    st = dict(inputs(case, g), case=case)
    if not own:
        return st
    from paper_2606_27866_amd import flexmoe as fm  # what a user's program keeps: the handle with its workspace
    c = case
    if c["op"].startswith("route"):
        st["handle"] = fm.Router(c["E"], c["k"], c["T"], score=c["score"], normalize=c["norm"], scale=c["scale"], groups=c["groups"],
                                 top_groups=c["top_groups"], group_best=c["best"])
    elif c["op"].startswith("norm"):
        st["handle"] = fm.RMSNorm(st["w"], c["T"], eps=EPS)
    elif c["op"] == "logprobs":
        st["handle"] = fm.TokenLogprobs(c["V"], c["T"], top=c["top"], temperature=c["temperature"])
    else:
        st["handle"] = fm.Distillation(c["V"], c["top"], c["T"], temperature=c["temperature"], tail=c["tail"], ce_weight=c["ce"])
    return st


def run(state):
    if own:
        return _run_own(state)
    return PLAIN[state["case"]["op"]](state, state["case"])


def _run_own(s):
    c, h = s["case"], s["handle"]
    if c["op"] == "route":
        return h.route(s["logits"], s["bias"])._asdict()
    if c["op"] == "route_grad":
        return h.backward(s["logits"], s["ids"], s["dw"])
    if c["op"] == "norm":
        if c["out"] == "int8":
            q, scale, r = h.quantized(s["x"], s["residual"])
            return {"y": _values(q, scale), "scale": scale, "r": r}
        y, r, rstd = h.forward(s["x"], s["residual"])
        return {"y": y, "rstd": rstd, "r": r}
    if c["op"] == "norm_grad":
        dx, dw = h.backward(s["dy"], s["x"], s["rstd"], dr=s["dr"])
        return {"dx": dx, "dw": dw}
    if c["op"] == "logprobs":
        return h(s["logits"], s["tokens"])._asdict()
    if c["grad"]:
        kl, ce, dlogits = h.gradient(s["logits"], s["ids"], s["lp"], s["labels"], row_scale=s["scale"])
        return {"kl": kl, "ce": ce, "dlogits": dlogits}
    kl, ce = h.forward(s["logits"], s["ids"], s["lp"], s["labels"], row_scale=s["scale"])
    return {"kl": kl, "ce": ce}


# ---- the plain forms --------------------------------------------------------
def _choose(logits, bias, c):
    """Ids [T, k] in order of their scores, ties to the lowest, -1 where no expert is left; in 64 bits, as scores next to each other need."""
    x = logits.double()
    s = torch.sigmoid(x) if c["score"] == "sigmoid" else _softmax(x)
    score = s if bias is None else s + bias.double()
    score = torch.where(x == -math.inf, -math.inf, score)
    if c["groups"] > 1:
        by_group = score.view(len(score), c["groups"], -1)
        best = by_group.sort(dim=2, descending=True).values[:, :, :c["best"]]
        group = torch.where(best[:, :, 0] == -math.inf, -math.inf, torch.where(best == -math.inf, 0.0, best).sum(2))
        kept = group.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        out = torch.ones_like(group, dtype=torch.bool).scatter_(1, kept, False)
        score = torch.where(out.unsqueeze(2), -math.inf, by_group).view(score.shape)
    top = score.sort(dim=1, descending=True, stable=True)
    return torch.where(top.values[:, :c["k"]] == -math.inf, -1, top.indices[:, :c["k"]]).int()


def _softmax(x):
    top = x.amax(1, keepdim=True)
    z = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    return z / z.sum(1, keepdim=True).clamp(min=1e-300 if x.dtype == torch.float64 else 1e-37)


def _chosen_scores(logits, ids, c):
    """Scores of all experts, those of the chosen (0 where none is) and their sum."""
    x = logits.float()
    s = torch.sigmoid(x) if c["score"] == "sigmoid" else _softmax(x)
    of = torch.where(ids >= 0, s.gather(1, ids.clamp(min=0).long()), 0.0)
    return s, of, of.sum(1, keepdim=True).clamp(min=1e-37)


def _plain_route(s, c):
    E, ids = c["E"], _choose(s["logits"], s["bias"], c)
    _, w, total = _chosen_scores(s["logits"], ids, c)
    w = c["scale"] * (w / total if c["norm"] else w)
    a = torch.where(ids < 0, E, ids).view(-1).long()
    counts = torch.bincount(a, minlength=E + 1)
    starts = counts.cumsum(0) - counts
    order = a.sort(stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(len(order), device=order.device)
    rows = starts[E]
    return {"topk_idx": ids, "topk_w": w, "counts": counts[:E].int(), "offsets": starts.int(),
            "perm": torch.where(torch.arange(len(order), device=order.device) < rows, order, -1).int(),
            "pos": torch.where(a < E, place, -1).int()}


def _plain_route_grad(s, c):
    ids, dw = s["ids"], s["dw"]
    p, w, total = _chosen_scores(s["logits"], ids, c)
    g = torch.where(ids >= 0, c["scale"] * dw, 0.0)  # of the chosen scores
    if c["norm"]:
        w = w / total
        g = (g - (g * w).sum(1, keepdim=True)) / total
        g = torch.where(ids >= 0, g, 0.0)
    ds = torch.zeros_like(p).scatter_add_(1, ids.clamp(min=0).long(), g)
    if c["score"] == "sigmoid":
        dl = ds * p * (1 - p)
    else:
        dl = p * (ds - (ds * p).sum(1, keepdim=True))
    return dl.to(s["logits"].dtype)


def _values(q, scale):
    """What rows in 8 bits stand for."""
    return torch.mul(q, scale.unsqueeze(1), out=torch.empty(q.shape, dtype=torch.bfloat16, device=q.device))


def _plain_norm(s, c):
    r = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    x = r.float()
    rstd = torch.rsqrt(x.square().mean(1) + EPS)
    y = x * rstd.unsqueeze(1) * s["w"].float()
    if c["out"] == "same":
        return {"y": y.to(r.dtype), "rstd": rstd, "r": r}
    top = y.abs().amax(1, keepdim=True)
    q = torch.round(y * ((1.0 / top) * 127.0))
    scale = (top / 127.0).squeeze(1)
    return {"y": _values(q, scale), "scale": scale, "r": r}


def _plain_norm_grad(s, c):
    n = s["x"].float() * s["rstd"].unsqueeze(1)
    g = s["dy"].float() * s["w"].float()
    dx = s["rstd"].unsqueeze(1) * (g - n * (g * n).mean(1, keepdim=True))
    if s["dr"] is not None:
        dx = dx + s["dr"].float()
    return {"dx": dx.to(s["x"].dtype), "dw": (s["dy"].float() * n).sum(0)}


def _order_keys(x):
    """Whole numbers that order as (value, lowest place first)."""
    b = (x.float() + 0.0).view(torch.int32).long()
    b = torch.where(b < 0, -(b & 0x7FFFFFFF), b)
    return (b << 32) - torch.arange(x.shape[1], device=x.device)


def _log_softmax(x):
    """(x - log of the sum of exps, that log, entropy)."""
    top = x.amax(1, keepdim=True)
    z = x - top
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    entropy = torch.log(total) - (e * z).sum(1, keepdim=True) / total
    return z - torch.log(total), (top + torch.log(total)).squeeze(1), entropy.squeeze(1)


def _plain_logprobs(s, c):
    logp, lse, entropy = _log_softmax(s["logits"].float() / c["temperature"])
    out = {"logprob": logp.gather(1, s["tokens"].long().unsqueeze(1)).squeeze(1), "entropy": entropy, "lse": lse}
    ids = (-_order_keys(s["logits"]).topk(c["top"], 1).values) & 0xFFFFFFFF
    return dict(out, top_ids=ids.int(), top_logprobs=logp.gather(1, ids))


def _plain_distill(s, c):
    t, ids = c["temperature"], s["ids"].long()
    live = s["scale"] != 0.0
    x = s["logits"].float()
    top = x.amax(1, keepdim=True)
    e = torch.exp((x - top) / t)
    total = e.sum(1, keepdim=True)
    # a divergence is a small difference of large logarithms: those of the listed tokens in 64 bits
    logq = (x.gather(1, ids).double() - top) / t - torch.log(total.double())
    if c["tail"]:
        logp = s["lp"].double()
        p = torch.exp(logp)
        rest = (1.0 - p.sum(1, keepdim=True)).clamp(min=0.0)
        q_rest = e.scatter(1, ids, 0.0).sum(1, keepdim=True).double() / total
        kl = (p * (logp - logq)).sum(1) + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(q_rest)), 0.0).squeeze(1)
        dense = e / total * (1.0 - rest / q_rest).float()
        dense = dense.scatter(1, ids, (torch.exp(logq) - p).float())
    else:
        logp = _log_softmax(s["lp"].double())[0]
        p = torch.exp(logp)
        kl = (p * (logp - logq)).sum(1)
        dense = (e / total).scatter(1, ids, (torch.exp(logq) - p).float())
    out = {"kl": torch.where(live, kl.float(), 0.0), "ce": torch.zeros_like(s["scale"])}
    dense = dense * t
    if c["ce"]:
        label = s["labels"].long().unsqueeze(1)
        logq = _log_softmax(x)[0]
        out["ce"] = torch.where(live, -logq.gather(1, label).squeeze(1), 0.0)
        dense = dense + c["ce"] * torch.exp(logq).scatter_add(1, label, torch.full_like(label, -1, dtype=torch.float32))
    if c["grad"]:
        out["dlogits"] = (dense * s["scale"].unsqueeze(1)).to(s["logits"].dtype)
    return out


PLAIN = {"route": _plain_route, "route_grad": _plain_route_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
         "logprobs": _plain_logprobs, "distill": _plain_distill}


# ---- the definitions in 64 bits ---------------------------------------------
def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "route":
        return _exact_route(s, c)
    if c["op"] == "route_grad":
        return _exact_route_grad(s, c)
    if c["op"] == "norm":
        return _exact_norm(s, c)
    if c["op"] == "norm_grad":
        return _exact_norm_grad(s, c)
    if c["op"] == "logprobs":
        lp = torch.log_softmax(s["logits"].double() / c["temperature"], 1)
        tok = s["tokens"].long()
        p = lp.exp()
        top = torch.sort(s["logits"].double(), dim=1, descending=True, stable=True).indices[:, :c["top"]]
        return {"logprob": lp[torch.arange(len(tok), device="cuda"), tok], "entropy": -(p * lp).sum(1),
                "lse": torch.logsumexp(s["logits"].double() / c["temperature"], 1), "top_ids": None, "top_logprobs": lp.gather(1, top)}
    return _exact_distill(s, c)


def _exact_log_scores(s, c):
    x = s["logits"].double()
    if c["score"] == "sigmoid":
        return torch.nn.functional.logsigmoid(x)
    return x - torch.logsumexp(x, 1, keepdim=True).nan_to_num(neginf=0.0)


def _exact_weights(logs, ids, c):
    """Weights of the chosen out of their log scores, 0 where none is chosen."""
    of = torch.where(ids < 0, -math.inf, logs.gather(1, ids.clamp(min=0).long()))
    if c["norm"]:
        of = of - torch.logsumexp(of, 1, keepdim=True).nan_to_num(neginf=0.0)
    return c["scale"] * of.exp()


def _exact_route(s, c):
    logs = _exact_log_scores(s, c)
    return dict.fromkeys(("topk_idx", "counts", "offsets", "perm", "pos")) | {"topk_w": _exact_weights(logs, _choose(s["logits"], s["bias"], c), c)}


def _exact_route_grad(s, c):
    with torch.enable_grad():
        x = s["logits"].double().clamp(min=-1e4).requires_grad_()  # padding has no chosen expert: its gradient is 0
        logs = _exact_log_scores({"logits": x}, c)
        of = logs.gather(1, s["ids"].clamp(min=0).long()).masked_fill(s["ids"] < 0, -1e4)
        if c["norm"]:
            of = of - torch.logsumexp(of, 1, keepdim=True)
        w = c["scale"] * of.exp()
        (w * s["dw"].double() * (s["ids"] >= 0)).sum().backward()
    return x.grad


def _exact_norm(s, c):
    r = s["x"] if s["residual"] is None else (s["x"].double() + s["residual"].double()).to(s["x"].dtype)
    x = r.double()
    rstd = 1.0 / (x.pow(2).sum(1) / c["d"] + EPS).sqrt()
    y = x * rstd[:, None] * s["w"].double()
    if c["out"] == "same":
        return {"y": y, "rstd": rstd, "r": r.double()}
    scale = y.abs().max(1).values / 127
    return {"y": torch.round(y / scale[:, None]) * scale[:, None], "scale": scale, "r": r.double()}


def _exact_norm_grad(s, c):
    x, dy, w, rstd = s["x"].double(), s["dy"].double(), s["w"].double(), s["rstd"].double()
    dot = (dy * w * x).sum(1)
    dx = dy * w * rstd[:, None] - x * (rstd ** 3 * dot / c["d"])[:, None]
    return {"dx": dx if s["dr"] is None else dx + s["dr"].double(), "dw": torch.matmul(rstd[None], dy * x)[0]}


def _exact_distill(s, c):
    t, ids, T = c["temperature"], s["ids"].long(), c["T"]
    x = s["logits"].double()
    scale = s["scale"].double()
    on = (scale != 0).double()
    lq = torch.log_softmax(x / t, 1)
    lp = s["lp"].double() if c["tail"] else torch.log_softmax(s["lp"].double(), 1)
    p = lp.exp()
    listed_q = lq.gather(1, ids)
    target = torch.zeros_like(lq).scatter_(1, ids, p)
    kl = (p * (lp - listed_q)).sum(1)
    q = lq.exp()
    if c["tail"]:
        rest = (1 - p.sum(1)).clamp(min=0)
        others = torch.logsumexp(lq.scatter(1, ids, -math.inf), 1)
        kl = kl + torch.special.xlogy(rest, rest) - rest * others
        # the rest's probability is spread over the others as the student spreads its own
        target += rest[:, None] * (lq - others[:, None]).exp().scatter(1, ids, 0.0)
        grad = t * (q * (p.sum(1) + rest)[:, None] - target)
    else:
        grad = t * (q - target)
    ce = torch.zeros(T, dtype=torch.float64, device="cuda")
    if c["ce"]:
        l1 = torch.log_softmax(x, 1)
        label = s["labels"].long()
        ce = -l1[torch.arange(T, device="cuda"), label]
        d1 = l1.exp()
        d1[torch.arange(T, device="cuda"), label] -= 1
        grad = grad + c["ce"] * d1
    out = {"kl": kl * on, "ce": ce * on}
    return dict(out, dlogits=grad * scale[:, None]) if c["grad"] else out


# ---- what a pass cannot do without ------------------------------------------
def work(case):
    c = case
    if c["op"].startswith("route"):
        n, k = c["T"] * c["E"], c["T"] * c["k"]
        es = 4 if c["dtype"] == "f32" else 2
        if c["op"] == "route":
            return {"bytes": n * es + 16 * k + 12 * c["E"], "flops": 10 * n}
        return {"bytes": 2 * n * es + 8 * k, "flops": 10 * n}
    es = 4 if c["dtype"] == "f32" else 2
    if c["op"].startswith("norm"):
        n = c["T"] * c["d"]
        if c["op"] == "norm_grad":
            return {"bytes": n * es * (4 if c["residual"] else 3) + 6 * c["d"], "flops": 10 * n}
        return {"bytes": n * (es * (3 if c["residual"] else 1) + (1 if c["out"] == "int8" else es)) + 4 * c["T"], "flops": 6 * n}
    n = c["T"] * c["V"]
    if c["op"] == "logprobs":
        return {"bytes": n * es + c["T"] * (16 + 8 * c["top"]), "flops": 6 * n}
    n = int(n * (1 - c["pad"]))
    return {"bytes": n * es + (c["T"] * c["V"] * es if c["grad"] else 0) + c["T"] * (16 + 8 * c["top"]), "flops": 8 * n}
