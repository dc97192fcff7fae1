"""The operators on a router's logits: what a pass through each of them reads, computes and returns.

Three operators, each with its backward pass, one dict of plain values per case:

  logprobs  log probabilities of given experts, log-sum-exp and entropy of every token's distribution, and its most
            likely experts; backward from all three.
  balance   the balance loss of groups of tokens (layers, sequences) with the counts per expert; backward.
  distill   the divergence of a router from the top logits of another one (a teacher); backward.

A case's `pass` is "forward" or "backward".  `padded` is the share of rows that do not count (they hold NaN), `out` the
share of experts that are out for a token (logit -infinity), `gap` the places between two rows of logits.
"""
import math

import torch

own = False     # True: run() calls the framework's operators, False: it computes their plain form
DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------------ cases
def _logprobs(name, way, rows, E, k, dtype="fp32", alternatives=0, temperature=1.0, padded=0.0, out=0.0, gap=0, zipf=1.0):
    return {"name": name, "operator": "logprobs", "pass": way, "rows": rows, "experts": E, "top_k": k, "dtype": dtype,
            "alternatives": alternatives, "temperature": temperature, "padded": padded, "out": out, "gap": gap, "zipf": zipf}


def _balance(name, way, rows, E, k, groups, ragged=False, dtype="fp32", padded=0.0, out=0.0, gap=0, zipf=1.0):
    return {"name": name, "operator": "balance", "pass": way, "rows": rows, "experts": E, "top_k": k, "groups": groups,
            "ragged": ragged, "dtype": dtype, "padded": padded, "out": out, "gap": gap, "zipf": zipf}


def _distill(name, way, rows, E, listed_, tail, dtype="fp32", temperature=1.0, padded=0.0, out=0.0, gap=0, zipf=1.0):
    return {"name": name, "operator": "distill", "pass": way, "rows": rows, "experts": E, "teacher": listed_, "tail": tail,
            "dtype": dtype, "temperature": temperature, "padded": padded, "out": out, "gap": gap, "zipf": zipf}


def listed():
    return [
        # one token of a decode step, 256 experts, top-8: gate weights and the next choices; latency is all there is
        _logprobs("gate_one_token", "forward", 1, 256, 8, alternatives=8),
        # the true router's lists for a forecaster: a million tokens of 256 experts, the eight most likely of each
        _logprobs("teacher_lists_e256", "forward", 1 << 20, 256, 8, alternatives=8, zipf=1.1),
        # picks of an earlier policy under the present router, 60 experts in rows of 64 places, fp16, padded batch
        _logprobs("replay_e60_fp16", "forward", 99_991, 60, 6, dtype="fp16", padded=0.1, out=0.05, gap=4, zipf=0.8),
        # gradient of gate weights, z-loss and entropy: eight layers of 64 GPUs, 8 experts, top-2
        _logprobs("gate_grad_e8", "backward", 8 << 20, 8, 2, zipf=1.2),
        # the balance loss of the benchmark workload: 32 layers of 2^20 tokens, 8 experts, top-2
        _balance("balance_32_layers_e8", "forward", 32 << 20, 8, 2, 32, zipf=1.2),
        # the loss of every sequence of a packed batch: 300 sequences of odd lengths, 61 experts (no wide loads)
        _balance("balance_sequences_e61", "forward", 65_537, 61, 4, 300, ragged=True, padded=0.05, zipf=0.8),
        # one layer of a small job, 16 GPUs of 2048 tokens, 8 experts: launches count
        _balance("balance_grad_small", "backward", 32_768, 8, 2, 1),
        # one layer of a 512-GPU training step's share: 2^20 tokens, 256 experts, top-8
        _balance("balance_grad_e256", "backward", 1 << 20, 256, 8, 1, zipf=1.1),
        # a forecaster of 64 experts on the tokens of a short prompt
        _distill("forecast_small", "forward", 333, 64, 8, True, temperature=2.0),
        # a bf16 forecaster of 64 experts on 2^20 tokens, the teacher's six best
        _distill("forecast_e64_bf16", "forward", 1 << 20, 64, 6, False, dtype="bf16", zipf=0.8),
        # training of a forecaster, 256 experts, eight best and the tail, 2^20 tokens
        _distill("forecast_grad_e256", "backward", 1 << 20, 256, 8, True, zipf=1.1),
        # 512 fine-grained experts in bf16, long lists, padded
        _distill("forecast_grad_e512_bf16", "backward", 131_071, 512, 32, True, dtype="bf16", temperature=2.0, padded=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    E = rng.choice([8, 16, 32, 60, 64, 96, 128, 160, 256, 512, 1024]) if rng.random() < 0.7 else _log_int(rng, 2, 1024)
    rows = _log_int(rng, 1, max(2, (1 << 27) // E))
    dtype = rng.choice(["fp32", "fp32", "bf16", "fp16"])
    way = rng.choice(["forward", "backward"])
    k = max(1, min(E // 2, rng.choice([1, 2, 4, 6, 8, 8, 16])))
    more = {"dtype": dtype, "padded": rng.choice([0.0, 0.0, 0.1, 0.5]), "out": rng.choice([0.0, 0.0, 0.25]), "zipf": round(rng.uniform(0.0, 1.2), 2),
            "gap": rng.choice([0, 0, 0, 4, 8, 3])}
    u = rng.random()
    if u < 0.35:
        c = _logprobs("", way, rows, E, k, alternatives=rng.choice([0, 0, min(4, k), k]) if way == "forward" else 0,
                      temperature=rng.choice([1.0, 1.0, 0.7, 2.0]), **more)
    elif u < 0.7:
        ragged = rng.random() < 0.5
        groups = _log_int(rng, 1, max(1, min(512, rows)))
        c = _balance("", way, rows if ragged else max(1, rows // groups) * groups, E, k, groups, ragged=ragged, **more)
    else:
        K = max(1, min(E, rng.choice([1, 4, 8, 16, 32, 64])))
        c = _distill("", way, rows, E, K, 2 * K <= E and rng.random() < 0.6, temperature=rng.choice([1.0, 1.0, 2.0, 4.0]), **more)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    T, E = float(case["rows"]), float(case["experts"])
    size = 4.0 if case["dtype"] == "fp32" else 2.0
    grad = case["pass"] == "backward"
    moved = T * E * size * (2 if grad else 1) + (T if case["padded"] else 0.0)
    if case["operator"] == "logprobs":
        k, m = case["top_k"], case["alternatives"]
        # indices and their values' gradients, two gradients a row; or indices, values, two values a row and the alternatives
        moved += T * (8 * k + 8) + T * 8 * m
    elif case["operator"] == "balance":
        # counts, sums and losses of the groups; picks only count on the way forward
        moved += case["groups"] * (8 * E + 12) + (0.0 if grad else T * 4 * case["top_k"] + case["groups"] * 4 * E)
    else:
        moved += T * 8 * case["teacher"] + (4 * T if case["tail"] else 0.0) + 4 * T
    return {"bytes": moved, "flops": (8.0 if grad else 6.0) * T * E}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    T, E, dtype = case["rows"], case["experts"], DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=gen)

    popular = -case["zipf"] * torch.log(torch.arange(1, E + 1, device=DEV, dtype=torch.float32))
    popular = popular[torch.randperm(E, device=DEV, generator=gen)]
    x = normal(T, E).add_(popular)
    if case["out"]:
        gone = torch.rand((T, E), device=DEV, generator=gen) < case["out"]
        gone[:, 0] &= E > 1                                          # a row may lose all its experts but one
        gone[torch.arange(T, device=DEV), torch.randint(0, E, (T,), device=DEV, generator=gen)] = False
        x.masked_fill_(gone, -math.inf)
    s = {"case": case, "row_mask": None}
    scale = 1.0 if dtype == torch.float16 else 1.0 / T               # the gradient of a mean; in fp16 it is scaled up, as its small values need
    if case["padded"]:
        s["row_mask"] = (torch.rand(T, device=DEV, generator=gen) >= case["padded"]).to(torch.uint8)
    if case["operator"] == "distill":
        t = normal(T, E).mul_(0.5).add_(x)                           # the teacher: near the student, the same experts out
        best = t.topk(case["teacher"], dim=1)
        s["teacher_idx"], s["teacher_logits"] = best.indices.to(torch.int32), best.values.contiguous()
        s["teacher_lse"] = torch.logsumexp(t / case["temperature"], dim=1) if case["tail"] else None
        s["d_loss"] = torch.rand(T, device=DEV, generator=gen).add_(0.5).mul_(scale)
        del t, best
    else:
        earlier = x if case["operator"] == "balance" else normal(T, E).mul_(0.1).add_(x)
        s["picks"] = earlier.topk(case["top_k"], dim=1).indices.to(torch.int32)
        del earlier
    if case["padded"]:
        x.masked_fill_((s["row_mask"] == 0)[:, None], math.nan)
        for name in ("picks", "teacher_idx"):
            if name in s:
                s[name].masked_fill_((s["row_mask"] == 0)[:, None], -1)
    places = torch.zeros((T, E + case["gap"]), device=DEV, dtype=dtype)
    places[:, :E] = x
    s["logits"] = places[:, :E]
    if case["operator"] == "logprobs" and case["pass"] == "backward":
        s["d_logp"], s["d_lse"], s["d_entropy"] = normal(T, case["top_k"]).mul_(scale), normal(T).mul_(0.01 * scale), normal(T).mul_(0.1 * scale)
    if case["operator"] == "balance":
        n = case["groups"]
        s["group_off"] = None
        if case["ragged"]:
            cuts = torch.randint(0, T + 1, (n - 1,), device=DEV, generator=gen).sort().values
            s["group_off"] = torch.cat([torch.zeros(1, device=DEV, dtype=torch.int64), cuts, torch.full((1,), T, device=DEV)]).to(torch.int64)
        if case["pass"] == "backward":
            s["counts"], s["tokens"] = _counts(s)
            s["d_loss"] = torch.rand(n, device=DEV, generator=gen).add_(0.5).mul_(scale * 64 * T)
    return s


def _group_of(s):
    """The group of every row."""
    row = torch.arange(s["case"]["rows"], device=DEV)
    if s["group_off"] is None:
        return row // (s["case"]["rows"] // s["case"]["groups"])
    return torch.bucketize(row, s["group_off"][1:], right=True)


def _counts(s):
    """Picks per group and expert, counted rows per group."""
    n, E = s["case"]["groups"], s["case"]["experts"]
    group = _group_of(s)
    live = _live(s)
    good = live[:, None] & (s["picks"] >= 0) & (s["picks"] < E)
    counts = torch.bincount((group[:, None] * E + s["picks"])[good], minlength=n * E).view(n, E)
    return counts, torch.bincount(group[live], minlength=n)


def _live(s):
    """Rows that count: not padded, and with an expert left."""
    some = s["logits"].amax(1) > -math.inf
    return some if s["row_mask"] is None else (s["row_mask"] != 0) & some


# ------------------------------------------------------------------------------------------------ one pass
COEF = 0.01


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2510_19262_amd as rs
    case = s["case"]
    if case["operator"] == "logprobs":
        if case["pass"] == "forward":
            return rs.route_logprobs(s["logits"], s["picks"], alternatives=case["alternatives"], temperature=case["temperature"],
                                     row_mask=s["row_mask"])
        return rs.route_logprobs_backward(s["logits"], s["picks"], s["d_logp"], s["d_lse"], s["d_entropy"],
                                          temperature=case["temperature"], row_mask=s["row_mask"])
    if case["operator"] == "balance":
        if case["pass"] == "forward":
            return rs.route_balance(s["logits"], s["picks"], groups=case["groups"], group_off=s["group_off"], coef=COEF,
                                    row_mask=s["row_mask"])
        return rs.route_balance_backward(s["logits"], case["top_k"], s["counts"], s["tokens"], s["d_loss"], group_off=s["group_off"],
                                         coef=COEF, row_mask=s["row_mask"])
    if case["pass"] == "forward":
        return rs.route_distill(s["logits"], s["teacher_idx"], s["teacher_logits"], s["teacher_lse"], temperature=case["temperature"],
                                row_mask=s["row_mask"])
    return rs.route_distill_backward(s["logits"], s["teacher_idx"], s["teacher_logits"], s["d_loss"], s["teacher_lse"],
                                     temperature=case["temperature"], row_mask=s["row_mask"])


def _softmax(s, z, live):
    """exp(z - max) and what it takes to go on: (shifted logits, exponentials, their sum), rows that do not count as zeros."""
    z = torch.where(live[:, None], z, torch.zeros_like(z))
    top = z.amax(1, keepdim=True)
    t = z - top
    e = torch.exp(t)
    return top, t, e, e.sum(1, keepdim=True)


def _run_plain(s):
    case = s["case"]
    return {"logprobs": _plain_logprobs, "balance": _plain_balance, "distill": _plain_distill}[case["operator"]](s, case, case["pass"] == "backward")


def _plain_logprobs(s, case, backward):
    E, live = case["experts"], _live(s)
    z = s["logits"].to(torch.float32) / case["temperature"]
    top, t, e, total = _softmax(s, z, live)
    log_total = torch.log(total)
    good = live[:, None] & (s["picks"] >= 0) & (s["picks"] < E)
    at = s["picks"].clamp(0, E - 1).to(torch.int64)
    entropy = log_total - torch.where(e > 0, e * t, torch.zeros_like(e)).sum(1, keepdim=True) / total
    if backward:
        p = e / total
        g = torch.where(good, s["d_logp"], torch.zeros_like(s["d_logp"]))
        log_p = torch.where(e > 0, t - log_total, torch.zeros_like(t))
        dx = -p * (g.sum(1, keepdim=True) - s["d_lse"][:, None] + s["d_entropy"][:, None] * (log_p + entropy))
        dx = dx.scatter_add_(1, at, g) / case["temperature"]
        return torch.where(live[:, None], dx, torch.zeros_like(dx)).to(s["logits"].dtype)
    none = torch.zeros((), device=DEV)
    logp = torch.where(good, t.gather(1, at) - log_total, none)
    lse = torch.where(live, (top + log_total)[:, 0], none)
    entropy = torch.where(live, entropy[:, 0], none)
    alt_idx = alt_logp = None
    if case["alternatives"]:
        order = torch.sort(s["logits"].to(torch.float32), dim=1, descending=True, stable=True).indices[:, :case["alternatives"]]
        value = t.gather(1, order)
        there = live[:, None] & (value > -math.inf)
        alt_idx = torch.where(there, order, torch.full_like(order, -1)).to(torch.int32)
        alt_logp = torch.where(there, value - log_total, torch.where(live[:, None], torch.full_like(value, -math.inf), torch.zeros_like(value)))
    return logp, lse, entropy, alt_idx, alt_logp


def _plain_balance(s, case, backward):
    n, E, k = case["groups"], case["experts"], case["top_k"]
    live = _live(s)
    _, _, e, total = _softmax(s, s["logits"].to(torch.float32), live)
    p = torch.where(live[:, None], e / total, torch.zeros_like(e))
    if backward:
        tokens = s["tokens"].to(torch.float64).clamp(min=1)
        # against the mean count: the same gradient, and nothing is lost where the counts are nearly equal
        weight = (s["d_loss"].to(torch.float64) * COEF * E / (k * tokens * tokens))[:, None] * (s["counts"] - s["counts"].to(torch.float64).mean(1, keepdim=True))
        a = weight.to(torch.float32)
        if n > 1:
            a = a[_group_of(s)]
        return (p * (a - (a * p).sum(1, keepdim=True))).to(s["logits"].dtype)
    counts, tokens = _counts(s)
    if s["group_off"] is None:
        sums = p.view(n, -1, E).sum(1)
    else:
        sums = torch.zeros((n, E), device=DEV, dtype=torch.float64).index_add_(0, _group_of(s), p.to(torch.float64)).to(torch.float32)
    many = tokens.to(torch.float64).clamp(min=1)
    loss = COEF * E / (k * many * many) * (counts * sums.to(torch.float64)).sum(1)
    return counts, tokens, sums, loss.to(torch.float32)


def _plain_distill(s, case, backward):
    E, tau, live = case["experts"], case["temperature"], _live(s)
    x, T = s["logits"].to(torch.float32), s["teacher_logits"]
    top, t, e, total = _softmax(s, x / tau, live)
    good = live[:, None] & (s["teacher_idx"] >= 0) & (s["teacher_idx"] < E) & (T > -math.inf)
    at = torch.where(good, s["teacher_idx"], torch.full_like(s["teacher_idx"], E)).to(torch.int64)
    none, one = torch.zeros((), device=DEV), torch.ones((), device=DEV)
    u = torch.where(good, T / tau, torch.full_like(T, -math.inf))
    if s["teacher_lse"] is None:
        best = u.amax(1, keepdim=True)
        best = torch.where(best > -math.inf, best, none)
        log_mass = best + torch.log(torch.exp(u - best).sum(1, keepdim=True))
    else:
        log_mass = s["teacher_lse"][:, None]
    q = torch.exp(u - log_mass)
    p = torch.where(good, (e / total).gather(1, at.clamp(max=E - 1)), none)
    outside = torch.ones((case["rows"], E + 1), device=DEV).scatter_(1, at, 0.0)[:, :E]
    rest_p = (e * outside).sum(1, keepdim=True) / total
    mass = q.sum(1, keepdim=True)
    rest_q = torch.where(rest_p > 0, (1 - mass).clamp(min=0), none) if s["teacher_lse"] is not None else torch.zeros_like(mass)
    if backward:
        listed_q = torch.zeros((case["rows"], E + 1), device=DEV).scatter_add_(1, at, q)[:, :E]
        # outside the list: p (1 - q_rest / p_rest), and the two rests differ by what the listed ones do
        push = torch.where(rest_q > 0, (q - p).sum(1, keepdim=True) / rest_p, mass)
        dx = e / total * torch.where(outside > 0, push, mass + rest_q) - listed_q
        return torch.where(live[:, None], dx * (tau * s["d_loss"][:, None]), none).to(s["logits"].dtype)
    # sum q log(q / p) as the sum of q log(q / p) - q + p, whose terms do not cancel where p is near q
    d = (x.gather(1, at.clamp(max=E - 1)) - T) / tau + (log_mass - top - torch.log(total))
    terms = torch.where(good, torch.where(q > 0, torch.where(d < 1, q * (torch.expm1(d) - d), p - q - q * d), p), none).sum(1, keepdim=True)
    if s["teacher_lse"] is None:
        terms = torch.where(mass > 0, terms + rest_p, none)
    else:
        apart = (q - p).sum(1, keepdim=True) / torch.where(rest_q > 0, rest_q, one)          # p_rest / q_rest - 1
        terms = terms + torch.where(rest_q > 0, rest_q * (apart - torch.log1p(apart)), rest_p + mass - one)
    return torch.where(live, tau * tau * terms[:, 0], none)


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
FAR = -1e9      # stands for -infinity where a derivative is taken: its exponential is zero all the same


def exact(case, seed):
    s = prepare(case, seed)
    E = case["experts"]
    live = _live(s)
    x = s["logits"].to(torch.float64).clamp(min=FAR)
    x = torch.where(live[:, None], x, torch.zeros_like(x)).requires_grad_(case["pass"] == "backward")
    with torch.set_grad_enabled(case["pass"] == "backward"):
        log_p = torch.log_softmax(x / case.get("temperature", 1.0), dim=1)
        value = {"logprobs": _exact_logprobs, "balance": _exact_balance, "distill": _exact_distill}[case["operator"]](s, case, live, x, log_p)
        if case["pass"] == "forward":
            return value
        return torch.autograd.grad(value, x)[0]


def _exact_logprobs(s, case, live, x, log_p):
    E = case["experts"]
    good = live[:, None] & (s["picks"] >= 0) & (s["picks"] < E)
    logp = log_p.gather(1, s["picks"].clamp(0, E - 1).to(torch.int64)) * good
    lse = torch.logsumexp(x / case["temperature"], dim=1) * live
    entropy = -(log_p.exp() * log_p).sum(1) * live
    if case["pass"] == "backward":
        return (logp * s["d_logp"]).sum() + (lse * s["d_lse"]).sum() + (entropy * s["d_entropy"]).sum()
    logp = torch.where(logp < FAR / 1e3, torch.full_like(logp, -math.inf), logp)
    if not case["alternatives"]:
        return logp, lse, entropy, None, None
    best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["alternatives"]]
    value = log_p.gather(1, best)
    gone = live[:, None] & (value < FAR / 1e3)
    alt_idx = torch.where(gone | ~live[:, None], -1, best).to(torch.int32)
    return logp, lse, entropy, alt_idx, torch.where(gone, -math.inf, value) * live[:, None]


def _exact_balance(s, case, live, x, log_p):
    n, E, k = case["groups"], case["experts"], case["top_k"]
    p = log_p.exp() * live[:, None]
    edges = s["group_off"].tolist() if s["group_off"] is not None else [g * (case["rows"] // n) for g in range(n + 1)]
    sums = torch.stack([p[a:b].sum(0) for a, b in zip(edges, edges[1:])])
    if case["pass"] == "backward":
        counts, tokens = s["counts"], s["tokens"]
    else:
        good = live[:, None] & (s["picks"] >= 0)
        counts = torch.stack([torch.bincount(s["picks"][a:b][good[a:b]], minlength=E) for a, b in zip(edges, edges[1:])])
        tokens = torch.stack([live[a:b].sum() for a, b in zip(edges, edges[1:])])
    share = counts / (k * tokens.clamp(min=1))[:, None]
    loss = COEF * E * (share * sums / tokens.clamp(min=1)[:, None]).sum(1)
    if case["pass"] == "backward":
        return (loss * s["d_loss"]).sum()
    return counts, tokens, sums, loss


def _exact_distill(s, case, live, x, log_p):
    tau = case["temperature"]
    u = s["teacher_logits"].to(torch.float64) / tau
    good = live[:, None] & (s["teacher_idx"] >= 0) & (u > -math.inf)
    at = s["teacher_idx"].clamp(min=0).to(torch.int64)
    log_q = u - s["teacher_lse"].to(torch.float64)[:, None] if case["tail"] else torch.log_softmax(u, dim=1)
    log_q = torch.where(good, log_q, FAR)
    loss = (log_q.exp() * (log_q - log_p.gather(1, at)) * good).sum(1)
    if case["tail"]:
        inside = torch.zeros_like(log_p, dtype=torch.bool).scatter_(1, at, True)
        rest_q = (1 - (log_q.exp() * good).sum(1)).clamp(min=0)
        rest_p = log_p.exp().masked_fill(inside, 0.0).sum(1)
        there = live & (rest_p > 0) & (rest_q > 0)
        rest_p, rest_q = torch.where(there, rest_p, 1.0), torch.where(there, rest_q, 1.0)
        loss = loss + torch.where(there, rest_q * (rest_q.log() - rest_p.log()), 0.0)
    loss = tau * tau * loss * live
    return (loss * s["d_loss"]).sum() if case["pass"] == "backward" else loss
