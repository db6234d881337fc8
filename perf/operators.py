"""The language-model operators that go with a nearest-neighbour search, as cases that can be timed and compared.

A search returns the stored vectors nearest to a hidden state, and each stored vector carries the token that followed it.
Around that: the neighbours' distances as a distribution over their tokens, the model's logits as a product of 8-bit rows,
log-probabilities of given tokens (of the model alone, or mixed with the neighbours' distribution), and a student model
trained towards a few listed tokens of a teacher.

  op          what one pass does
  head        hidden states quantised to 8 bits, then their product with the 8-bit output embedding: logits
  scores      the product of 8-bit queries and 8-bit stored vectors, with a bias for each stored vector
  neighbours  search results (ids and distances) as distinct tokens with log-probabilities
  logprobs    log-probability of a given token, entropy and the best alternatives for each row of logits
  policy      log-probabilities and entropy, then their gradient with respect to the logits
  distill     loss towards a teacher's listed tokens: the loss and the gradient in one call, or forward, then backward

`run` is the plain form where `own` is false and calls the library where it is true.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
NONE = -1        # the token of an unused place


def listed():
    return [
        # serving, one sequence: the hidden state of one token against the output embedding (latency, bound by the weights)
        {"name": "head for one token", "op": "head", "rows": 1, "d": 4096, "vocab": 32_768, "dtype": "bf16"},
        # scoring or training: all the tokens of a batch
        {"name": "head for a batch", "op": "head", "rows": 2_048, "d": 4_096, "vocab": 32_768, "dtype": "bf16"},
        # every stored vector of a block scored for an odd number of queries, 96-d descriptors held in 8 bits; the bias
        # -|x|^2/2 makes the largest score the nearest vector
        {"name": "scores of stored vectors", "op": "scores", "rows": 777, "d": 96, "stored": 100_003},
        # an interactive service: the ten neighbours of one hidden state
        {"name": "neighbours of one state", "op": "neighbours", "rows": 1, "k": 10, "table": 1_000_000, "vocab": 32_768},
        # a benchmark's batch, k = 100
        {"name": "neighbours of a batch", "op": "neighbours", "rows": 10_000, "k": 100, "table": 10_000_000, "vocab": 65_536},
        # the next token of one sequence, the model's distribution mixed with the neighbours'
        {"name": "next token of one sequence", "op": "logprobs", "rows": 1, "vocab": 131_072, "dtype": "bf16", "top": 20, "k": 64,
         "temperature": 1.0, "masked": False},
        # prompts scored in a batch, with the 20 best alternatives at each place
        {"name": "prompts scored", "op": "logprobs", "rows": 4_096, "vocab": 65_536, "dtype": "bf16", "top": 20, "k": 0,
         "temperature": 1.0, "masked": False},
        # an odd vocabulary in full precision, most of it masked in some rows (a grammar), sharpened
        {"name": "masked odd vocabulary", "op": "logprobs", "rows": 777, "vocab": 50_001, "dtype": "fp32", "top": 5, "k": 0,
         "temperature": 0.7, "masked": True},
        # a policy-gradient step with an entropy bonus
        {"name": "policy gradient", "op": "policy", "rows": 2_048, "vocab": 65_536, "dtype": "bf16", "temperature": 1.0},
        # few rows: the last places of a few sequences, trained towards their neighbours
        {"name": "distil few rows", "op": "distill", "rows": 8, "vocab": 131_072, "dtype": "bf16", "k": 20, "temperature": 1.0,
         "one_call": True},
        # a training step towards the neighbours' tokens
        {"name": "distil a batch", "op": "distill", "rows": 4_096, "vocab": 65_536, "dtype": "bf16", "k": 100, "temperature": 1.0,
         "one_call": True},
        # a teacher model's top logits, softened; odd sizes, half precision, the loss first and its gradient later
        {"name": "distil forward, backward", "op": "distill", "rows": 333, "vocab": 32_001, "dtype": "fp16", "k": 64,
         "temperature": 2.0, "one_call": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["head", "scores", "neighbours", "logprobs", "logprobs", "policy", "distill", "distill"])
    if op == "head":
        return {"op": op, "rows": _log_int(rng, 1, 2_048), "d": _log_int(rng, 64, 4_096), "vocab": _log_int(rng, 1_000, 32_768),
                "dtype": rng.choice(["bf16", "fp16", "fp32"])}
    if op == "scores":
        rows = _log_int(rng, 1, 4_096)
        return {"op": op, "rows": rows, "d": _log_int(rng, 16, 256), "stored": _log_int(rng, 1_000, min(200_000, 60_000_000 // rows))}
    if op == "neighbours":
        k = _log_int(rng, 1, 1_024)
        return {"op": op, "rows": _log_int(rng, 1, min(10_000, 90_000_000 // (k * k))), "k": k,
                "table": _log_int(rng, 100_000, 10_000_000), "vocab": _log_int(rng, 1_000, 131_072)}
    vocab = _log_int(rng, 1_000, 131_072)
    case = {"op": op, "rows": _log_int(rng, 1, min(4_096, 130_000_000 // vocab)), "vocab": vocab,
            "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "temperature": rng.choice([1.0, 1.0, 0.7, 2.0])}
    if op == "logprobs":
        case["top"] = rng.choice([0, 1, 5, 20, _log_int(rng, 1, 128)])
        case["k"] = rng.choice([0, 0, _log_int(rng, 1, 128)])
        case["masked"] = rng.random() < 0.3
        if case["k"]:                        # mixed with neighbours: serving, few rows of 16-bit logits
            case.update(dtype="bf16", rows=min(case["rows"], 256), masked=False)
    if op == "distill":
        case["k"] = _log_int(rng, 1, min(512, vocab // 2))
        case["one_call"] = rng.random() < 0.6
    return case


# ---- inputs

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _logits(gen, rows, vocab, dtype):
    """Logits of a model: normal, with a bias towards the frequent (low) tokens."""
    bias = -0.5 * torch.log1p(torch.arange(vocab, device="cuda", dtype=torch.float32))
    return (_normal(gen, rows, vocab).mul_(2.5).add_(bias)).to(dtype)


def _listed_tokens(gen, logits, k):
    """k distinct tokens a row that the row's logits find likely, at random, and a log-probability for each; of most rows
    some places at the end are unused, and of a few rows all."""
    rows = logits.shape[0]
    noisy = _normal(gen, *logits.shape).mul_(3.0).add_(logits)
    tokens = torch.topk(noisy, k, dim=1).indices.to(torch.int32)
    given = torch.log_softmax(_normal(gen, rows, k).mul_(2.0), dim=1)
    used = torch.randint(1, k + 1, (rows, 1), generator=gen, device="cuda")
    used = torch.where(torch.rand((rows, 1), generator=gen, device="cuda") < 0.3, k, used)
    if rows > 4:
        used[rows // 2] = 0
    off = torch.arange(k, device="cuda") >= used
    given -= torch.where(off, -math.inf, given).logsumexp(dim=1, keepdim=True).clamp(min=-1e3)
    return tokens.masked_fill_(off, NONE), given.masked_fill_(off, -math.inf)


def _codes(values):
    """Rows as 8-bit codes with a scale each, stored with a row length that is a multiple of 16 bytes."""
    n, d = values.shape
    scales = values.abs().amax(dim=1) / 127.0
    codes = torch.zeros((n, -(-d // 16) * 16), dtype=torch.int8, device="cuda")[:, :d]
    codes.copy_(torch.round(values / scales[:, None]).clamp_(-127, 127))
    return codes, scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, rows = case["op"], case["rows"]
    state = {"case": case}
    if op == "head":
        d, vocab = case["d"], case["vocab"]
        x = _normal(gen, rows, d)
        x *= torch.where(torch.rand(d, generator=gen, device="cuda") < 0.01, 8.0, 1.0)       # a few channels stand out
        state["x"] = x.to(TYPES[case["dtype"]])
        state["codes"], state["scales"] = _codes(_normal(gen, vocab, d).mul_(d ** -0.5))
        return state
    if op == "scores":
        d, stored = case["d"], case["stored"]
        q, x = _normal(gen, rows, d), _normal(gen, stored, d)
        q, x = q / q.norm(dim=1, keepdim=True), x / x.norm(dim=1, keepdim=True)
        state["q"], state["x"] = _codes(q), _codes(x)
        codes, scales = state["x"]
        state["bias"] = -0.5 * (codes.float().square().sum(dim=1) * scales.square())
        return state
    if op == "neighbours":
        k, table = case["k"], case["table"]
        state["ids"] = torch.randint(table, (rows, k), generator=gen, device="cuda")
        steps = torch.rand((rows, k), generator=gen, device="cuda").mul_(600.0)
        steps[:, 0] += 20_000.0
        state["dists"] = steps.cumsum(dim=1)                                               # ascending, as a search gives them
        short = torch.rand((rows, 1), generator=gen, device="cuda") < 0.05                 # few vectors in the probed lists
        off = short & (torch.arange(k, device="cuda") >= k // 2)
        state["ids"].masked_fill_(off, -1)
        state["dists"].masked_fill_(off, math.inf)
        state["tokens"] = (torch.rand(table, generator=gen, device="cuda").pow_(4) * case["vocab"]).to(torch.int32)
        state["temperature"] = 2_000.0
        return state
    vocab = case["vocab"]
    logits = _logits(gen, rows, vocab, TYPES[case["dtype"]])
    state["logits"] = logits
    if op == "distill":
        state["tokens"], state["given"] = _listed_tokens(gen, logits, case["k"])
        state["row_grads"] = torch.rand(rows, generator=gen, device="cuda").add_(0.5)
        return state
    state["targets"] = (torch.rand(rows, generator=gen, device="cuda").pow_(3) * vocab).to(torch.int32)
    if op == "policy":
        state["grad_logprobs"] = _normal(gen, rows)
        state["grad_entropy"] = torch.full((rows,), -0.01, device="cuda")
        return state
    if case["masked"]:
        few = torch.rand((rows, 1), generator=gen, device="cuda") < 0.3                    # rows that a grammar holds to few tokens
        keep = torch.rand((rows, vocab), generator=gen, device="cuda") < 0.002
        keep.scatter_(1, state["targets"].long()[:, None], True)
        logits.masked_fill_(few & ~keep, -math.inf)
    if case["k"]:
        k = min(case["k"], vocab // 2)
        state["neighbours"] = _listed_tokens(gen, logits, k)
        state["weight"] = 0.25
    return state


# ---- the plain form

def _plain_quantise(x):
    x = x.float()
    scales = x.abs().amax(dim=1) / 127.0
    return torch.round(x / scales[:, None]).clamp_(-127, 127), scales


def _plain_product(a, a_scales, b, b_scales):
    return (a.float() @ b.float().t()) * a_scales[:, None] * b_scales[None, :]


def _plain_neighbours(ids, dists, table, temperature):
    rows, k = ids.shape
    used = (ids >= 0) & (ids < table.shape[0]) & torch.isfinite(dists)
    tokens = torch.where(used, table[ids.clamp(0, table.shape[0] - 1)], NONE)
    used &= tokens >= 0
    x = torch.where(used, -dists / temperature, -math.inf)
    top = x.amax(dim=1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    total = (x - top).exp().sum(dim=1, keepdim=True).log()
    same = (tokens[:, :, None] == tokens[:, None, :]) & used[:, None, :]
    each = torch.where(same, x[:, None, :], -math.inf)
    best = each.amax(dim=2)
    best = torch.where(torch.isfinite(best), best, 0.0)
    logprobs = best - top - total + (each - best[:, :, None]).exp().sum(dim=2).log()
    place = torch.arange(k, device=ids.device)
    first = used & (torch.where(same, place[None, None, :], k).amin(dim=2) == place)
    at = torch.where(first, first.cumsum(dim=1) - 1, k)
    out_tokens = torch.full((rows, k + 1), NONE, dtype=torch.int32, device=ids.device).scatter_(1, at, tokens)
    out_logprobs = torch.full((rows, k + 1), -math.inf, device=ids.device).scatter_(1, at, logprobs)
    out_tokens[:, k], out_logprobs[:, k] = NONE, -math.inf
    return out_tokens[:, :k], out_logprobs[:, :k]


def _plain_statistics(logits, temperature):
    """-> the logits less their largest, divided by the temperature, exp of that, its sum, and what normalises a row: its
    largest logit and the logarithm of the sum."""
    x = logits.float()
    top = x.amax(dim=1, keepdim=True)
    x = (x - top) / temperature
    e = x.exp()
    total = e.sum(dim=1, keepdim=True)
    return x, e, total, torch.cat([top, total.log()], dim=1)


def _plain_best(values, top):
    """The places of the `top` largest of non-negative or finite values a row, ties to the lowest place."""
    bits = (values + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    keys = (bits << 32) - torch.arange(values.shape[1], device=values.device)
    return torch.topk(keys, top, dim=1).indices


def _plain_logprobs(state):
    case, logits = state["case"], state["logits"]
    top, targets = min(case["top"], case["vocab"]), state["targets"].long()[:, None]
    x, e, total, norms = _plain_statistics(logits, case["temperature"])
    p = e / total
    logp = x - total.log()
    if case["k"]:
        tokens, given = state["neighbours"]
        used = tokens >= 0
        weight = torch.where(used.any(dim=1, keepdim=True), state["weight"], 0.0)        # a row without neighbours is the model's
        share = torch.where(used, given.exp() * weight, 0.0)
        p *= 1.0 - weight
        p.scatter_add_(1, torch.where(used, tokens, 0).long(), share)
        logp = p.log()
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(dim=1)
    out = {"logprobs": logp.gather(1, targets)[:, 0], "entropy": entropy, "norms": norms}
    if top:
        best = _plain_best(p if case["k"] else logits.float(), top)
        best_logp = logp.gather(1, best)
        out["top_tokens"] = torch.where(best_logp > -math.inf, best, NONE).to(torch.int32)
        out["top_logprobs"] = best_logp
    return out


def _plain_policy(state):
    temperature, targets = state["case"]["temperature"], state["targets"].long()[:, None]
    x, e, total, _ = _plain_statistics(state["logits"], temperature)
    p = e / total
    logp = x - total.log()
    logprobs = logp.gather(1, targets)[:, 0]
    entropy = -(p * logp).sum(dim=1)
    g, h = state["grad_logprobs"][:, None], state["grad_entropy"][:, None]
    grad = -p * (g + h * (logp + entropy[:, None]))
    grad.scatter_add_(1, targets, g)
    return logprobs, entropy, (grad / temperature).to(state["logits"].dtype)


def _plain_distill(state):
    temperature = state["case"]["temperature"]
    tokens, given = state["tokens"], state["given"]
    x, e, total, _ = _plain_statistics(state["logits"], temperature)
    used = tokens >= 0
    at = torch.where(used, tokens, 0).long()
    t = torch.where(used, given / temperature, -math.inf)
    t_top = t.amax(dim=1, keepdim=True)
    t = t - torch.where(torch.isfinite(t_top), t_top, 0.0)
    t_sum = t.exp().sum(dim=1, keepdim=True)
    some = t_sum > 0
    share = torch.where(some, t.exp() / torch.where(some, t_sum, 1.0), 0.0)
    log_share = t - t_sum.log()
    log_student = x.gather(1, at) - total.log()
    loss = torch.where(share > 0, share * (log_share - log_student), 0.0).sum(dim=1) * temperature ** 2
    grad = torch.where(some, e / total, 0.0)
    grad.scatter_add_(1, at, -share)
    return loss, (grad * (state["row_grads"][:, None] * temperature)).to(state["logits"].dtype)


def _plain(state):
    case = state["case"]
    op = case["op"]
    if op == "head":
        codes, scales = _plain_quantise(state["x"])
        return _plain_product(codes, scales, state["codes"], state["scales"]).to(TYPES[case["dtype"]])
    if op == "scores":
        return _plain_product(*state["q"], *state["x"]) + state["bias"]
    if op == "neighbours":
        return _plain_neighbours(state["ids"], state["dists"], state["tokens"], state["temperature"])
    return {"logprobs": _plain_logprobs, "policy": _plain_policy, "distill": _plain_distill}[op](state)


# ---- the library's

def _own(state):
    import paper_2301_06672_amd as ivfpq
    case = state["case"]
    op = case["op"]
    if op == "head":
        codes, scales = ivfpq.ivfpq_quantize_rows(state["x"])
        return ivfpq.ivfpq_q8_matmul(codes, scales, state["codes"], state["scales"], out_dtype=TYPES[case["dtype"]])
    if op == "scores":
        return ivfpq.ivfpq_q8_matmul(*state["q"], *state["x"], bias=state["bias"])
    if op == "neighbours":
        return ivfpq.ivfpq_neighbour_tokens(state["ids"], state["dists"], state["tokens"], state["temperature"])
    logits, temperature = state["logits"], case["temperature"]
    if op == "logprobs":
        top = min(case["top"], case["vocab"])
        got = ivfpq.ivfpq_token_logprobs(logits, state["targets"], top=top, temperature=temperature,
                                         neighbours=state.get("neighbours"), weight=state.get("weight", 0.0))
        out = {"logprobs": got.logprobs, "entropy": got.entropy, "norms": got.norms}
        if top:
            out.update(top_tokens=got.top_tokens, top_logprobs=got.top_logprobs)
        return out
    if op == "policy":
        got = ivfpq.ivfpq_token_logprobs(logits, state["targets"], temperature=temperature)
        grad = ivfpq.ivfpq_token_logprobs_backward(logits, state["targets"], got.norms, got.entropy, state["grad_logprobs"],
                                                   state["grad_entropy"], temperature=temperature)
        return got.logprobs, got.entropy, grad
    tokens, given = state["tokens"], state["given"]
    if case["one_call"]:
        return ivfpq.ivfpq_distill_topk_step(logits, tokens, given, state["row_grads"], temperature=temperature)
    loss, norms = ivfpq.ivfpq_distill_topk(logits, tokens, given, temperature=temperature)
    return loss, ivfpq.ivfpq_distill_topk_backward(logits, norms, tokens, given, state["row_grads"], temperature=temperature)


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without

def work(case):
    op, rows = case["op"], case["rows"]
    if op in ("head", "scores"):
        d, n = case["d"], case["vocab"] if op == "head" else case["stored"]
        size = 4 if op == "scores" or case["dtype"] == "fp32" else 2
        moved = rows * d * (size if op == "head" else 1) + n * d + 4 * n + size * rows * n + (8 * n if op == "scores" else 0)
        return {"bytes": moved, "flops": 2.0 * rows * n * d}
    if op == "neighbours":
        return {"bytes": rows * case["k"] * (8 + 4 + 4 + 8), "flops": 4.0 * rows * case["k"]}
    size = 4 if case["dtype"] == "fp32" else 2
    values = rows * case["vocab"]
    if op == "logprobs":
        return {"bytes": size * values + rows * (16 + 8 * case["top"] + 8 * case["k"]), "flops": 6.0 * values}
    if op == "policy":
        return {"bytes": 2 * size * values + 20 * rows, "flops": 12.0 * values}
    return {"bytes": 2 * size * values + rows * (8 + 8 * case["k"]), "flops": 10.0 * values}


# ---- the definition, in 64 bits

def _exact_distribution(logits, temperature):
    z = logits.double() / temperature
    return z, torch.logsumexp(z, dim=1, keepdim=True)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "head":
        x = state["x"].double()
        scales = (x.abs().amax(dim=1, keepdim=True) / 127.0).float().double()          # a scale is a 32-bit number by definition
        a = (x / scales).round().clamp(-127, 127) * scales
        return a @ (state["codes"].double() * state["scales"].double()[:, None]).t().contiguous()
    if op == "scores":
        a, b = (codes.double() * scales.double()[:, None] for codes, scales in (state["q"], state["x"]))
        return a @ b.t().contiguous() + state["bias"].double()
    if op == "neighbours":
        ids, k = state["ids"].cpu(), case["k"]
        dists, table = state["dists"].cpu().double(), state["tokens"].cpu()
        all_tokens = torch.full((case["rows"], k), NONE, dtype=torch.int32)
        all_logprobs = torch.full((case["rows"], k), -math.inf, dtype=torch.float64)
        for r in range(case["rows"]):
            groups = {}
            pairs = [(int(table[i]), -d / state["temperature"]) for i, d in zip(ids[r].tolist(), dists[r].tolist()) if i >= 0 and math.isfinite(d)]
            for token, value in pairs:
                groups.setdefault(token, []).append(value)
            if not pairs:
                continue
            most = max(v for _, v in pairs)
            total = math.fsum(math.exp(v - most) for _, v in pairs)
            for at, (token, values) in enumerate(groups.items()):
                high = max(values)
                all_tokens[r, at] = token
                all_logprobs[r, at] = high - most + math.log(math.fsum(math.exp(v - high) for v in values)) - math.log(total)
        return all_tokens, all_logprobs
    z, lse = _exact_distribution(state["logits"], case["temperature"])
    if op == "distill":
        teacher = torch.full_like(z, 0.0)
        for_loss = torch.zeros(case["rows"], dtype=torch.float64, device=z.device)
        used = state["tokens"] >= 0
        at = state["tokens"].clamp(min=0).long()
        given = torch.where(used, state["given"].double() / case["temperature"], -math.inf)
        any_used = used.any(dim=1, keepdim=True)
        log_share = given - torch.where(any_used, torch.logsumexp(given, dim=1, keepdim=True), 0.0)
        share = log_share.exp()
        teacher.scatter_add_(1, at, share)
        for_loss += torch.where(used, share * (log_share - (z - lse).gather(1, at)), 0.0).sum(dim=1) * case["temperature"] ** 2
        grad = ((z - lse).exp() * any_used - teacher) * (case["temperature"] * state["row_grads"].double()[:, None])
        return for_loss, grad
    targets = state["targets"].long()[:, None]
    logp = z - lse
    if op == "policy":
        p = logp.exp()
        entropy = -(p * logp).sum(dim=1, keepdim=True)
        hot = torch.zeros_like(p).scatter_(1, targets, 1.0)
        grad = state["grad_logprobs"].double()[:, None] * (hot - p) - state["grad_entropy"].double()[:, None] * p * (logp + entropy)
        return logp.gather(1, targets)[:, 0], entropy[:, 0], grad / case["temperature"]
    if case["k"]:
        tokens, given = state["neighbours"]
        weight = state["weight"] * (tokens >= 0).any(dim=1, keepdim=True).double()
        mixed = (1.0 - weight) * logp.exp()
        mixed.scatter_add_(1, tokens.clamp(min=0).long(), weight * torch.where(tokens >= 0, given.double().exp(), 0.0))
        logp = mixed.log()
    p = logp.exp()
    most = z.amax(dim=1, keepdim=True)
    out = {"logprobs": logp.gather(1, targets)[:, 0], "entropy": -torch.where(p > 0, p * logp, 0.0).sum(dim=1),
           "norms": torch.cat([state["logits"].double().amax(dim=1, keepdim=True), (z - most).exp().sum(dim=1, keepdim=True).log()], dim=1)}
    top = min(case["top"], case["vocab"])
    if top:
        values, places = torch.sort(logp, dim=1, descending=True, stable=True)
        out["top_tokens"] = torch.where(values[:, :top] > -math.inf, places[:, :top], NONE).to(torch.int32)
        out["top_logprobs"] = values[:, :top]
    return out
