"""The operators of a model pass over drafted tokens, as cases that can be timed and compared.

A search over hidden states finds stored states, and the text behind each of them goes on in some way.  These continuations are drafts of
what the model will say: a tree of tokens for every sequence.  One pass of the model takes the last token and the drafts together: their keys
and values are appended to a paged cache with the rotation of their positions, every row attends to the cache and to its own branch of
the tree, and the model's probabilities decide which drafts are kept; the kept rows of the cache move up behind each other.

  op          what one pass does
  drafts      search results (ids, distances) and the stored text to a tree of drafted tokens
  append      queries and keys rotated, keys and values written to their places in a paged cache
  attention   every row over the cache and its ancestors among the drafted rows (single tokens, trees, or a piece of a prompt)
  verify      drafted tokens against the model's logits: the kept rows, the next token and their log-probabilities
  keep        the kept rows of all layers' caches moved to the front

`run` is the plain form where `own` is false and calls the library where it is true.

Layouts.  Sequence s has lens[s] places in the cache and m rows in the pass, of which the first counts[s] are used; row i lies at place
lens[s] + i of the pages listed in pages[s].  Keys are [pages][heads][page][d], values [pages][heads][page / 8][d][8]: the values of 8 places
side by side.
"""
import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
NONE = -1        # the token of an unused place


def listed():
    return [
        # an interactive service: the 32 neighbours of one hidden state, a small tree
        {"name": "drafts of one sequence", "op": "drafts", "n": 1, "k": 32, "depth": 6, "m": 24, "table": 1_000_000, "vocab": 32_768},
        # a server's batch with long continuations and full trees
        {"name": "drafts of a batch", "op": "drafts", "n": 1_024, "k": 100, "depth": 10, "m": 64, "table": 10_000_000, "vocab": 65_536},
        # decoding without drafts: one token of every sequence of a batch
        {"name": "append one token each", "op": "append", "n": 64, "m": 1, "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "longest": 4_000,
         "dtype": "bf16", "rotated": 128, "interleaved": False, "tree": False, "ragged": False},
        # prompts of different lengths, a rotation of half the head, neighbouring components in pairs, small pages
        {"name": "append prompts", "op": "append", "n": 5, "m": 2_047, "heads": 32, "kv_heads": 8, "d": 128, "page": 16, "longest": 1_001,
         "dtype": "fp16", "rotated": 64, "interleaved": True, "tree": False, "ragged": True},
        # one token of one sequence (latency)
        {"name": "attention of one token", "op": "attention", "n": 1, "m": 1, "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "longest": 2_049,
         "dtype": "bf16", "tree": False, "ragged": False},
        # one token of every sequence of a batch, long caches: bound by reading them
        {"name": "attention of a batch", "op": "attention", "n": 32, "m": 1, "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "longest": 16_384,
         "dtype": "bf16", "tree": False, "ragged": False},
        # full trees over middling caches: between reading and multiplying
        {"name": "attention of trees", "op": "attention", "n": 16, "m": 64, "heads": 32, "kv_heads": 8, "d": 128, "page": 32, "longest": 8_191,
         "dtype": "fp16", "tree": True, "ragged": True},
        # a piece of a prompt behind a cache: bound by multiplying
        {"name": "attention of a prompt", "op": "attention", "n": 1, "m": 1_024, "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "longest": 7_001,
         "dtype": "bf16", "tree": False, "ragged": False},
        # trees of neighbours' drafts against the model
        {"name": "verify trees", "op": "verify", "n": 16, "m": 64, "vocab": 65_536, "dtype": "bf16", "temperature": 1.0, "student": False,
         "greedy": False, "depth": 8},
        # what a distilled student drew, few tokens a sequence, a large odd vocabulary
        {"name": "verify a student's drafts", "op": "verify", "n": 33, "m": 6, "vocab": 131_071, "dtype": "bf16", "temperature": 0.8, "student": True,
         "greedy": False, "depth": 5},
        # one sequence's kept rows in all layers
        {"name": "keep of one sequence", "op": "keep", "layers": 32, "n": 1, "m": 24, "kv_heads": 8, "d": 128, "page": 64, "longest": 77,
         "dtype": "bf16", "depth": 6},
        # a batch's
        {"name": "keep of a batch", "op": "keep", "layers": 16, "n": 64, "m": 64, "kv_heads": 8, "d": 128, "page": 32, "longest": 201,
         "dtype": "fp16", "depth": 9},
    ]


def _log_int(rng, lo, hi):
    return lo if hi <= lo else int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["drafts", "append", "attention", "attention", "attention", "verify", "verify", "keep"])
    if op == "drafts":
        k = _log_int(rng, 1, 512)
        depth = rng.randint(1, 15)
        return {"op": op, "n": _log_int(rng, 1, min(1_024, 100_000_000 // (k * k * depth))), "k": k, "depth": depth, "m": rng.randint(2, 64),
                "table": _log_int(rng, 100_000, 10_000_000), "vocab": _log_int(rng, 1_000, 131_072)}
    if op == "verify":
        vocab, m = _log_int(rng, 1_000, 131_072), _log_int(rng, 1, 64)
        student = m > 1 and rng.random() < 0.4
        return {"op": op, "n": _log_int(rng, 1, max(1, min(64, 60_000_000 // (vocab * m)))), "m": m, "vocab": vocab, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                "temperature": rng.choice([1.0, 1.0, 0.7, 1.5]), "student": student, "greedy": not student and rng.random() < 0.3,
                "depth": m - 1 if student else rng.randint(1, 12)}
    heads = rng.choice([1, 2, 4, 8])
    case = {"op": op, "kv_heads": heads, "d": rng.choice([64, 80, 128, 128, 256]), "page": rng.choice([16, 32, 64, 128, 256]),
            "dtype": rng.choice(["bf16", "fp16"])}
    if op == "keep":
        case.update(layers=_log_int(rng, 1, 32), n=_log_int(rng, 1, 32), m=rng.randint(12, 64), longest=_log_int(rng, 1, 300), depth=rng.randint(1, 5))
        return case
    case["heads"] = heads * rng.choice([1, 2, 4, 5, 8])
    kind = rng.choice(["token", "tree", "tree", "prompt"])
    case["tree"] = kind == "tree"
    case["ragged"] = kind != "token" and rng.random() < 0.5
    case["m"] = 1 if kind == "token" else _log_int(rng, 2, 64) if kind == "tree" else _log_int(rng, 65, 1_024)
    if op == "append":
        most = 8_000_000 // (case["heads"] * case["d"] * case["m"])
        case.update(n=_log_int(rng, 1, max(1, min(64, most))), longest=_log_int(rng, 1, 4_000), interleaved=rng.random() < 0.5)
        case["rotated"] = rng.choice([0, 16, case["d"] // 2, case["d"], case["d"]])
        return case
    case["longest"] = _log_int(rng, 1, 16_384)
    reads = 40_000_000 // (case["longest"] * heads * case["d"] // 4 + 1)                                  # of the caches
    multiplies = 15_000_000_000 // ((case["longest"] + case["m"]) * case["m"] * case["heads"] * case["d"])
    case["n"] = _log_int(rng, 1, max(1, min(64, reads, multiplies)))
    return case


# ---- sizes that follow from a case alone

def _lens(case):
    """Places in the cache of each sequence: from the longest down to a quarter of it, and in a batch the last sequence is new."""
    n, longest = case["n"], case["longest"]
    lens = [longest - (longest * 3 * s) // (4 * n) for s in range(n)]
    if n > 2:
        lens[-1] = 0
    return lens


def _counts(case):
    """Used rows of each sequence: all, or from all down to a half, and none for one idle sequence of a batch."""
    n, m = case["n"], case["m"]
    if not case.get("ragged"):
        return [m] * n
    counts = [m - (m * s) // (2 * n) for s in range(n)]
    if n > 4:
        counts[n // 2] = 0
    return counts


def _kept(case):
    return [1 + (s + case["depth"] - 1) % case["depth"] for s in range(case["n"])]


# ---- inputs

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pages(case, rng, lens):
    """-> (pages [n][most], number of pages): pages in any order, room for all rows of the pass; unused entries are -1."""
    each = [-(-(at + case["m"]) // case["page"]) for at in lens]
    total = sum(each) + 3
    order = list(range(total))
    rng.shuffle(order)
    table, at = [], 0
    for count in each:
        table.append(order[at:at + count] + [NONE] * (max(each) - count))
        at += count
    return _int32(table), total


def _trees(rng, n, m, depth):
    """-> (parents, depths, place among the siblings), each [n][m]: the parent of a row is any earlier one that is not too deep."""
    parents, depths, ranks = [], [], []
    for _ in range(n):
        p, deep, rank, children = [NONE], [0], [0], [0] * m
        for j in range(1, m):
            up = rng.randrange(j)
            while deep[up] >= depth:
                up = p[up]
            p.append(up)
            deep.append(deep[up] + 1)
            rank.append(children[up])
            children[up] += 1
        parents.append(p)
        depths.append(deep)
        ranks.append(rank)
    return parents, depths, ranks


def _prepare_drafts(case, gen, rng, state):
    n, k, table, depth = case["n"], case["k"], case["table"], case["depth"]
    # a text in which the places of a few thousand phrases are the same tokens: neighbours agree on how it goes on, for some tokens
    phrases = (torch.rand(4_096, 16, generator=gen, device="cuda").pow_(4) * case["vocab"]).to(torch.int32)
    blocks = torch.randint(4_096, (table // 16 + 2,), generator=gen, device="cuda")
    text = phrases[blocks].reshape(-1)[:table].clone()
    text[torch.rand(table, generator=gen, device="cuda") < 0.05] = 7
    text[torch.rand(table, generator=gen, device="cuda") < 1e-3] = NONE                                  # ends of documents
    # the neighbours of a query are places of few phrases
    wanted = torch.randint(blocks.numel() - 2, (n, 6), generator=gen, device="cuda")
    same = torch.argsort(blocks)                                                                         # places by phrase
    rank = torch.argsort(same)
    which = torch.gather(wanted, 1, (torch.rand((n, k), generator=gen, device="cuda").pow_(2) * 6).long())
    near = same[(rank[which] + torch.randint(0, 64, (n, k), generator=gen, device="cuda")).clamp_(max=blocks.numel() - 1)]
    ids = (near * 16 + torch.randint(0, 3, (n, k), generator=gen, device="cuda")).clamp_(max=table - 1)
    steps = torch.rand((n, k), generator=gen, device="cuda").mul_(600.0)
    steps[:, 0] += 20_000.0
    dists = steps.cumsum(dim=1)                                                                          # ascending, as a search gives them
    short = (torch.rand((n, 1), generator=gen, device="cuda") < 0.05) & (torch.arange(k, device="cuda") >= k // 2)
    state.update(ids=ids.masked_fill_(short, -1), dists=dists.masked_fill_(short, math.inf), text=text, temperature=4_000.0,
                 last=torch.randint(case["vocab"], (n,), generator=gen, device="cuda").to(torch.int32))


def _prepare_cache(case, gen, rng, state):
    lens, kv_heads, d, page, dtype = _lens(case), case["kv_heads"], case["d"], case["page"], TYPES[case["dtype"]]
    state["pages"], total = _pages(case, rng, lens)
    state["lens"] = _int32(lens)
    state["counts"] = _int32(_counts(case)) if case.get("ragged") else None
    layers = (case["layers"],) if "layers" in case else ()
    shapes = (*layers, total, kv_heads, page, d), (*layers, total, kv_heads, page // 8, d, 8)
    if case["op"] == "append":
        state["k_cache"], state["v_cache"] = (torch.zeros(shape, dtype=dtype, device="cuda") for shape in shapes)
    else:
        state["k_cache"], state["v_cache"] = (torch.randn(shape, generator=gen, device="cuda", dtype=dtype) for shape in shapes)


def _prepare_verify(case, gen, rng, state):
    n, m, vocab = case["n"], case["m"], case["vocab"]
    bias = -0.5 * torch.log1p(torch.arange(vocab, device="cuda", dtype=torch.float32))
    logits = _normal(gen, n * m, vocab).mul_(2.5).add_(bias)                                             # frequent (low) tokens are likely
    likely = torch.topk(_normal(gen, n * m, vocab).mul_(3.0).add_(logits), 8, dim=1).indices
    logits.scatter_add_(1, likely[:, :1], torch.full((n * m, 1), 4.0, device="cuda"))                    # in most places one token stands out
    dtype = TYPES[case["dtype"]]
    state["logits"] = logits.to(dtype)
    state["uniforms"] = None if case["greedy"] else torch.rand((n, m), generator=gen, device="cuda")
    state["last"] = torch.randint(vocab, (n,), generator=gen, device="cuda").to(torch.int32)
    tokens = torch.empty((n, m), dtype=torch.int32, device="cuda")
    tokens[:, 0] = state["last"]
    state["parents"] = state["draft_logits"] = state["accept"] = None
    if case["student"]:
        drafts = logits.view(n, m, vocab)[:, :-1].reshape(n * (m - 1), vocab)
        drafts = (drafts + _normal(gen, n * (m - 1), vocab)).to(dtype)                                   # a student that is near the model
        gumbel = -torch.log(-torch.log(torch.rand(drafts.shape, generator=gen, device="cuda").clamp_(1e-9, 1 - 1e-7)))
        tokens[:, 1:] = (drafts.float() / case["temperature"] + gumbel).argmax(dim=1).view(n, m - 1)
        state.update(draft_logits=drafts, accept=torch.rand((n, m), generator=gen, device="cuda"))
    else:
        parents, _, ranks = _trees(rng, n, m, case["depth"])
        state["parents"] = _int32(parents)
        at = (torch.arange(n, device="cuda")[:, None] * m + state["parents"].clamp(min=0)).long()
        tokens[:, 1:] = likely[at, _int32(ranks).long() % 8][:, 1:].to(torch.int32)
    state["tokens"] = tokens


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = random.Random(int(seed))
    op, n, m = case["op"], case["n"], case["m"]
    state = {"case": case}
    if op == "drafts":
        _prepare_drafts(case, gen, rng, state)
        return state
    if op == "verify":
        _prepare_verify(case, gen, rng, state)
        return state
    _prepare_cache(case, gen, rng, state)
    if op == "keep":
        # kept rows that lie behind the places they go to, so that a second pass finds the same
        kept = _kept(case)
        paths = [[0] + sorted(rng.sample(range(count, m), count - 1)) + [NONE] * (m - count) for count in kept]
        state.update(path=_int32(paths), kept=_int32(kept))
        return state
    dtype, d, kv_heads = TYPES[case["dtype"]], case["d"], case["kv_heads"]
    state["parents"] = state["depths"] = None
    if case["tree"]:
        parents, depths, _ = _trees(rng, n, m, 8)
        state.update(parents=_int32(parents), depths=_int32(depths))
    state["q"] = _normal(gen, n, m, case["heads"], d).mul_(2.0).to(dtype)
    if op == "append":
        state["k"], state["v"] = (_normal(gen, n, m, kv_heads, d).to(dtype) for _ in range(2))
        half = case["rotated"] // 2
        state["inv_freq"] = torch.pow(10_000.0, -torch.arange(half, device="cuda", dtype=torch.float32) / half) if half else None
        state["amplitude"] = 1.0
    else:
        state["scale"] = d ** -0.5
    return state


# ---- the plain form

def _plain_drafts(state):
    case = state["case"]
    ids, dists, text = state["ids"], state["dists"], state["text"]
    n, k, m, depth = case["n"], case["k"], case["m"], case["depth"]
    table = text.shape[0]
    place = torch.arange(k, device=ids.device)
    used = (ids >= 0) & (ids < table) & torch.isfinite(dists)
    alive = used & (text[ids.clamp(0, table - 1)] >= 0)
    d = torch.where(alive, dists.double(), math.inf)
    nearest = d.amin(dim=1, keepdim=True)
    weight = torch.where(alive, torch.exp((nearest - d) / state["temperature"]), 0.0)
    weight = torch.round(torch.where(alive, weight, 0.0) * 2.0 ** 32).long()
    alive &= weight > 0
    total = weight.sum(dim=1, keepdim=True)
    same = torch.ones((n, k, k), dtype=torch.bool, device=ids.device)
    keys, tokens, ups, first = [], [], [], None
    for t in range(depth):
        at = ids + t
        alive &= at < table
        token = torch.where(alive, text[at.clamp(0, table - 1)], NONE)
        alive &= token >= 0
        same &= (token[:, :, None] == token[:, None, :]) & alive[:, :, None] & alive[:, None, :]
        through = torch.where(same, weight[:, None, :], 0).sum(dim=2)
        up = None if first is None else first + (t - 1) * k
        first = torch.where(same, place, k).amin(dim=2)
        is_first = alive & (first == place)
        keys.append(torch.where(is_first, (through << 14) | ((14 - t) << 10) | (1023 - place), 0))
        tokens.append(token)
        ups.append(torch.full_like(ids, NONE) if up is None else up)
    keys, tokens, ups = torch.cat(keys, dim=1), torch.cat(tokens, dim=1), torch.cat(ups, dim=1)
    rows = min(m - 1, keys.shape[1])
    best, node = torch.topk(keys, rows, dim=1)
    some = best > 0
    row_of = torch.zeros((n, keys.shape[1] + 1), dtype=torch.long, device=ids.device)
    row_of.scatter_(1, node, torch.arange(1, rows + 1, device=ids.device).expand(n, rows).contiguous())
    up = ups.gather(1, node)
    parent = torch.where(up < 0, 0, row_of.gather(1, up.clamp(min=0)))
    out = {"tokens": torch.full((n, m), NONE, dtype=torch.int32, device=ids.device), "parents": torch.full((n, m), NONE, dtype=torch.int32, device=ids.device),
           "depths": torch.zeros((n, m), dtype=torch.int32, device=ids.device), "logprobs": torch.full((n, m), -math.inf, device=ids.device)}
    out["tokens"][:, 0], out["logprobs"][:, 0] = state["last"], 0.0
    out["tokens"][:, 1:rows + 1] = torch.where(some, tokens.gather(1, node), NONE)
    out["parents"][:, 1:rows + 1] = torch.where(some, parent, NONE)
    out["depths"][:, 1:rows + 1] = torch.where(some, node // k + 1, 0)
    out["logprobs"][:, 1:rows + 1] = torch.where(some, torch.log((best >> 14).double() / total), -math.inf)
    out["counts"] = (1 + some.sum(dim=1)).to(torch.int32)
    return out


def _places(state):
    """-> for each row its page and its place in there, and whether the row is used."""
    case = state["case"]
    page = case["page"]
    row = torch.arange(case["m"], device="cuda")
    at = state["lens"].long()[:, None] + row
    used = torch.ones_like(at, dtype=torch.bool) if state["counts"] is None else row < state["counts"][:, None]
    return state["pages"].long().gather(1, at // page), at % page, used


def _plain_rotated(x, cos, sin, rotated, interleaved):
    y = x.float()
    part = y[..., :rotated]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :rotated // 2], part[..., rotated // 2:])
    turned = a * cos - b * sin, b * cos + a * sin
    part = torch.stack(turned, dim=-1).flatten(-2) if interleaved else torch.cat(turned, dim=-1)
    return torch.cat([part, y[..., rotated:]], dim=-1).to(x.dtype)


def _plain_append(state):
    case = state["case"]
    q, k, v, k_cache, v_cache = (state[name] for name in ("q", "k", "v", "k_cache", "v_cache"))
    page, at, used = _places(state)
    if case["rotated"]:
        row = torch.arange(case["m"], device=q.device) if state["depths"] is None else state["depths"]
        position = (state["lens"][:, None] + row).double()
        angle = position[:, :, None] * state["inv_freq"].double()                                        # far positions need 64 bits
        cos, sin = ((f(angle) * state["amplitude"]).float()[:, :, None, :] for f in (torch.cos, torch.sin))
        q, k = (_plain_rotated(x, cos, sin, case["rotated"], case["interleaved"]) for x in (q, k))
    on = used[:, :, None, None]
    k_cache[page, :, at] = torch.where(on, k, k_cache[page, :, at])
    v_cache[page, :, at // 8, :, at % 8] = torch.where(on, v, v_cache[page, :, at // 8, :, at % 8])
    return torch.where(on, q, 0.0), k_cache, v_cache


def _ancestors(parents):
    """[n][m][m]: whether column j is row i itself or one of its ancestors."""
    m = parents.shape[1]
    up = parents.long().clamp(min=0)[:, :, None] == torch.arange(m, device=parents.device)
    reach = (up & (parents >= 0)[:, :, None]).float() + torch.eye(m, device=parents.device)
    for _ in range(max(1, (m - 1).bit_length())):
        reach = (torch.bmm(reach, reach) > 0).float()
    return reach > 0


def _visible(state, places):
    """[n][m][places]: what each row sees of its sequence's places."""
    case = state["case"]
    m, lens = case["m"], state["lens"].long()
    at = torch.arange(places, device="cuda") - lens[:, None]
    if state["parents"] is None:
        inside = torch.ones((m, m), dtype=torch.bool, device="cuda").tril().expand(case["n"], m, m)
    else:
        inside = _ancestors(state["parents"])
    drafted = inside.gather(2, at.clamp(0, m - 1)[:, None, :].expand(-1, m, -1)) & ((at >= 0) & (at < m))[:, None, :]
    return drafted | (at < 0)[:, None, :]


def _cached(state):
    """Keys and values of every sequence as [n * kv_heads][places][d], in 32 bits; places without a page read page 0."""
    case = state["case"]
    n, kv_heads, d, page = case["n"], case["kv_heads"], case["d"], case["page"]
    pages = state["pages"].long().clamp(min=0)
    k = state["k_cache"][pages].permute(0, 2, 1, 3, 4).reshape(n * kv_heads, -1, d).float()
    v = state["v_cache"][pages].permute(0, 2, 1, 3, 5, 4).reshape(n * kv_heads, -1, d).float()
    return k, v


def _plain_attention(state):
    case, q = state["case"], state["q"]
    n, m, heads, kv_heads, d = case["n"], case["m"], case["heads"], case["kv_heads"], case["d"]
    group = heads // kv_heads
    k, v = _cached(state)
    places = k.shape[1]
    rows = q.view(n, m, kv_heads, group, d).permute(0, 2, 1, 3, 4).reshape(n * kv_heads, m * group, d).float()
    s = torch.bmm(rows, k.transpose(1, 2)).mul_(state["scale"])
    hidden = ~_visible(state, places)
    s.view(n, kv_heads, m, group, places).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    s = s.sub_(s.amax(dim=2, keepdim=True)).exp_()
    s = s.div_(s.sum(dim=2, keepdim=True))
    out = torch.bmm(s, v).view(n, kv_heads, m, group, d).permute(0, 2, 1, 3, 4).reshape(n, m, heads, d)
    if state["counts"] is not None:
        used = torch.arange(m, device=q.device) < state["counts"][:, None]
        out = torch.where(used[:, :, None, None], out, 0.0)
    return out.to(q.dtype)


def _pick(weights, uniforms):
    """The lowest place of each row whose weights up to there are over that share of their sum."""
    sums = weights.cumsum(dim=-1)
    return (sums <= uniforms.double().unsqueeze(-1) * sums[..., -1:]).sum(dim=-1).clamp_(max=weights.shape[-1] - 1)


def _plain_verify(state):
    case = state["case"]
    n, m, vocab, temperature = case["n"], case["m"], case["vocab"], case["temperature"]
    logits, tokens = state["logits"], state["tokens"].long()
    row = torch.arange(m, device=logits.device)
    seq = torch.arange(n, device=logits.device)

    def distribution(x):                                                                                 # in 64 bits: a sum's borders decide
        z = x.double()
        z = (z - z.amax(dim=1, keepdim=True)) / temperature
        e = z.exp()
        return z, e, e.sum(dim=1, keepdim=True)

    z, e, total = distribution(logits)
    path = torch.full((n, m), NONE, dtype=torch.long, device=logits.device)
    chosen = torch.full((n, m), NONE, dtype=torch.long, device=logits.device)
    path[:, 0] = 0
    if case["student"]:
        p = (e / total).view(n, m, vocab)
        _, e_q, total_q = distribution(state["draft_logits"])
        q = (e_q / total_q).view(n, m - 1, vocab)
        drafted = tokens[:, 1:, None]
        passes = state["accept"][:, 1:].double() * q.gather(2, drafted)[..., 0] < p[:, :-1].gather(2, drafted)[..., 0]
        kept = passes.long().cumprod(dim=1).sum(dim=1) + 1                                               # with row 0
        stop = kept - 1
        left = torch.where((kept < m)[:, None], (p[seq, stop] - q[seq, stop.clamp(max=m - 2)]).clamp_(min=0.0), p[seq, stop])
        left = torch.where(left.sum(dim=1, keepdim=True) > 0, left, p[seq, stop])
        following = _pick(left, state["uniforms"].gather(1, stop[:, None])[:, 0])
        path = torch.where(row < kept[:, None], row, NONE)
        chosen[:, :-1] = torch.where(row[:-1] < stop[:, None], tokens[:, 1:], NONE)
        chosen.scatter_(1, stop[:, None], following[:, None])
    else:
        best = logits.float().argmax(dim=1).view(n, m) if case["greedy"] else _pick(e.view(n, m, vocab), state["uniforms"])
        at, going = torch.zeros(n, dtype=torch.long, device=logits.device), torch.ones(n, dtype=torch.bool, device=logits.device)
        kept, following = torch.ones_like(at), torch.zeros_like(at)
        for step in range(min(case["depth"], m - 1) + 1):
            token = best[seq, at]
            chosen[:, step] = torch.where(going, token, NONE)
            following = torch.where(going, token, following)
            child = (state["parents"] == at[:, None]) & (tokens == token[:, None]) & (row > 0)
            going = going & child.any(dim=1)
            at = torch.where(going, child.float().argmax(dim=1), at)
            if step + 1 < m:
                path[:, step + 1] = torch.where(going, at, NONE)
            kept += going
    rows = seq[:, None] * m + path.clamp(min=0)
    logprobs = z[rows, chosen.clamp(min=0)] - total[rows, 0].log()
    return {"path": path.to(torch.int32), "kept": kept.to(torch.int32), "next_tokens": following.to(torch.int32),
            "logprobs": torch.where(path >= 0, logprobs, -math.inf).float()}


def _plain_keep(state):
    case = state["case"]
    k_cache, v_cache, path = state["k_cache"], state["v_cache"], state["path"].long()
    page, lens, pages = case["page"], state["lens"].long()[:, None], state["pages"].long()
    to = lens + torch.arange(case["m"], device=path.device)
    used = torch.arange(case["m"], device=path.device) < state["kept"][:, None]
    source = torch.where(used, lens + path, to)                                                          # other rows onto themselves
    from_page, to_page = pages.gather(1, source // page), pages.gather(1, to // page)
    source, to = source % page, to % page
    k_cache[:, to_page, :, to] = k_cache[:, from_page, :, source]
    v_cache[:, to_page, :, to // 8, :, to % 8] = v_cache[:, from_page, :, source // 8, :, source % 8]
    return k_cache, v_cache


def _plain(state):
    return {"drafts": _plain_drafts, "append": _plain_append, "attention": _plain_attention, "verify": _plain_verify, "keep": _plain_keep}[state["case"]["op"]](state)


# ---- the library's

def _own(state):
    import paper_2301_06672_amd as ivfpq
    case = state["case"]
    op = case["op"]
    if op == "drafts":
        got = ivfpq.ivfpq_neighbour_drafts(state["ids"], state["dists"], state["text"], state["last"], state["temperature"], depth=case["depth"], rows=case["m"])
        return {"tokens": got.tokens, "parents": got.parents, "depths": got.depths, "logprobs": got.logprobs, "counts": got.counts}
    if op == "verify":
        got = ivfpq.ivfpq_verify_drafts(state["logits"], state["tokens"], parents=state["parents"], uniforms=state["uniforms"], temperature=case["temperature"],
                                        draft_logits=state["draft_logits"], accept=state["accept"])
        return {"path": got.path, "kept": got.kept, "next_tokens": got.next_tokens, "logprobs": got.logprobs}
    k_cache, v_cache, pages, lens = (state[name] for name in ("k_cache", "v_cache", "pages", "lens"))
    if op == "keep":
        ivfpq.ivfpq_cache_keep(k_cache, v_cache, pages, lens, state["path"], state["kept"])
        return k_cache, v_cache
    if op == "append":
        q = ivfpq.ivfpq_cache_append(state["k"], state["v"], k_cache, v_cache, pages, lens, q=state["q"], inv_freq=state["inv_freq"], depths=state["depths"],
                                     counts=state["counts"], interleaved=case["interleaved"], amplitude=state["amplitude"])
        return q, k_cache, v_cache
    return ivfpq.ivfpq_draft_attention(state["q"], k_cache, v_cache, pages, lens, parents=state["parents"], counts=state["counts"], scale=state["scale"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without

def work(case):
    op, n, m = case["op"], case["n"], case["m"]
    if op == "drafts":
        return {"bytes": n * (case["k"] * (12 + 4 * case["depth"]) + 16 * m + 8), "flops": 4.0 * n * case["k"] * case["depth"]}
    if op == "verify":
        rows = n * m + (n * (m - 1) if case["student"] else 0)
        values = rows * case["vocab"]
        return {"bytes": (4 if case["dtype"] == "fp32" else 2) * values + 24 * n * m, "flops": (1.0 if case["greedy"] else 4.0) * values}
    row = 2 * case["kv_heads"] * case["d"] * 2                                                           # keys and values of one place
    if op == "keep":
        moved = sum(count - 1 for count in _kept(case)) * case["layers"]
        return {"bytes": 2 * moved * row + 4 * n * (m + 2), "flops": float(moved)}
    used = sum(_counts(case))
    q = case["heads"] * case["d"] * 2
    if op == "append":
        return {"bytes": used * (2 * q + 2 * row), "flops": 3.0 * used * case["rotated"] * (case["heads"] + case["kv_heads"])}
    seen = 0
    places = 0
    for length, count in zip(_lens(case), _counts(case)):
        places += length + count if count else 0
        seen += count * length + count * (9 if case["tree"] else count + 1) // 2
    return {"bytes": places * row + used * 2 * q, "flops": 4.0 * case["d"] * case["heads"] * seen}


# ---- the definition, in 64 bits

def _exact_drafts(state):
    case = state["case"]
    n, k, m, depth = case["n"], case["k"], case["m"], case["depth"]
    ids, dists, last = state["ids"].tolist(), state["dists"].double().tolist(), state["last"].tolist()
    table = state["text"].shape[0]
    at = (state["ids"].clamp(min=0)[:, :, None] + torch.arange(depth, device="cuda")).clamp_(max=table - 1)
    words = state["text"][at].tolist()
    out = {"tokens": torch.full((n, m), NONE, dtype=torch.int32), "parents": torch.full((n, m), NONE, dtype=torch.int32),
           "depths": torch.zeros((n, m), dtype=torch.int32), "logprobs": torch.full((n, m), -math.inf, dtype=torch.float64),
           "counts": torch.ones(n, dtype=torch.int32)}
    for s in range(n):
        out["tokens"][s, 0], out["logprobs"][s, 0] = last[s], 0.0
        valid = [j for j in range(k) if 0 <= ids[s][j] < table and math.isfinite(dists[s][j]) and words[s][j][0] >= 0]
        if not valid:
            continue
        nearest = min(dists[s][j] for j in valid)
        nodes, total = {}, 0
        for j in valid:
            w = round(math.exp((nearest - dists[s][j]) / state["temperature"]) * 2.0 ** 32)
            total += w
            prefix = ()
            for t in range(depth if w else 0):
                if ids[s][j] + t >= table or words[s][j][t] < 0:
                    break
                prefix += (words[s][j][t],)
                held = nodes.setdefault(prefix, [0, j])
                held[0] += w
        order = sorted(nodes, key=lambda prefix: (-nodes[prefix][0], len(prefix), nodes[prefix][1]))[:m - 1]
        row = {(): 0, **{prefix: i + 1 for i, prefix in enumerate(order)}}
        for prefix in order:
            i = row[prefix]
            out["tokens"][s, i], out["parents"][s, i], out["depths"][s, i] = prefix[-1], row[prefix[:-1]], len(prefix)
            out["logprobs"][s, i] = math.log(nodes[prefix][0] / total)
        out["counts"][s] = 1 + len(order)
    return out


def _exact_append(state):
    case = state["case"]
    q, k, v = (state[name].double() for name in ("q", "k", "v"))
    k_cache, v_cache = state["k_cache"].double(), state["v_cache"].double()
    page, half = case["page"], case["rotated"] // 2
    pages, lens, counts = state["pages"].tolist(), _lens(case), _counts(case)
    for s in range(case["n"]):
        count = counts[s]
        q[s, count:] = 0.0
        if not count:
            continue
        row = torch.arange(count, device="cuda")
        if half:
            depth = row if state["depths"] is None else state["depths"][s, :count]
            turn = torch.exp(1j * (lens[s] + depth).double()[:, None] * state["inv_freq"].double())[:, None, :]      # a pair as a complex number
            for x in (q[s, :count], k[s, :count]):
                a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
                pair = torch.complex(x[..., a], x[..., b]) * turn
                x[..., a], x[..., b] = pair.real, pair.imag
        at = lens[s] + row
        held = torch.tensor(pages[s], device="cuda")[at // page]
        k_cache[held, :, at % page] = k[s, :count]
        v_cache[held, :, (at % page) // 8, :, at % 8] = v[s, :count]
    return q, k_cache, v_cache


def _exact_attention(state):
    case = state["case"]
    n, m, heads, kv_heads, d, page = (case[name] for name in ("n", "m", "heads", "kv_heads", "d", "page"))
    group = heads // kv_heads
    out = torch.zeros((n, m, heads, d), dtype=torch.float64, device="cuda")
    for s, (length, count) in enumerate(zip(_lens(case), _counts(case))):
        if not count:
            continue
        held = state["pages"][s].long()[:-(-(length + count) // page)]
        k = state["k_cache"][held].double().transpose(0, 1).reshape(kv_heads, -1, d)[:, :length + count]
        v = state["v_cache"][held].double().permute(1, 0, 2, 4, 3).reshape(kv_heads, -1, d)[:, :length + count]
        sees = torch.ones((count, length + count), dtype=torch.bool, device="cuda")
        if state["parents"] is None:
            sees[:, length:] = torch.ones((count, count), dtype=torch.bool).tril().cuda()
        else:
            inside = torch.zeros((count, count), dtype=torch.bool)
            for i, up in enumerate(state["parents"][s, :count].tolist()):
                if up >= 0:
                    inside[i] = inside[up]
                inside[i, i] = True
            sees[:, length:] = inside.cuda()
        for h in range(heads):
            score = (state["q"][s, :count, h].double() @ k[h // group].t().contiguous()) * state["scale"]
            out[s, :count, h] = torch.softmax(score.masked_fill(~sees, -math.inf), dim=1) @ v[h // group]
    return out


def _exact_verify(state):
    case = state["case"]
    n, m = case["n"], case["m"]
    tokens = state["tokens"].tolist()
    parents = None if state["parents"] is None else state["parents"].tolist()
    uniforms = None if state["uniforms"] is None else state["uniforms"].double().tolist()
    accept = None if state["accept"] is None else state["accept"].double().tolist()
    path = torch.full((n, m), NONE, dtype=torch.int32)
    logprobs = torch.full((n, m), -math.inf, dtype=torch.float64)
    kept, following = torch.zeros(n, dtype=torch.int32), torch.zeros(n, dtype=torch.int32)

    def softmax(x):
        return torch.softmax(x.cpu().double() / case["temperature"], dim=0)

    def sample(p, u):
        sums = p.cumsum(dim=0)
        return min(int(torch.searchsorted(sums, sums[-1:] * u, right=True)), p.numel() - 1)

    for s in range(n):
        at, count = 0, 0
        while True:
            path[s, count] = at
            row = state["logits"][s * m + at]
            p = softmax(row)
            child = None
            if case["student"]:
                token = tokens[s][at + 1] if at + 1 < m else None
                if token is not None:
                    q = softmax(state["draft_logits"][s * (m - 1) + at])
                    if accept[s][at + 1] * float(q[token]) < float(p[token]):
                        child = at + 1
                    else:
                        left = (p - q).clamp(min=0.0)
                        token = sample(left if float(left.sum()) > 0 else p, uniforms[s][at])
                else:
                    token = sample(p, uniforms[s][at])
            else:
                token = int(row.cpu().float().argmax()) if case["greedy"] else sample(p, uniforms[s][at])
                child = next((j for j in range(1, m) if parents[s][j] == at and tokens[s][j] == token), None)
            logprobs[s, count] = torch.log(p[token])
            count += 1
            if child is None:
                kept[s], following[s] = count, token
                break
            at = child
    return {"path": path, "kept": kept, "next_tokens": following, "logprobs": logprobs}


def _exact_keep(state):
    case = state["case"]
    k_cache, v_cache = state["k_cache"].double(), state["v_cache"].double()
    path, pages, page = state["path"].tolist(), state["pages"].tolist(), case["page"]
    for s, (length, kept) in enumerate(zip(_lens(case), _kept(case))):
        for i in range(kept):
            a, b = length + path[s][i], length + i
            k_cache[:, pages[s][b // page], :, b % page] = k_cache[:, pages[s][a // page], :, a % page]
            v_cache[:, pages[s][b // page], :, b % page // 8, :, b % 8] = v_cache[:, pages[s][a // page], :, a % page // 8, :, a % 8]
    return k_cache, v_cache


def exact(case, seed):
    state = prepare(case, seed)
    return {"drafts": _exact_drafts, "append": _exact_append, "attention": _exact_attention, "verify": _exact_verify, "keep": _exact_keep}[case["op"]](state)
