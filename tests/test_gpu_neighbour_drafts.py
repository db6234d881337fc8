"""ivfpq_neighbour_drafts against trees of dictionaries, weights as the whole numbers that they are.

Tokens, parents, depths and counts are equal.  The random data keeps weights of different beginnings apart by more than one unit in 2^32 (ties are exact:
equal distances).  A log-probability is one rounding of a 64-bit number: half a step of fp32, and the weights' own units (an exp of 64 bits
may round to a neighbouring unit: 2^-32 of the nearest neighbour's weight, of k neighbours, relative to the node's)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def plain(ids, dists, text, last, temperature, depth, m):
    n, k = ids.shape
    table, words = text.numel(), text.tolist()
    rows = []
    for s in range(n):
        near = [(int(i), float(d)) for i, d in zip(ids[s], dists[s].double())]
        valid = [j for j, (i, d) in enumerate(near) if 0 <= i < table and math.isfinite(d) and words[i] >= 0]
        nodes, total = {}, 0
        if valid:
            low = min(near[j][1] for j in valid)
            for j in valid:
                w = round(math.exp((low - near[j][1]) / temperature) * 2.0 ** 32)
                total += w
                prefix = ()
                for t in range(depth if w else 0):
                    at = near[j][0] + t
                    if at >= table or words[at] < 0:
                        break
                    prefix += (words[at],)
                    nodes.setdefault(prefix, [0, j])[0] += w
        order = sorted(nodes, key=lambda p: (-nodes[p][0], len(p), nodes[p][1]))[:m - 1]
        row = {(): 0, **{p: i + 1 for i, p in enumerate(order)}}
        pad = m - 1 - len(order)
        rows.append(([int(last[s])] + [p[-1] for p in order] + [-1] * pad, [-1] + [row[p[:-1]] for p in order] + [-1] * pad,
                     [0] + [len(p) for p in order] + [0] * pad, [0.0] + [math.log(nodes[p][0] / total) for p in order] + [-math.inf] * pad, 1 + len(order),
                     [1.0] + [nodes[p][0] / 2.0 ** 32 for p in order] + [1.0] * pad))
    return [torch.tensor(x, dtype=torch.float64 if i in (3, 5) else torch.int32).reshape((n, m) if i != 4 else (n,)) for i, x in enumerate(zip(*rows))]


def check(P, ids, dists, text, last, temperature, depth, m):
    got = P.ivfpq_neighbour_drafts(ids.cuda(), dists.cuda(), text.cuda(), last.cuda(), temperature, depth=depth, rows=m)
    tokens, parents, depths, logprobs, counts, weights = plain(ids, dists, text, last, temperature, depth, m)
    assert torch.equal(got.counts.cpu(), counts)
    assert torch.equal(got.tokens.cpu(), tokens) and torch.equal(got.parents.cpu(), parents) and torch.equal(got.depths.cpu(), depths)
    lp = got.logprobs.cpu().double()
    assert torch.equal(torch.isneginf(lp), torch.isneginf(logprobs))
    fine = torch.isfinite(logprobs)
    off = torch.where(fine, (lp - logprobs).abs(), 0.0)
    most = 2.0 ** -24 * torch.where(fine, logprobs, 0.0).abs() + 2 * ids.shape[1] * 2.0 ** -32 / weights.clamp(min=2.0 ** -32)
    assert bool((off <= most).all()), float((off - most).max())
    return got


def inputs(n, k, table, vocab, seed, phrases=50):
    """A text that repeats some phrases, and neighbours at their beginnings."""
    gen = torch.Generator().manual_seed(seed)
    phrase = torch.randint(vocab, (phrases, 12), generator=gen)
    phrase[1::2, :5] = phrase[0::2, :5]                                  # phrases that begin alike
    which = torch.randint(phrases, (table // 12 + 1,), generator=gen)
    text = phrase[which].reshape(-1)[:table].clone()
    text[torch.rand(table, generator=gen) < 0.02] = -1
    few = torch.randint(phrases, (n, 5), generator=gen)
    ids = torch.randint(table, (n, k), generator=gen)
    for s in range(n):
        starts = torch.nonzero(torch.isin(which, few[s]))[:, 0] * 12
        if len(starts):
            pick = starts[torch.randint(len(starts), (k,), generator=gen)] + torch.randint(3, (k,), generator=gen)
            ids[s] = torch.where(torch.rand(k, generator=gen) < 0.8, pick.clamp(max=table - 1), ids[s])
    dists = torch.rand(n, k, generator=gen).cumsum(dim=1) * 3.0
    last = torch.randint(vocab, (n,), generator=gen).int()
    return ids, dists, text.int(), last


@pytest.mark.parametrize("k", [1, 2, 31, 64, 65, 128, 129, 256, 257, 700, 1024])
@pytest.mark.parametrize("depth,m", [(1, 64), (6, 24), (15, 64), (4, 2), (7, 1)])
def test_trees(P, k, depth, m):
    check(P, *inputs(7, k, 3_000, 100, seed=k + depth), 20.0, depth, m)


@pytest.mark.parametrize("k", [40, 100, 300, 1024])
def test_nothing_in_common(P, k):
    """Every continuation is another: more nodes than any list holds."""
    gen = torch.Generator().manual_seed(k)
    text = torch.randperm(50_000, generator=gen).int()
    ids = torch.randint(40_000, (5, k), generator=gen)
    dists = torch.rand(5, k, generator=gen) * 3
    got = check(P, ids, dists, text, torch.zeros(5, dtype=torch.int32), 1.0, 15, 64)
    assert (got.counts == 64).all()


def test_ties(P):
    """Equal weights: the shallower node, then the earlier neighbour."""
    text = torch.arange(1_000).int()
    ids = torch.tensor([[10, 500, 30, 10, 30, 700], [5, 6, 7, 8, 9, 5]])
    dists = torch.ones(2, 6)
    for m in (2, 5, 9, 30):
        check(P, ids, dists, text, torch.tensor([3, 4], dtype=torch.int32), 1.0, 5, m)


def test_unused_neighbours(P):
    """Padding, infinite and NaN distances, ids out of range, texts that end."""
    text = torch.tensor([4, 5, -1, 6, 7, 8, 9, 6, 7, 5])
    ids = torch.tensor([[-1, -1, -1], [2, 10, 11], [9, 8, 7], [0, 3, 7], [2 ** 62, -2 ** 62, 3], [3, 3, 3]])
    dists = torch.tensor([[1.0, 1.0, 1.0], [1.0, 1.0, 1.0], [1.0, 2.0, 3.0], [math.inf, math.nan, 5.0], [0.0, 0.0, -1.0], [-3e38, 3e38, 1.0]])
    got = check(P, ids, dists, text.int(), torch.arange(6).int(), 2.0, 6, 12)
    assert got.counts.tolist()[:2] == [1, 1]
    check(P, ids, dists, text.int(), torch.arange(6).int(), 1e30, 6, 12)
    check(P, ids, dists, text.int(), torch.arange(6).int(), 1e-30, 6, 12)


def test_empty(P):
    none = torch.empty((0, 5), dtype=torch.int64, device="cuda")
    got = P.ivfpq_neighbour_drafts(none, torch.empty((0, 5), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), 1.0)
    assert got.tokens.shape == (0, 64)
    got = P.ivfpq_neighbour_drafts(torch.zeros((2, 5), dtype=torch.int64, device="cuda"), torch.zeros((2, 5), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"),
                                   torch.tensor([7, 8], dtype=torch.int32, device="cuda"), 1.0, rows=3)
    assert got.tokens.tolist() == [[7, -1, -1], [8, -1, -1]] and got.counts.tolist() == [1, 1]


def test_same_bits_and_graph(P):
    ids, dists, text, last = (x.cuda() for x in inputs(50, 300, 3_000, 40, seed=1))
    call = lambda: P.ivfpq_neighbour_drafts(ids, dists, text, last, 20.0, depth=10)
    first = call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in range(1, 4):
        for to, x in zip((ids, dists, text, last), inputs(50, 300, 3_000, 40, seed=seed)):
            to.copy_(x)
        eager = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
        if seed == 1:
            assert all(torch.equal(a, b) for a, b in zip(first, eager))
