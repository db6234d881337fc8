"""The calls around drafted tokens as they are used together: prompts into the cache, a search, trees of the neighbours' drafts, two layers over them, verification, the
kept rows moved up, and the next token behind them.  Every step is compared with its plain form on what the step before it gave; the first layer's cache, whose keys and
values are those of the tokens alone, has to hold afterwards, bit for bit, what a pass without drafts writes."""
import pytest
import torch

from test_gpu_draft_attention import allowed
from test_gpu_neighbour_drafts import plain as plain_drafts
from test_gpu_verify import plain as plain_verify
from util_drafts import plain_attention

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
VOCAB, HEADS, KV_HEADS, D, PAGE, LAYERS = 200, 4, 2, 64, 16, 2
WIDTH = HEADS * D


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


class Model:
    def __init__(self, P, seed=1):
        gen = torch.Generator().manual_seed(seed)
        normal = lambda *shape, size=1.0: (torch.randn(*shape, generator=gen) * size).to(BF16).cuda()
        self.P, self.embedding = P, normal(VOCAB, WIDTH)
        self.wq, self.wk, self.wv, self.wo = (normal(LAYERS, WIDTH, n, size=WIDTH ** -0.5) for n in (WIDTH, KV_HEADS * D, KV_HEADS * D, WIDTH))
        self.head = P.ivfpq_quantize_rows(normal(VOCAB, WIDTH, size=0.3))
        self.first = [(self.embedding @ w[0]) for w in (self.wq, self.wk, self.wv)]      # of every token, so that a row's numbers do not depend on its batch
        self.inv_freq = (10_000.0 ** (-torch.arange(D // 2, dtype=torch.float32) / (D // 2))).cuda()

    def run(self, tokens, k, v, pages, lens, trees=None, counts=None, layers=LAYERS, seen=None):
        """-> logits [n * m][vocab] of a pass over caches [layers][...]; seen: is given each attention call's arguments and result."""
        P, (n, m) = self.P, tokens.shape
        at = tokens.clamp(min=0).long()
        x = self.embedding[at]
        for layer in range(layers):
            if layer == 0:
                q, key, value = (table[at] for table in self.first)
            else:
                q, key, value = (x @ w[layer] for w in (self.wq, self.wk, self.wv))
            q, key, value = q.view(n, m, HEADS, D), key.view(n, m, KV_HEADS, D), value.view(n, m, KV_HEADS, D)
            q = P.ivfpq_cache_append(key, value, k[layer], v[layer], pages, lens, q=q, inv_freq=self.inv_freq, depths=None if trees is None else trees.depths, counts=counts)
            out = P.ivfpq_draft_attention(q, k[layer], v[layer], pages, lens, parents=None if trees is None else trees.parents, counts=counts)
            if seen is not None:
                seen(q, k[layer], v[layer], out)
            x = x + (out.view(n, m, WIDTH) @ self.wo[layer] if layers > 1 else out.view(n, m, WIDTH))
        codes, scales = P.ivfpq_quantize_rows(x.reshape(n * m, WIDTH))
        return P.ivfpq_q8_matmul(codes, scales, *self.head)


def caches(n, places, layers=LAYERS):
    each = -(-places // PAGE)
    pages = torch.randperm(n * each, generator=torch.Generator().manual_seed(3)).view(n, each).int().cuda()
    k = torch.full((layers, n * each + 1, KV_HEADS, PAGE, D), float("nan"), dtype=BF16, device="cuda")
    v = torch.full((layers, n * each + 1, KV_HEADS, PAGE // 8, D, 8), float("nan"), dtype=BF16, device="cuda")
    return k, v, pages


def search(P, n, k=16):
    """Hidden states of a text, an index of them, and the neighbours of states near some of them."""
    gen = torch.Generator().manual_seed(5)
    phrases = torch.randint(VOCAB, (30, 8), generator=gen)
    which = torch.randint(30, (700,), generator=gen)
    text = phrases[which].reshape(-1).int()
    vectors = torch.randn(30, 8, 64, generator=gen)
    states = vectors[which].reshape(-1, 64) + 0.05 * torch.randn(700 * 8, 64, generator=gen)
    index = P.Index.ivfpq_build_device(states.cuda(), n_lists=32, pq_dim=32, pq_bits=8, kmeans_iters=5, seed=1).ivfpq_upload()
    asked = (states[torch.randint(5_000, (n,), generator=gen)] + 0.05 * torch.randn(n, 64, generator=gen)).cuda()
    ids, dists = index.ivfpq_search(asked, n_probes=8, k=k)
    index.ivfpq_free()
    return ids, dists, text.cuda()


@pytest.mark.parametrize("greedy", [False, True])
def test_a_pass_over_drafts(P, greedy):
    n, m, places = 3, 20, 96
    model = Model(P)
    k, v, pages = caches(n, places)
    gen = torch.Generator().manual_seed(7)
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    prompts = torch.randint(VOCAB, (n, 41), generator=gen, dtype=torch.int32).cuda()
    counts = torch.tensor([41, 17, 32], dtype=torch.int32, device="cuda")

    def seen(parents, counts):
        def compare(q, k_layer, v_layer, out):
            want, _, size, reach = plain_attention(q.cpu(), k_layer.cpu(), v_layer.cpu(), pages.cpu(), lens.cpu(), None if parents is None else parents.cpu(),
                                                   None if counts is None else counts.cpu())
            assert bool(((out.cpu().double() - want).abs() <= allowed(BF16, D, places, want, size, reach)).all())
        return compare

    model.run(prompts, k, v, pages, lens, counts=counts, seen=seen(None, counts))
    lens += counts

    ids, dists, text = search(P, n)
    last = torch.randint(VOCAB, (n,), generator=gen, dtype=torch.int32).cuda()
    trees = P.ivfpq_neighbour_drafts(ids, dists, text, last, 2.0, depth=6, rows=m)
    want = plain_drafts(ids.cpu(), dists.cpu(), text.cpu(), last.cpu(), 2.0, 6, m)
    assert all(torch.equal(got.cpu(), x) for got, x in zip((trees.tokens, trees.parents, trees.depths, trees.counts), want[:3] + want[4:5]))
    assert (trees.counts > 5).all()

    logits = model.run(trees.tokens, k, v, pages, lens, trees=trees, counts=trees.counts, seen=seen(trees.parents, trees.counts))
    # the model likes what the first draft says, so that something is kept
    for s in range(n):
        row = 0
        for _ in range(3):
            child = next((j for j in range(1, int(trees.counts[s])) if int(trees.parents[s, j]) == row), None)
            if child is None:
                break
            logits[s * m + row, int(trees.tokens[s, child])] = float(logits.max()) + 20.0
            row = child
    uniforms = None if greedy else torch.rand(n, m, generator=gen).cuda()
    got = P.ivfpq_verify_drafts(logits, trees.tokens, parents=trees.parents, counts=trees.counts, uniforms=uniforms)
    path, kept, following, _ = plain_verify(logits.cpu(), trees.tokens.cpu(), trees.parents.cpu(), trees.counts.cpu(), None if greedy else uniforms.cpu(), 1.0, None, None)
    assert torch.equal(got.path.cpu(), path) and torch.equal(got.kept.cpu(), kept) and torch.equal(got.next_tokens.cpu(), following)
    assert (kept >= 2).all()
    P.ivfpq_cache_keep(k, v, pages, lens, got.path, got.kept)

    # without drafts: the kept tokens behind each other
    plain_k, plain_v, _ = caches(n, places)
    zero = torch.zeros_like(lens)
    longest = int((counts + got.kept).max())
    tokens = torch.zeros((n, longest), dtype=torch.int32)
    for s in range(n):
        said = [int(trees.tokens[s, i]) for i in path[s, :kept[s]].tolist()]
        tokens[s, :int(counts[s]) + len(said)] = torch.tensor(prompts[s, :int(counts[s])].tolist() + said, dtype=torch.int32)
    model.run(tokens.cuda(), plain_k, plain_v, pages, zero, counts=counts + got.kept, layers=1)
    lens += got.kept
    for s in range(n):
        at = torch.arange(int(lens[s]), device="cuda")
        page, off = pages[s, at // PAGE].long(), at % PAGE
        assert torch.equal(k[0][page, :, off], plain_k[0][page, :, off])
        assert torch.equal(v[0][page, :, off // 8, :, off % 8], plain_v[0][page, :, off // 8, :, off % 8])

    logits = model.run(got.next_tokens[:, None].contiguous(), k, v, pages, lens, seen=seen(None, None))
    assert torch.isfinite(logits).all()


def test_a_pass_replayed_from_a_graph(P):
    """Drafts to kept rows in one graph, several times with other contents, eager passes in between; a second graph shares the memory pool of the first."""
    n, m = 3, 12
    model = Model(P)
    ids, dists, text = search(P, n)
    k, v, pages = caches(n, 80, layers=1)
    k.copy_(torch.randn(k.shape, generator=torch.Generator().manual_seed(1)).to(BF16))
    v.copy_(torch.randn(v.shape, generator=torch.Generator().manual_seed(2)).to(BF16))
    lens = torch.tensor([3, 40, 16], dtype=torch.int32, device="cuda")
    last, uniforms = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, m, device="cuda")

    def call():
        trees = P.ivfpq_neighbour_drafts(ids, dists, text, last, 2.0, depth=6, rows=m)
        logits = model.run(trees.tokens, k, v, pages, lens, trees=trees, counts=trees.counts, layers=1)
        got = P.ivfpq_verify_drafts(logits, trees.tokens, parents=trees.parents, counts=trees.counts, uniforms=uniforms)
        P.ivfpq_cache_keep(k, v, pages, lens, got.path, got.kept)
        return (*trees, logits, *got)

    start = k.clone(), v.clone()
    call()
    torch.cuda.synchronize()
    graphs, held = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0].pool() if graphs else None):
            held.append(call())
        graphs.append(graph)
    for turn in range(4):
        gen = torch.Generator().manual_seed(turn)
        last.copy_(torch.randint(VOCAB, (n,), generator=gen, dtype=torch.int32))
        uniforms.copy_(torch.rand(n, m, generator=gen))
        lens.copy_(torch.randint(0, 60, (n,), generator=gen, dtype=torch.int32))
        k.copy_(start[0]), v.copy_(start[1])
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in held[turn % 2]] + [k.clone(), v.clone()]
        k.copy_(start[0]), v.copy_(start[1])
        eager = [*call(), k, v]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, eager))
