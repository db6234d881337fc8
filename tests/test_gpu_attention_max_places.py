"""ivfpq_draft_attention whose max_places is not what the longest sequence has: it decides how the work is divided, never what is seen."""
import pytest
import torch

from test_gpu_draft_attention import BF16, FP16, check, fill_rows, queries
from util_drafts import Cache, tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


@pytest.mark.parametrize("m,share,d,trees", [(1, 4, 128, False), (5, 2, 80, True), (40, 1, 64, True), (64, 3, 128, True), (70, 2, 64, False), (20, 1, 256, False)])
@pytest.mark.parametrize("max_places", [0, 1, 100, 256, 400, 10 ** 6])
def test_places_behind_the_bound_are_seen(P, m, share, d, trees, max_places):
    lens = [700, 0, 130, 321]
    cache = fill_rows(Cache(lens, m, 1, d, 32, FP16 if d == 64 else BF16, seed=m))
    check(P, queries(len(lens), m, share, d, cache.dtype), cache, parents=tree(len(lens), m, 3) if trees else None, max_places=max_places)


@pytest.mark.parametrize("m", [1, 9])
def test_graph_over_growing_sequences(P, m):
    """A call that was captured over short sequences, its bound among them, is replayed as they grow."""
    cache = fill_rows(Cache([2_000, 1_500], m, 2, 128, 64, BF16, seed=2))
    k, v, table, lens = cache.gpu()
    q = queries(2, m, 4, 128, BF16).cuda()
    call = lambda bound: P.ivfpq_draft_attention(q, k, v, table, lens, max_places=bound)
    lens.copy_(torch.tensor([300, 30], dtype=torch.int32))
    call(300 + m)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(300 + m)
    for grown in ([300, 30], [301, 31], [1_000, 64], [2_000, 1_500]):
        lens.copy_(torch.tensor(grown, dtype=torch.int32))
        eager = call(300 + m)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    check(P, q.cpu(), cache, max_places=300 + m)                       # what the last replay was compared with is right itself
    assert torch.equal(out, P.ivfpq_draft_attention(q, k, v, table, cache.lens().cuda(), max_places=300 + m))


def test_table_of_more_tiles_than_are_numbered(P):
    """40 sequences of 1.7 10^9 places would be 2^31 tiles: not dealt to parts, and right all the same."""
    lens, m, page = [90] * 39 + [2_600], 2, 256
    cache = fill_rows(Cache(lens, m, 1, 64, page, BF16, seed=7))
    q = queries(len(lens), m, 2, 64, BF16)
    k, v, table, lengths = cache.gpu()
    most = 2 ** 31 * 32 // 40 // page + 1
    assert len(lens) * (most * page // 32 + 2) >= 2 ** 31
    wide = torch.full((len(lens), most), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    bounded = P.ivfpq_draft_attention(q.cuda(), k, v, wide, lengths, max_places=2_602)
    del wide
    assert torch.equal(bounded, P.ivfpq_draft_attention(q.cuda(), k, v, table, lengths, max_places=0))       # not divided either
    check(P, q, cache, max_places=0)
