"""ivfpq_draft_attention against a plain implementation in 64 bits: head layouts, trees and chains, pages that end inside of tiles, lengths of zero and one,
what must not have an influence (NaNs and infinities in places that a row does not see), missing pages, strides, graphs, streams.

Tolerance.  A weight is rounded to the cache's type, half a step off, and so is the result; a score is a sum of d products in fp32 (each addition off by
2^-24 of what the sum holds, at most the sum of |q||k|), and an error e of the scores changes weights by a factor of exp(2 e) at most.  fp16
cuts weights under 2^-30 of the largest by 2^-31: at most that many times the number of places of the values' size, and values of fp16 results
under 2^-14 have steps of 2^-24."""
import math

import pytest
import torch

from util_drafts import Cache, half_step, plain_attention, tree

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def allowed(dtype, d, places, out, size, reach):
    u = half_step(dtype)
    scores = math.expm1(min(2 * (d + 4) * 2.0 ** -24 * float(reach.max()) + 2.0 ** -18, 1.0))       # and 2^-18 for exp2 of numbers up to 2^5
    tiny = 2.0 ** -25 if dtype == FP16 else 0.0
    biggest = float(size[torch.isfinite(size)].max()) if torch.isfinite(size).any() else 0.0
    return (u + scores) * size + u * out.abs() * (1 + 2 * u) + tiny + places * 2.0 ** -31 * biggest


def check(P, q, cache, parents=None, counts=None, scale=None, max_places=None, pages=None, lens=None):
    k, v, table, lengths = cache.gpu()
    table = table if pages is None else pages.cuda()
    lengths = lengths if lens is None else lens.cuda()
    got, lse = P.ivfpq_draft_attention(q.cuda(), k, v, table, lengths, parents=None if parents is None else parents.cuda(),
                                       counts=None if counts is None else counts.cuda(), scale=scale, max_places=max_places, with_lse=True)
    want, want_lse, size, reach = plain_attention(q, cache.k, cache.v, table.cpu(), lengths.cpu(), parents, counts, scale)
    got, lse = got.cpu().double(), lse.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = torch.isfinite(want)
    off = torch.where(fine, (got - want).abs(), 0.0)
    most = allowed(cache.dtype, cache.d, int(lengths.max()) + cache.m, torch.where(fine, want, 0.0), torch.where(fine, size, 0.0), torch.where(torch.isfinite(reach), reach, 0.0))
    assert bool((off <= most).all()), (float((off - most).max()), float(off.max()))
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    same = torch.isfinite(want_lse)
    assert torch.equal(torch.isneginf(lse), torch.isneginf(want_lse))
    lse_off = torch.where(same, (lse - want_lse).abs(), 0.0)
    sure = torch.where(torch.isfinite(reach[..., 0]), reach[..., 0], 0.0)
    assert bool((lse_off <= (cache.d + 4) * 2.0 ** -24 * sure + 2.0 ** -18 + 2.0 ** -22 * torch.where(same, want_lse, 0.0).abs()).all()), float(lse_off.max())
    return got


def queries(n, m, heads, d, dtype, seed=5, size=1.0):
    return (torch.randn(n, m, heads, d, generator=torch.Generator().manual_seed(seed)) * size).to(dtype)


LENS = [0, 1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 129]


def fill_rows(cache, seed=9, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    for s, length in enumerate(cache.lens_list):
        for i in range(cache.m):
            cache.put(s, max(length, 0) + i, torch.randn(cache.kv_heads, cache.d, generator=gen) * scale, torch.randn(cache.kv_heads, cache.d, generator=gen))
    return cache


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("d,kv_heads,share", [(128, 2, 4), (64, 1, 1), (256, 1, 3), (80, 3, 2), (8, 2, 1), (200, 1, 16), (120, 1, 20)])
def test_single_tokens(P, dtype, page, d, kv_heads, share):
    cache = fill_rows(Cache(LENS, 1, kv_heads, d, page, dtype, seed=d + page))
    check(P, queries(len(LENS), 1, kv_heads * share, d, dtype), cache)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("m,d,kv_heads,share", [(2, 128, 1, 1), (5, 64, 2, 2), (17, 128, 1, 2), (31, 80, 2, 1), (33, 256, 1, 1), (64, 128, 1, 4), (64, 64, 1, 5), (63, 256, 2, 2), (64, 40, 1, 1)])
def test_trees(P, dtype, page, m, d, kv_heads, share):
    lens = LENS[::2]
    cache = fill_rows(Cache(lens, m, kv_heads, d, page, dtype, seed=m))
    check(P, queries(len(lens), m, kv_heads * share, d, dtype, size=2.0), cache, parents=tree(len(lens), m, m))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("m,d,kv_heads,share,page", [(2, 64, 1, 2, 16), (65, 128, 1, 1, 32), (130, 128, 1, 3, 16), (100, 256, 1, 1, 64), (257, 48, 1, 1, 16)])
def test_chains(P, dtype, m, d, kv_heads, share, page):
    lens = [0, 1, 40, 95]
    cache = fill_rows(Cache(lens, m, kv_heads, d, page, dtype, seed=m))
    check(P, queries(len(lens), m, kv_heads * share, d, dtype), cache)


@pytest.mark.parametrize("parents", [False, True])
def test_counts(P, parents):
    """Unused rows are zero, and neither they nor their places are read."""
    lens, m, d = [3, 0, 33, 64, 7, 20], 40, 64
    counts = torch.tensor([40, 1, 0, 17, -5, 99], dtype=torch.int32)
    cache = Cache(lens, m, 2, d, 16, BF16, seed=1)
    gen = torch.Generator().manual_seed(2)
    for s, length in enumerate(lens):
        for i in range(min(max(int(counts[s]), 0), m)):
            cache.put(s, length + i, torch.randn(2, d, generator=gen), torch.randn(2, d, generator=gen))
    q = queries(len(lens), m, 4, d, BF16)
    for s in range(len(lens)):
        q[s, min(max(int(counts[s]), 0), m):] = math.nan
    got = check(P, q, cache, parents=tree(len(lens), m, 3) if parents else None, counts=counts)
    assert (got[2] == 0).all() and (got[3, 17:] == 0).all() and (got[4] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("share,d", [(1, 64), (4, 128), (8, 80), (2, 256)])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_other_branches_have_no_influence(P, dtype, share, d, what):
    """Infinities and NaNs in the keys or values of rows that a row does not see."""
    m, lens = 24, [0, 5, 41, 70]
    cache = fill_rows(Cache(lens, m, 1, d, 16, dtype, seed=3))
    parents = tree(len(lens), m, 11, chain_bias=0.3)
    for s, length in enumerate(lens):
        for i, where in ((7, "v"), (11, "k"), (12, "v"), (20, "both")):
            k, v = cache.get(s, length + i)
            k, v = k.clone(), v.clone()
            if where != "v":
                k[:, 3] = what
            if where != "k":
                v[:, 1::5] = what
            cache.put(s, length + i, k, v)
    check(P, queries(len(lens), m, share, d, dtype), cache, parents=parents)


def test_values_over_the_cache(P):
    """Numbers that are none in the cache itself reach every row."""
    cache = fill_rows(Cache([50, 70], 3, 1, 64, 16, BF16, seed=3))
    for s, place, what in ((0, 10, math.inf), (1, 33, math.nan)):
        k, v = cache.get(s, place)
        v = v.clone()
        v[0, 5] = what
        cache.put(s, place, k, v)
    got = check(P, queries(2, 3, 2, 64, BF16), cache)
    assert torch.isinf(got[0, :, :, 5]).all() and torch.isnan(got[1, :, :, 5]).all()


def test_missing_pages(P):
    lens, m, d, page = [100, 100, 100, 40, -3, 10], 4, 64, 16
    cache = fill_rows(Cache(lens, m, 1, d, page, FP16, seed=4))
    pages = cache.pages()
    pages[0, 2] = -1                                                                   # inside of the cache
    pages[1, 1], pages[1, 3] = cache.k.shape[0], 2 ** 31 - 1                           # no pages of this cache
    pages[2, :] = -7                                                                   # nothing at all
    pages[3, 2] = -1                                                                   # of the rows themselves
    got = check(P, queries(len(lens), m, 2, d, FP16), cache, parents=tree(len(lens), m, 5), pages=pages)
    assert (got[2] == 0).all()


def test_lengths_over_the_table(P):
    """Places behind the last page of the table are not there, however long a sequence says it is."""
    cache = fill_rows(Cache([60, 60], 4, 1, 64, 16, BF16, seed=4))
    q = queries(2, 4, 1, 64, BF16)
    lens = torch.tensor([2 ** 31 - 1, 1_000_000], dtype=torch.int32)
    k, v, table, _ = cache.gpu()
    got = P.ivfpq_draft_attention(q.cuda(), k, v, table, lens.cuda()).cpu().double()
    # every row sees the 64 places, none of them a row's own
    for i in range(4):
        alone, _, size, reach = plain_attention(q[:, i:i + 1], cache.k, cache.v, table.cpu(), torch.tensor([63, 63]))
        assert bool(((got[:, i:i + 1] - alone).abs() <= allowed(BF16, 64, 64, alone, size, reach)).all())


def test_no_pages(P):
    empty = torch.empty((0, 1, 16, 64), dtype=BF16, device="cuda"), torch.empty((0, 1, 2, 64, 8), dtype=BF16, device="cuda")
    table = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    out, lse = P.ivfpq_draft_attention(queries(2, 2, 1, 64, BF16).cuda(), *empty, table, torch.tensor([20, 0], dtype=torch.int32, device="cuda"), with_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()
    k, v = torch.ones((1, 1, 16, 64), dtype=BF16, device="cuda"), torch.ones((1, 1, 2, 64, 8), dtype=BF16, device="cuda")
    out, lse = P.ivfpq_draft_attention(queries(2, 2, 1, 64, BF16).cuda(), k, v, torch.zeros((2, 0), dtype=torch.int32, device="cuda"),
                                       torch.tensor([20, 0], dtype=torch.int32, device="cuda"), with_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()
    assert P.ivfpq_draft_attention(torch.empty((0, 1, 1, 64), dtype=BF16, device="cuda"), k, v, torch.zeros((0, 1), dtype=torch.int32, device="cuda"),
                                   torch.zeros(0, dtype=torch.int32, device="cuda")).shape == (0, 1, 1, 64)


@pytest.mark.parametrize("size", [0.0, 30.0])
def test_scores_of_any_size(P, size):
    """All places alike, and one place far ahead of the others; references follow upwards over the places."""
    cache = Cache([300, 301], 2, 1, 64, 32, FP16, seed=6)
    for s, length in enumerate(cache.lens_list):
        for p in range(length + 2):
            cache.put(s, p, torch.full((1, 64), 0.01 * p) if size else torch.randn(1, 64), torch.randn(1, 64, generator=torch.Generator().manual_seed(p)))
    q = torch.full((2, 2, 2, 64), size ** 0.5 if size else 0.0).to(FP16)
    check(P, q, cache)


def test_scores_that_are_no_numbers(P):
    """An infinite score takes everything: the plain softmax of it is NaN, in that row alone."""
    cache = fill_rows(Cache([20, 20], 3, 1, 64, 16, BF16, seed=8))
    k, v = cache.get(0, 22)
    k = k.clone()
    k[0, 0] = math.inf
    cache.put(0, 22, k, v)
    got = check(P, queries(2, 3, 1, 64, BF16).abs(), cache)
    assert torch.isnan(got[0, 2]).all() and not torch.isnan(got[0, :2]).any()


@pytest.mark.parametrize("m,d", [(1, 128), (7, 80), (40, 64), (40, 256)])
def test_places_divided(P, m, d):
    """Long caches of few rows are divided among workgroups and joined; where places are looked at follows max_places."""
    lens = [1500, 700, 64, 0]
    cache = fill_rows(Cache(lens, m, 1, d, 64, BF16, seed=d))
    q = queries(len(lens), m, 2, d, BF16)
    longest = max(lens) + m
    assert P.lib().ivfpq_draft_attention_workspace_bytes(len(lens), m, 2, 1, d, longest) > 0
    first = check(P, q, cache)
    assert torch.equal(first, check(P, q, cache))                                      # the same bits again
    check(P, q, cache, max_places=longest)
    k, v, table, lengths = cache.gpu()
    # a bound far over what there is divides into more parts, most of them empty
    wide = torch.full((len(lens), 4000), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    check(P, q, cache, pages=wide, max_places=4000 * 64)


def test_strides(P):
    """Queries inside of a wider projection, at addresses of 16 bytes and at others."""
    lens, m, d, heads = [40, 9], 3, 64, 2
    cache = fill_rows(Cache(lens, m, 1, d, 16, BF16, seed=2))
    k, v, table, lengths = cache.gpu()
    wide = torch.randn(2, m, 500, generator=torch.Generator().manual_seed(1)).to(BF16)
    for start in (0, 8, 3):
        q = wide[:, :, start:start + heads * d].unflatten(2, (heads, d))
        got = P.ivfpq_draft_attention(wide.cuda()[:, :, start:start + heads * d].unflatten(2, (heads, d)), k, v, table, lengths)
        want, _, size, reach = plain_attention(q, cache.k, cache.v, table.cpu(), lengths.cpu())
        assert bool(((got.cpu().double() - want).abs() <= allowed(BF16, d, 60, want, size, reach)).all())
    turned = queries(m, 2, heads, d, BF16).transpose(0, 1)                             # rows of another order
    got = P.ivfpq_draft_attention(turned.cuda(), k, v, table, lengths)
    assert torch.equal(got, P.ivfpq_draft_attention(turned.contiguous().cuda(), k, v, table, lengths))


def test_offsets_over_32_bits(P):
    """Pages at both ends of a cache of more than 2^32 bytes a tensor."""
    page, heads, d = 256, 8, 128
    pages = 2 ** 32 // (page * heads * d * 2) + 5
    k = torch.zeros((pages, heads, page, d), dtype=BF16, device="cuda")
    v = torch.zeros((pages, heads, page // 8, d, 8), dtype=BF16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    for at in (0, pages - 1):
        k[at] = torch.randn(heads, page, d, generator=gen, device="cuda").to(BF16)
        v[at] = torch.randn(heads, page // 8, d, 8, generator=gen, device="cuda").to(BF16)
    table = torch.tensor([[pages - 1, 0]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([300], dtype=torch.int32, device="cuda")
    q = queries(1, 2, heads, d, BF16)
    got = P.ivfpq_draft_attention(q.cuda(), k, v, table, lens)
    small_k, small_v = k[[pages - 1, 0]].cpu(), v[[pages - 1, 0]].cpu()
    want, _, size, reach = plain_attention(q, small_k, small_v, torch.tensor([[0, 1]]), lens.cpu())
    assert bool(((got.cpu().double() - want).abs() <= allowed(BF16, d, 302, want, size, reach)).all())


def test_graph_and_stream(P):
    """A captured call follows its inputs' new contents, on another stream, with eager calls in between."""
    lens, m = [900, 31], 4
    cache = fill_rows(Cache(lens, m, 2, 128, 64, BF16, seed=2))
    k, v, table, lengths = cache.gpu()
    parents = tree(2, m, 1).cuda()
    q = queries(2, m, 4, 128, BF16).cuda()
    call = lambda: P.ivfpq_draft_attention(q, k, v, table, lengths, parents=parents)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        assert torch.equal(call(), call())
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for turn in range(4):
        q.copy_(queries(2, m, 4, 128, BF16, seed=turn).cuda())
        lengths.copy_(torch.tensor([900 - 100 * turn, 31 - turn], dtype=torch.int32))
        eager = call()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
