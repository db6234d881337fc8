"""ivfpq_cache_keep and ivfpq_cache_append over passes of more than 256 rows, which a workgroup goes through in turns: rows whose places and sources lie on both sides of
a turn's border, and long prompts."""
import pytest
import torch

from test_gpu_cache import BF16, FP16, FP32, check_append, plain_keep
from util_drafts import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def paths(m, seed):
    """Ascending rows, -1 behind them, and how many: moved up by one, by a turn, by more; every other one; any; some that stay before some that move."""
    gen = torch.Generator().manual_seed(seed)
    shift = lambda by: [0] + list(range(1 + by, m))
    some = torch.randperm(m, generator=gen)[:m // 2 + 1].sort().values.tolist()
    each = [shift(1), shift(min(256, m - 2)), shift(100), list(range(0, m, 2)), some, list(range(255)) + list(range(256, m)), list(range(m)), []]
    path = torch.full((len(each), m), -1, dtype=torch.int32)
    for s, held in enumerate(each):
        path[s, :len(held)] = torch.tensor(held, dtype=torch.int32)
    return path, torch.tensor([len(held) for held in each], dtype=torch.int32)


@pytest.mark.parametrize("dtype,layers,kv_heads,d,page", [(BF16, 2, 1, 64, 16), (FP16, None, 3, 8, 64), (BF16, 1, 2, 200, 256)])
@pytest.mark.parametrize("m", [256, 257, 258, 300, 512, 513, 600])
def test_keep(P, dtype, layers, kv_heads, d, page, m):
    path, kept = paths(m, m)
    lens = [0, 1, 7, 8, 31, 100, 13, 5]
    cache = Cache(lens, m, kv_heads, d, page, dtype, layers=layers)
    gen = torch.Generator().manual_seed(m)
    cache.k, cache.v = torch.randn(cache.k.shape, generator=gen).to(dtype), torch.randn(cache.v.shape, generator=gen).to(dtype)
    want = plain_keep(cache, path, kept, m)
    k, v, table, lengths = cache.gpu()
    P.ivfpq_cache_keep(k, v, table, lengths, path.cuda(), kept.cuda())
    assert torch.equal(k.cpu(), want[0]) and torch.equal(v.cpu(), want[1])


@pytest.mark.parametrize("dtype,cache_dtype,interleaved", [(BF16, BF16, False), (FP32, FP16, True)])
def test_append(P, dtype, cache_dtype, interleaved):
    check_append(P, [0, 3, 41], 600, 2, 1, 40, 32, dtype, cache_dtype, 16, interleaved, counts=torch.tensor([600, 257, 513], dtype=torch.int32))
