"""How far the sums over a row may be off where a chain of additions is at its worst.

Every thread's first chunk holds a logit of 0, the row's largest, and all others are under half a unit in the last place of it: added
one after the other each of them is lost, of 256 in a thread 227 e of the sum together (e = 2^-24).  Added among themselves
first they count.

Tolerance.  A thread's values come in tiles of 32 bytes a thread (a chunk of 16 in the kernel that holds a row): a tree of at most 4 additions in
a tile, vocab / 256 / 8 or 16 tiles in a chain (at most 16 chunks a thread where a row is held), 6 + 16 joins, 2 e of an exponential, e of
the quotient, the maximum's share and e |log S| of the logarithm: e (chain + 36 + |log S|).  The small values are 2^-24.2 of the largest, so
their own relative error, 3 e 24, is nothing of the sum."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
VALUE = -16.75                       # exact in every type; exp of it is 0.89 e


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def rows(n, vocab, dtype, threads):
    x = torch.full((vocab,), VALUE, dtype=dtype, device="cuda")
    vec = 16 // x.element_size()
    x[: threads * vec: vec] = 0.0
    ones = threads
    total = ones + (vocab - ones) * math.exp(VALUE)
    u = (vocab - ones) * math.exp(VALUE) * VALUE
    return x.expand(n, vocab).contiguous(), math.log(total), math.log(total) - u / total


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("top", [0, 20])
@pytest.mark.parametrize("n,vocab", [(1600, 65536), (800, 65536)])
def test_statistics(P, dtype, top, n, vocab):
    x, log_s, entropy = rows(n, vocab, dtype, 256)
    targets = torch.zeros(n, dtype=torch.int32, device="cuda")
    got = P.ivfpq_token_logprobs(x, targets, top=top)
    tol = E * (vocab / 256 / (8 if dtype == torch.float32 else 16) + 36 + log_s)
    assert float((got.norms[:, 1].double() - log_s).abs().max()) <= tol
    assert float((got.logprobs.double() + log_s).abs().max()) <= tol
    # a quotient of two such sums, its own terms off by e (3 + 2) of themselves, is 0.0003 beside log S
    assert float((got.entropy.double() - entropy).abs().max()) <= tol + E * 200 * (entropy - log_s) + E * log_s
    loss, norms = P.ivfpq_distill_topk(x, targets[:, None].contiguous(), torch.zeros(n, 1, device="cuda"))
    assert float((loss.double() - log_s).abs().max()) <= tol and float((norms[:, 1].double() - log_s).abs().max()) <= tol


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,vocab,threads", [(64, 32768, 256), (300, 65536, 512), (300, 131072, 1024)])
def test_rows_held_in_registers(P, dtype, n, vocab, threads):
    x, log_s, _ = rows(n, vocab, dtype, threads)
    targets = torch.zeros((n, 1), dtype=torch.int32, device="cuda")
    loss, _ = P.ivfpq_distill_topk_step(x, targets, torch.zeros(n, 1, device="cuda"))
    assert float((loss.double() - log_s).abs().max()) <= E * (16 + 36 + log_s)
