"""ivfpq_verify_drafts over vocabularies of more than 64 blocks of 2048 logits, which a wave goes through in turns of 64: what a row's sums, its most likely token and a
draw carry from one turn to the next.  Compared with the plain implementation in 64 bits: tokens and rows equal, log-probabilities within a rounding."""
import math

import pytest
import torch

from test_gpu_verify import TYPES, check, likely_tree, rows

pytestmark = pytest.mark.gpu
TURN = 64 * 2048
VOCABS = [131_079, 150_001, 262_147]


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def inside(p, token):
    """A number of fp32 that falls amid a token's probability."""
    sums = p.cumsum(dim=0)
    return float(((sums[token] - p[token] / 2) / sums[-1]).float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("start", [0, 1, 7])
def test_trees(P, dtype, vocab, start):
    """Rows at addresses of any alignment, tokens drawn and most likely."""
    n, m = 2, 4
    wide, gen = rows(n, m, vocab + 9, dtype, seed=vocab + start, size=4.0)
    logits = wide[:, start:start + vocab]
    parents, tokens = likely_tree(logits, n, m, gen)
    for uniforms in (torch.rand(n, m, generator=gen), torch.full((n, m), 0.999), None):
        check(P, logits, tokens, parents, uniforms=uniforms, gpu_logits=wide.cuda()[:, start:start + vocab])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_most_likely_behind_the_first_turn(P, dtype, vocab):
    """The largest logit behind the first 64 blocks only, tied within its block, with a later one and with the last; and in the first block and a late one."""
    logits, _ = rows(5, 1, vocab, dtype, seed=3, size=1.0)
    late = TURN + 2                                                      # in block 64 at any alignment
    for row, places in enumerate(([late], [late, late + 3], [late, vocab - 1], [vocab - 1], [5, late, vocab - 1])):
        logits[row, places] = 20.0
    got = check(P, logits, torch.zeros(5, 1, dtype=torch.int32))
    assert got.next_tokens.tolist() == [late, late, late, vocab - 1, 5]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_draws_on_both_sides_of_a_turn(P, dtype, vocab):
    """Tokens in the first blocks, on both sides of the border between turns, just behind it and at the end of the last block."""
    wanted = [0, 2_048, TURN - 2_049, TURN - 9, TURN - 1, TURN, TURN + 1, vocab - 2, vocab - 1]
    n = len(wanted)
    one, _ = rows(1, 1, vocab, dtype, seed=vocab, size=2.0)
    one[0, wanted] = 6.0                                                 # wide enough for a number of fp32 to fall into
    logits = one.repeat(n, 1)
    p = torch.softmax(one[0].double(), dim=0)
    got = check(P, logits, torch.zeros(n, 1, dtype=torch.int32), uniforms=torch.tensor([[inside(p, token)] for token in wanted]))
    assert got.next_tokens.tolist() == wanted


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_few_tokens_left(P, dtype, vocab):
    """Masks that leave one late block, blocks of both turns, or nothing; a NaN and an infinity in a late block."""
    logits = torch.full((6, vocab), -math.inf).to(dtype)
    gen = torch.Generator().manual_seed(4)
    late = slice(TURN, vocab)
    logits[0, late] = torch.randn(vocab - TURN, generator=gen).to(dtype)
    logits[1, vocab - 1] = -3.0
    logits[2, [100, vocab - 2]] = 1.0
    logits[4] = torch.randn(vocab, generator=gen).to(dtype)
    logits[5] = logits[4]
    logits[4, vocab - 1] = math.nan
    logits[5, TURN + 1] = math.inf
    tokens = torch.zeros(6, 1, dtype=torch.int32)
    for uniforms in (None, torch.full((6, 1), 0.25), torch.full((6, 1), 0.75), torch.zeros(6, 1), torch.ones(6, 1)):
        got = check(P, logits, tokens, uniforms=uniforms)
        assert got.next_tokens.tolist()[3:] == [-1, -1, -1] and got.next_tokens.tolist()[1] == vocab - 1
    assert check(P, logits, tokens, uniforms=torch.full((6, 1), 0.75)).next_tokens.tolist()[2] == vocab - 2


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_students_drafts(P, dtype, vocab):
    """Remainders of more than 64 blocks, over all of them, in the last tokens only, and in the first only."""
    n, m = 4, 3
    logits, gen = rows(n, m, vocab, dtype, seed=vocab, size=2.0)
    drafts = (logits.float().view(n, m, vocab)[:, :-1].reshape(n * (m - 1), vocab) + 0.5 * torch.randn(n * (m - 1), vocab, generator=gen)).to(dtype)
    model = logits.view(n, m, vocab)[:, :-1].reshape(n * (m - 1), vocab)
    for s, places in ((2, slice(vocab - 3, vocab)), (3, slice(0, 3))):   # alike but for a few tokens that the model finds likelier
        drafts[s * (m - 1):(s + 1) * (m - 1)] = model[s * (m - 1):(s + 1) * (m - 1)]
        drafts[s * (m - 1):(s + 1) * (m - 1), places] -= 4.0
    tokens = torch.randint(vocab, (n, m), generator=gen, dtype=torch.int32)
    tokens[:, 1:] = torch.multinomial(torch.softmax(drafts.double(), dim=1), 1, generator=gen).view(n, m - 1).int()
    for accept in (torch.rand(n, m, generator=gen), torch.ones(n, m)):
        for uniforms in (torch.rand(n, m, generator=gen), torch.full((n, m), 0.99)):
            check(P, logits, tokens, uniforms=uniforms, accept=accept, drafts=drafts)
