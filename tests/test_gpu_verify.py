"""ivfpq_verify_drafts against plain implementations in 64 bits.

Kept rows and tokens are equal: a drawn token differs only if its random number falls within the sums' error of a border (weights right to
1.1 10^-12, sums of 64 bits), and the plain implementation asserts that none lies within 10^-10 of its share.  A log-probability is one rounding of a 64-bit
number: half a step of fp32, and 10^-11 for the sum."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def clamp(u):
    u = float(u)
    return 0.0 if not u > 0 else min(u, 1 - 2.0 ** -24)


def distribution(x, temperature):
    """-> p, log p in 64 bits; None, and what is said of it, for a row without a distribution."""
    z = x.double() / temperature
    if torch.isnan(z).any() or torch.isposinf(z).any():
        return None, math.nan
    if torch.isneginf(z).all():
        return None, -math.inf
    return torch.softmax(z, dim=0), torch.log_softmax(z, dim=0)


def sample(w, u):
    sums = w.cumsum(dim=0)
    target = clamp(u) * float(sums[-1])
    assert target == 0 or float((sums - target).abs().min()) > 1e-10 * float(sums[-1])
    return int((sums <= target).sum())


def plain(logits, tokens, parents, counts, uniforms, temperature, drafts, accept):
    n, m = tokens.shape
    path, logprobs = torch.full((n, m), -1, dtype=torch.int32), torch.full((n, m), -math.inf, dtype=torch.float64)
    kept, following = torch.zeros(n, dtype=torch.int32), torch.full((n,), -1, dtype=torch.int32)
    vocab = logits.shape[1]
    for s in range(n):
        count = m if counts is None else min(max(int(counts[s]), 0), m)
        at = 0
        while at < count:
            i = int(kept[s])
            path[s, i] = at
            kept[s] += 1
            p, logp = distribution(logits[s * m + at], temperature)
            if p is None:
                logprobs[s, i], following[s] = logp, -1
                break
            child = None
            if drafts is not None:
                left = p
                if at + 1 < count:
                    x = int(tokens[s, at + 1])
                    q, _ = distribution(drafts[s * (m - 1) + at], temperature)
                    q = torch.zeros_like(p) if q is None else q
                    if 0 <= x < vocab and clamp(accept[s, at + 1]) * float(q[x]) < float(p[x]):
                        child, token = at + 1, x
                    elif float((p - q).clamp(min=0).sum()) > 0:
                        left = (p - q).clamp(min=0)
                if child is None:
                    token = sample(left, uniforms[s, at])
            else:
                token = int(logits[s * m + at].float().argmax()) if uniforms is None else sample(p, uniforms[s, at])
                for j in range(1, count):
                    up = j - 1 if parents is None else int(parents[s, j])
                    if 0 <= up < j and up == at and int(tokens[s, j]) == token:
                        child = j
                        break
            logprobs[s, i] = logp[token]
            if child is None:
                following[s] = token
                break
            at = child
    return path, kept, following, logprobs


def check(P, logits, tokens, parents=None, counts=None, uniforms=None, temperature=1.0, drafts=None, accept=None, gpu_logits=None):
    put = lambda t: None if t is None else t.cuda()
    got = P.ivfpq_verify_drafts(put(logits) if gpu_logits is None else gpu_logits, put(tokens), parents=put(parents), counts=put(counts), uniforms=put(uniforms),
                                temperature=temperature, draft_logits=put(drafts), accept=put(accept))
    path, kept, following, logprobs = plain(logits, tokens, parents, counts, uniforms, temperature, drafts, accept)
    assert torch.equal(got.kept.cpu(), kept), (got.kept.cpu(), kept)
    assert torch.equal(got.path.cpu(), path) and torch.equal(got.next_tokens.cpu(), following)
    lp = got.logprobs.cpu().double()
    assert torch.equal(torch.isnan(lp), torch.isnan(logprobs)) and torch.equal(torch.isneginf(lp), torch.isneginf(logprobs))
    fine = torch.isfinite(logprobs)
    off = torch.where(fine, (lp - logprobs).abs(), 0.0)
    assert bool((off <= 2.0 ** -24 * torch.where(fine, logprobs, 0.0).abs() + 1e-11).all()), float(off.max())
    return got


def rows(n, m, vocab, dtype, seed, size=3.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(n * m, vocab, generator=gen) * size).to(dtype), gen


def likely_tree(logits, n, m, gen, wide=3):
    """A tree whose rows hold likely tokens of their parents' logits."""
    parents, tokens = torch.full((n, m), -1, dtype=torch.int32), torch.randint(logits.shape[1], (n, m), generator=gen, dtype=torch.int32)
    best = torch.topk(logits.float(), min(4, logits.shape[1]), dim=1).indices
    for s in range(n):
        for i in range(1, m):
            up = max(0, i - 1 - int(torch.randint(wide, (), generator=gen)))
            parents[s, i] = up
            tokens[s, i] = best[s * m + up, int(torch.randint(best.shape[1], (), generator=gen))]
    return parents, tokens


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,m,vocab", [(1, 1, 1), (3, 2, 2), (5, 7, 100), (4, 64, 2047), (2, 33, 2048), (3, 16, 2049), (2, 5, 50_001), (1, 4, 131_072)])
@pytest.mark.parametrize("greedy", [False, True])
def test_trees(P, dtype, n, m, vocab, greedy):
    logits, gen = rows(n, m, vocab, dtype, seed=vocab + m, size=4.0)
    parents, tokens = likely_tree(logits, n, m, gen)
    for temperature in (1.0, 0.3):
        check(P, logits, tokens, parents, uniforms=None if greedy else torch.rand(n, m, generator=gen), temperature=temperature)


@pytest.mark.parametrize("greedy", [False, True])
def test_whole_branches_are_kept(P, greedy):
    """Logits that leave no doubt: a chain is kept to its end, and a tree's branch."""
    n, m, vocab = 3, 64, 300
    gen = torch.Generator().manual_seed(1)
    tokens = torch.randint(vocab, (n, m), generator=gen, dtype=torch.int32)
    logits = torch.randn(n * m, vocab, generator=gen)
    logits[torch.arange(n * m - 1), tokens.reshape(-1)[1:].long()] = 60.0
    u = None if greedy else torch.rand(n, m, generator=gen)
    got = check(P, logits, tokens, uniforms=u)
    assert (got.kept == m).all()
    counts = torch.tensor([64, 10, 1], dtype=torch.int32)
    got = check(P, logits, tokens, uniforms=u, counts=counts)
    assert got.kept.cpu().equal(counts)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,m,vocab", [(1, 2, 1), (6, 2, 3), (40, 5, 64), (7, 64, 500), (9, 6, 2049), (3, 4, 50_001)])
def test_students_drafts(P, dtype, n, m, vocab):
    logits, gen = rows(n, m, vocab, dtype, seed=vocab, size=2.0)
    drafts = (logits.float().view(n, m, vocab)[:, :-1].reshape(n * (m - 1), vocab) + 0.5 * torch.randn(n * (m - 1), vocab, generator=gen)).to(dtype)
    tokens = torch.randint(vocab, (n, m), generator=gen, dtype=torch.int32)
    tokens[:, 1:] = torch.multinomial(torch.softmax(drafts.float() / 0.7, dim=1), 1, generator=gen).view(n, m - 1).int()
    counts = torch.randint(0, m + 1, (n,), generator=gen, dtype=torch.int32)
    u, a = torch.rand(n, m, generator=gen), torch.rand(n, m, generator=gen)
    check(P, logits, tokens, uniforms=u, accept=a, drafts=drafts, temperature=0.7)
    check(P, logits, tokens, uniforms=u, accept=a, drafts=drafts, temperature=0.7, counts=counts)


def test_student_like_the_model(P):
    """p = q: every draft is kept, whatever the numbers (those at the ends of their range too)."""
    n, m, vocab = 4, 8, 1_000
    logits, gen = rows(n, m, vocab, torch.bfloat16, seed=3)
    drafts = logits.view(n, m, vocab)[:, :-1].reshape(-1, vocab).clone()
    tokens = torch.randint(vocab, (n, m), generator=gen, dtype=torch.int32)
    accept = torch.rand(n, m, generator=gen)
    accept[0], accept[1, ::2] = 1.0, math.nan
    got = check(P, logits, tokens, uniforms=torch.rand(n, m, generator=gen), accept=accept, drafts=drafts)
    assert (got.kept == m).all()


@pytest.mark.parametrize("students", [False, True])
def test_rows_without_a_distribution(P, students):
    n, m, vocab = 6, 4, 2_500
    logits, gen = rows(n, m, vocab, torch.float32, seed=5)
    tokens = torch.zeros(n, m, dtype=torch.int32)
    logits[:, 0] = 40.0                                                  # every row says token 0, every draft is right
    logits[0 * m + 1, 7] = math.nan
    logits[1 * m + 0, 2_400] = math.inf
    logits[2 * m + 2] = -math.inf
    logits[3 * m + 1, 1:] = -math.inf                                    # nothing but token 0
    logits[4 * m + 3, 1] = -3.4e38
    drafts = None
    if students:
        drafts = torch.randn(n * (m - 1), vocab, generator=gen)
        drafts[5 * 3 + 0] = -math.inf                                    # drafts that nothing stands behind
        drafts[5 * 3 + 1, 9] = math.nan
    got = check(P, logits, tokens, uniforms=torch.rand(n, m, generator=gen) * 0.9, accept=torch.rand(n, m, generator=gen) if students else None, drafts=drafts)
    assert got.next_tokens.tolist()[:3] == [-1, -1, -1]
    if not students:
        check(P, logits, tokens)


def test_masks_and_lowest_values(P):
    """Few tokens left by a mask, at the ends of blocks; masks of the type's lowest value; equal logits."""
    n, m, vocab = 5, 3, 6_200
    for dtype in TYPES:
        logits = torch.full((n * m, vocab), -math.inf).to(dtype)
        logits[:m, [0, 2_047, 2_048, 6_199]] = torch.tensor([1.0, 2.0, 2.0, 1.5]).to(dtype)
        logits[m:2 * m] = torch.finfo(dtype).min
        logits[m:2 * m, [5, 4_096]] = 0.5
        logits[2 * m:3 * m] = torch.finfo(dtype).min                     # uniform
        logits[3 * m:4 * m] = 0.0
        logits[4 * m:, 3_000] = torch.finfo(dtype).max
        gen = torch.Generator().manual_seed(2)
        tokens = torch.full((n, m), 2_048, dtype=torch.int32)
        for u in (torch.rand(n, m, generator=gen), torch.zeros(n, m), None):
            check(P, logits, tokens, uniforms=u)
        got = P.ivfpq_verify_drafts(logits.cuda(), tokens.cuda(), uniforms=torch.full((n, m), 2.0).cuda())        # counts as the largest number under 1
        assert got.next_tokens.tolist()[0] == 6_199 and got.next_tokens.tolist()[3] == vocab - 1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("middle,size,temperature", [(0.0, 3.0, 1.0), (-100.0, 1.0, 1.0), (100.0, 1.0, 1.0), (-100.0, 1.0, 0.01), (100.0, 1.0, 0.01), (0.0, 3.0, 1e6),
                                                     (1e4, 1.0, 1e-6), (-1e4, 1.0, 1e-6)])
def test_signs_and_spreads(P, dtype, middle, size, temperature):
    """All values of one sign, of both; some far under the largest, so that their weights are cut off, in some blocks of a row only; sums about numbers that no
    longer fit 2^30 steps of 1/32.  (Shares of 64 bits are right to 10^-11 in the plain form up to 10^4 temperatures; beyond, logits here are equal or far apart.)"""
    n, m, vocab = 2, 4, 9_001
    logits, gen = rows(n, m, vocab, torch.float32, 31, size)
    logits += middle
    logits[0, 2_500:2_510] = middle - 2_000.0
    logits[1, ::2] = middle - 900.0
    logits[2, 4_100:] = -math.inf
    logits = logits.to(dtype)
    parents, tokens = likely_tree(logits, n, m, gen)
    for uniforms in (torch.rand(n, m, generator=gen), None):
        check(P, logits, tokens, parents, uniforms=uniforms, temperature=temperature)


@pytest.mark.parametrize("dtype,bits", [(torch.float32, 0xFFC00000 - (1 << 32)), (torch.float16, 0xFE00 - (1 << 16)), (torch.bfloat16, 0xFFC0 - (1 << 16))])
def test_nan_of_either_sign(P, dtype, bits):
    n, m, vocab = 3, 1, 5_000
    logits, gen = rows(n, m, vocab, dtype, 32)
    as_whole = torch.int32 if dtype == torch.float32 else torch.int16
    logits.view(as_whole)[0, 4_999] = bits                               # the sign set
    logits[1, 2_047] = math.nan
    logits[0, 0] = -1.0
    assert math.isnan(float(logits[0, 4_999]))
    tokens = torch.zeros(n, m, dtype=torch.int32)
    for uniforms in (torch.rand(n, m, generator=gen), None):
        assert check(P, logits, tokens, uniforms=uniforms).next_tokens.tolist()[:2] == [-1, -1]
    logits = -logits.abs()                                               # and with nothing but signs set
    check(P, logits, tokens, uniforms=torch.rand(n, m, generator=gen))


def test_bad_parents_and_tokens(P):
    """Parents out of range follow the cache and are never reached from a row; tokens out of range are never said."""
    n, m, vocab = 2, 6, 50
    logits, gen = rows(n, m, vocab, torch.float32, seed=9)
    best = logits.argmax(dim=1).view(n, m).int()
    tokens = best[:, :1].expand(n, m).contiguous()
    parents = torch.tensor([[-1, 1, 3, -9, 0, 0], [-1, 2 ** 31 - 1, 0, 0, 2, 2]], dtype=torch.int32)
    got = check(P, logits, tokens, parents)
    assert got.path[0, 1] == 4 and got.path[1, 1] == 2                   # of two children that hold the token the first
    tokens = torch.full((n, m), -1, dtype=torch.int32)
    tokens[1] = vocab
    check(P, logits, tokens, parents)
    drafts = torch.randn(n * (m - 1), vocab, generator=gen)
    check(P, logits, tokens, uniforms=torch.rand(n, m, generator=gen), accept=torch.zeros(n, m), drafts=drafts)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignments(P, dtype):
    n, m, vocab = 2, 4, 4_500
    wide = (torch.randn(n * m, vocab + 40, generator=torch.Generator().manual_seed(4)) * 3).to(dtype)
    gen = torch.Generator().manual_seed(5)
    u = torch.rand(n, m, generator=gen)
    for start in (0, 1, 5, 8, 39):
        logits = wide[:, start:start + vocab]
        parents, tokens = likely_tree(logits, n, m, gen)
        check(P, logits, tokens, parents, uniforms=u, gpu_logits=wide.cuda()[:, start:start + vocab])
        check(P, logits, tokens, parents, gpu_logits=wide.cuda()[:, start:start + vocab])


def test_empty_and_single(P):
    got = P.ivfpq_verify_drafts(torch.empty((0, 10), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"))
    assert got.path.shape == (0, 3) and got.kept.shape == (0,)
    logits, gen = rows(4, 1, 300, torch.float16, seed=1)
    none = torch.empty((0, 300), dtype=torch.float16)
    u = torch.rand(4, 1, generator=gen)
    check(P, logits, torch.zeros(4, 1, dtype=torch.int32), uniforms=u)
    got = P.ivfpq_verify_drafts(logits.cuda(), torch.zeros(4, 1, dtype=torch.int32, device="cuda"), uniforms=u.cuda(), draft_logits=none.cuda(), accept=u.cuda())
    assert torch.equal(got.next_tokens, P.ivfpq_verify_drafts(logits.cuda(), torch.zeros(4, 1, dtype=torch.int32, device="cuda"), uniforms=u.cuda()).next_tokens)


@pytest.mark.parametrize("students", [False, True])
def test_what_is_said_has_the_models_distribution(P, students):
    """40,000 sequences of one distribution: the first token behind row 0 comes out as often as the model says, to 5 standard deviations."""
    n, m, vocab = 40_000, 3, 6
    gen = torch.Generator().manual_seed(11)
    one = torch.randn(m, vocab, generator=gen)
    logits = one.repeat(n, 1)
    drafted = torch.randn(m - 1, vocab, generator=gen)
    q = torch.softmax(drafted.double(), dim=1)
    tokens = torch.zeros(n, m, dtype=torch.int32)
    if students:
        for i in range(1, m):
            tokens[:, i] = torch.multinomial(q[i - 1], n, replacement=True, generator=gen).int()
    else:
        tokens[:, 1], tokens[:, 2] = 4, 1
    got = P.ivfpq_verify_drafts(logits.cuda(), tokens.cuda(), uniforms=torch.rand(n, m, generator=gen).cuda(), draft_logits=drafted.repeat(n, 1).cuda() if students else None,
                                accept=torch.rand(n, m, generator=gen).cuda() if students else None)
    kept, following = got.kept.cpu(), got.next_tokens.cpu()
    said = torch.where(kept > 1, tokens[:, 1], following)
    p = torch.softmax(one[0].double(), dim=0)
    often = torch.bincount(said.long(), minlength=vocab).double()
    assert bool(((often - n * p).abs() <= 5 * (n * p * (1 - p)).sqrt()).all()), often / n - p
    second = torch.where(kept > 2, tokens[:, 2], following)[kept > 1]
    p, k = torch.softmax(one[1].double(), dim=0), int((kept > 1).sum())
    often = torch.bincount(second.long(), minlength=vocab).double()
    assert bool(((often - k * p).abs() <= 5 * (k * p * (1 - p)).sqrt()).all()), often / k - p


@pytest.mark.parametrize("students", [False, True])
def test_graph_and_stream(P, students):
    n, m, vocab = 3, 5, 5_000
    state = {}

    def fresh(seed):
        logits, gen = rows(n, m, vocab, torch.bfloat16, seed=seed)
        drafts, a, u = torch.randn(n * (m - 1), vocab, generator=gen).to(torch.bfloat16), torch.rand(n, m, generator=gen), torch.rand(n, m, generator=gen)
        return {"logits": logits, "drafts": drafts, "accept": a, "uniforms": u, "tokens": torch.randint(vocab, (n, m), generator=gen, dtype=torch.int32)}
    state = {k: v.cuda() for k, v in fresh(0).items()}
    call = lambda: P.ivfpq_verify_drafts(state["logits"], state["tokens"], uniforms=state["uniforms"], draft_logits=state["drafts"] if students else None,
                                         accept=state["accept"] if students else None)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for seed in range(1, 4):
        for key, x in fresh(seed).items():
            state[key].copy_(x)
        eager = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
