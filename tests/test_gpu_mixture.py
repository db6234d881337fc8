"""The mixture with listed tokens over rows that a mask or a temperature has changed, against the definitions in 64 bits.

Tolerances.  e = 2^-24, c = vocab / 256 + 72: a log-probability of the mixture is off by at most e (c + 8 |log m|), each part of it as for the
model alone, one more addition and a logarithm; the entropy, sums of such terms exchanged in 64 bits, by 4 e c (1 + entropy)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
LEAST = -3.4028235677973366e38                     # what is below rounds to -inf in fp32
LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.float16: -65504.0, torch.bfloat16: torch.finfo(torch.bfloat16).min}


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def listed(n, vocab, k, seed):
    """Distinct tokens with log-probabilities that sum to one; of every other row a part unused."""
    gen = torch.Generator().manual_seed(seed)
    tokens = torch.stack([torch.randperm(vocab, generator=gen)[:k] for _ in range(n)]).int()
    logq = torch.randn(n, k, generator=gen) * 2
    used = torch.where(torch.arange(n) % 2 == 0, k, torch.randint(1, k + 1, (n,), generator=gen))
    off = torch.arange(k)[None] >= used[:, None]
    logq = torch.log_softmax(torch.where(off, -math.inf, logq), dim=1)
    return torch.where(off, -1, tokens), logq


def reference(x, tokens, logq, weight, temperature):
    raw = x.cpu().double()
    top = raw.amax(dim=1, keepdim=True)
    none = top == -math.inf
    t = torch.where(none, -math.inf, (raw - torch.where(none, 0.0, top)) / temperature)
    logp = torch.where(none, -math.inf, t - torch.logsumexp(t, dim=1, keepdim=True))
    used = tokens >= 0
    w = torch.where(used.any(dim=1, keepdim=True), weight, 0.0).double()
    w = torch.where(none & used.any(dim=1, keepdim=True), 1.0, w)
    model = torch.log1p(-w) + logp
    near = torch.full_like(model, -math.inf)
    for r in range(x.shape[0]):
        for j in torch.nonzero(used[r])[:, 0].tolist():
            near[r, tokens[r, j]] = w[r, 0].log() + logq[r, j].double()
    logm = torch.logaddexp(model, near)
    logm = torch.where(logm > LEAST, logm, -math.inf)
    m = logm.exp()
    return logm, -torch.where(m > 0, m * logm, 0.0).sum(dim=1)


def close(got, want, tol):
    got = got.detach().cpu().double()
    finite = torch.isfinite(want)
    assert torch.equal(got[~finite], want[~finite])
    off = (got - want).abs()[finite]
    tol = tol.expand_as(want)[finite]
    assert bool((off <= tol).all()), float((off / tol).max())


def check(P, x, tokens, logq, targets, top, weight, temperature):
    n, vocab = x.shape
    got = P.ivfpq_token_logprobs(x, targets.cuda(), top=top, temperature=temperature, neighbours=(tokens.cuda(), logq.cuda()), weight=weight)
    logm, entropy = reference(x, tokens, logq, weight, temperature)
    c = vocab / 256 + 72
    tol = lambda v: E * (c + 8 * torch.where(torch.isfinite(v), v.abs(), 0.0))
    want = logm.gather(1, targets.long()[:, None])[:, 0]
    close(got.logprobs, want, tol(want))
    close(got.entropy, entropy, 4 * E * c * (1 + entropy))
    if not top:
        return
    have, places = got.top_logprobs.cpu().double(), got.top_tokens.cpu().long()
    there = places >= 0
    assert torch.equal(there.sum(dim=1), (logm > -math.inf).sum(dim=1).clamp(max=top)) and torch.equal(there, have > -math.inf)
    theirs = torch.where(there, logm.gather(1, places.clamp(min=0)), -math.inf)
    close(got.top_logprobs, theirs, tol(theirs))
    best = torch.sort(logm, dim=1, descending=True).values[:, :top]
    close(got.top_logprobs, best, tol(best))
    assert (have[:, 1:] <= have[:, :-1]).all()
    for r in range(n):
        assert len(set(places[r][there[r]].tolist())) == int(there[r].sum())


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,vocab,k,top", [(1, 40000, 64, 20), (6, 5001, 17, 100), (1600, 300, 8, 5), (5, 20000, 700, 0)])
@pytest.mark.parametrize("temperature", [0.05, 0.7, 2.5])
@pytest.mark.parametrize("weight", [0.02, 0.6])
def test_temperatures(P, dtype, n, vocab, k, top, temperature, weight):
    gen = torch.Generator().manual_seed(n + k)
    x = (torch.randn(n, vocab, generator=gen) * 3.0).to(dtype).cuda()
    targets = torch.randint(vocab, (n,), generator=gen).int()
    tokens, logq = listed(n, vocab, k, vocab)
    targets = torch.where((tokens[:, 0] >= 0) & (torch.arange(n) % 3 == 0), tokens[:, 0], targets)
    check(P, x, tokens, logq, targets, top, weight, temperature)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,vocab,k,top", [(7, 30011, 40, 60), (1600, 400, 20, 30)])
@pytest.mark.parametrize("temperature", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("mask", ["-inf", "lowest"])
def test_masks(P, dtype, n, vocab, k, top, temperature, mask):
    """Rows of which a mask leaves a part, few tokens or none, with listed tokens and targets inside of it and outside."""
    gen = torch.Generator().manual_seed(n + vocab)
    x = (torch.randn(n, vocab, generator=gen) * 3.0).to(dtype)
    tokens, logq = listed(n, vocab, k, 5)
    share = torch.tensor([0.5, 0.01, 0.0, 1.0, 3.0 / vocab, 0.9, 0.1])[torch.arange(n) % 7]
    keep = torch.rand(n, vocab, generator=gen) < share[:, None]
    keep.scatter_(1, tokens[:, 1:2].clamp(min=0).long(), (torch.arange(n) % 4 == 0)[:, None] | keep[:, :1])
    x = torch.where(keep, x, -math.inf if mask == "-inf" else LOWEST[dtype]).to(dtype).cuda()
    targets = torch.randint(vocab, (n,), generator=gen).int()
    targets = torch.where((tokens[:, 0] >= 0) & (torch.arange(n) % 2 == 0), tokens[:, 0], targets)
    check(P, x, tokens, logq, targets, top, 0.25, temperature)
