"""Log-probabilities, entropy, alternatives, their mixture with listed tokens and the gradient, against the definitions
in 64 bits.

Tolerances.  With e = 2^-24 (half a unit in the last place of fp32): t = (x - M) / T carries at most 3 e |t|, an exponential
under 4 e of itself, and a row's sum, made of up to vocab / 256 + 64 additions in a chain, at most that many e of itself; hence
a log-probability is off by at most e (vocab / 256 + 64 + 4 |log p|), the entropy, a quotient of two such sums, by e times
twice that chain times (1 + entropy), and p relative to itself by as much as log p.  A gradient in 16 bits is rounded once more, to
nearest: it lies between the roundings of the ends of that interval."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.float16: -65504.0, torch.bfloat16: torch.finfo(torch.bfloat16).min}
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def chain(vocab):
    return vocab / 256 + 64


def logits_of(n, vocab, dtype, seed, pad=0, offset=0):
    """[n][vocab] with `pad` more values between the rows, the first `offset` values into its memory."""
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, vocab, generator=gen) * 3.0).to(dtype)
    room = torch.full((n * (vocab + pad) + offset,), 77.0, dtype=dtype, device="cuda")
    view = room[offset:].as_strided((n, vocab), (vocab + pad, 1), offset)
    view.copy_(x)
    return view


def reference(x, temperature=1.0):
    """-> log p, entropy, norms in 64 bits; rows without a finite logit: -inf, 0."""
    raw = x.detach().cpu().double()
    top = raw.amax(dim=1, keepdim=True)
    none = top == -math.inf
    t = torch.where(none, torch.full_like(raw, -math.inf), (raw - torch.where(none, 0.0, top)) / temperature)
    total = t.exp().sum(dim=1, keepdim=True)
    logp = torch.where(none, torch.full_like(raw, -math.inf), t - total.log())
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(dim=1)
    norms = torch.cat([top, total.log()], dim=1)
    return logp, entropy, norms


def best_of(x, top):
    """Descending logits, ties to the lower token, without -inf; padded with -1."""
    raw = x.detach().cpu().double().numpy()
    out = np.full((raw.shape[0], top), -1, np.int32)
    for r in range(raw.shape[0]):
        order = np.lexsort((np.arange(raw.shape[1]), -raw[r]))
        order = order[raw[r][order] > -np.inf][:top]
        out[r, :len(order)] = order
    return out


def close(got, want, tol):
    got, want = got.detach().cpu().double().numpy(), want.numpy()
    finite = np.isfinite(want)
    np.testing.assert_array_equal(np.where(finite, 0.0, got), np.where(finite, 0.0, want))      # infinities alike, no NaN
    tol = np.broadcast_to(np.asarray(tol), want.shape)
    off = np.abs(np.where(finite, got - want, 0.0))
    assert np.all(off <= tol), (off - tol).max()


def check_scores(got, x, targets, top, temperature=1.0):
    vocab = x.shape[1]
    logp, entropy, norms = reference(x, temperature)
    c = chain(vocab)
    want = logp.gather(1, targets.cpu().long()[:, None])[:, 0]
    finite = lambda v: torch.where(torch.isfinite(v), v.abs(), 0.0).numpy()
    close(got.logprobs, want, E * (c + 4 * finite(want)))
    close(got.entropy, entropy, E * 2 * c * (1 + entropy.numpy()))
    close(got.norms[:, 0], norms[:, 0], 0.0)
    close(got.norms[:, 1], norms[:, 1], E * (c + 4 * finite(norms[:, 1])))
    if top:
        tokens = best_of(x, top)
        np.testing.assert_array_equal(got.top_tokens.cpu().numpy(), tokens)
        at = torch.from_numpy(tokens).long()
        lp = torch.where(at >= 0, logp.gather(1, at.clamp(min=0)), -math.inf)
        close(got.top_logprobs, lp, E * (c + 4 * finite(lp)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab,top,pad,offset", [
    (1, 1, 1, 0, 0), (3, 2, 5, 0, 0), (5, 7, 3, 2, 1), (2, 63, 20, 1, 3), (4, 64, 64, 0, 0), (3, 65, 128, 0, 5), (9, 255, 20, 1, 1),
    (6, 1000, 1, 0, 0), (2, 4097, 20, 7, 3), (1, 50001, 128, 0, 1), (7, 50001, 5, 0, 0), (1, 131073, 20, 0, 0), (1100, 2500, 20, 0, 0),
    (1030, 257, 128, 0, 0), (2100, 9001, 0, 3, 1)])
def test_scores(P, dtype, n, vocab, top, pad, offset):
    x = logits_of(n, vocab, dtype, seed=n + vocab, pad=pad, offset=offset)
    targets = torch.randint(vocab, (n,), generator=torch.Generator().manual_seed(vocab)).int().cuda()
    got = P.ivfpq_token_logprobs(x, targets, top=top)
    check_scores(got, x, targets, top)


@pytest.mark.parametrize("temperature", [0.01, 0.7, 3.0, 1000.0])
def test_temperature(P, temperature):
    x = logits_of(13, 3001, torch.float32, seed=5)
    targets = torch.arange(13, dtype=torch.int32, device="cuda") * 200
    check_scores(P.ivfpq_token_logprobs(x, targets, top=10, temperature=temperature), x, targets, 10, temperature)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 40, 1200])          # rows split between workgroups, and not
def test_masks_ties_and_orders(P, dtype, n):
    """Rows that a mask leaves little or nothing of, of -inf and of the type's lowest value, constant rows, sorted rows, and rows
    whose large values all sit where one part of a workgroup reads them."""
    vocab = 20011
    x = logits_of(n, vocab, dtype, seed=3)
    at = torch.arange(vocab, device="cuda")
    low = LOWEST[dtype]
    kinds = [
        lambda v: torch.full_like(v, -math.inf),
        lambda v: torch.full_like(v, low),
        lambda v: torch.where(at == vocab - 1, v, low),
        lambda v: torch.where(at % 5000 == 7, v, -math.inf),
        lambda v: torch.where(at < 12, v, low),
        lambda v: torch.full_like(v, 1.5),
        lambda v: torch.full_like(v, -0.0).where(at % 3 == 0, torch.zeros_like(v)),
        lambda v: (at / 1024.0).to(dtype),
        lambda v: (-at / 1024.0).to(dtype),
        lambda v: torch.where((at // 8) % 64 < 40, 8.0 + (at % 1000) / 128.0, -4.0 - (at % 16)).to(dtype),
        lambda v: torch.where((at // 4) % 256 < 130, 8.0 + (at % 1000) / 128.0, -4.0 - (at % 16)).to(dtype),
        lambda v: torch.where(at > vocab - 3000, v + 30, v),
    ]
    for r in range(n):
        x[r] = kinds[(r + 3 * (n == 1)) % len(kinds)](x[r])
    targets = torch.full((n,), vocab - 1, dtype=torch.int32, device="cuda")
    for top in (1, 20, 128):
        check_scores(P.ivfpq_token_logprobs(x, targets, top=top), x, targets, top)
    if n == 1:
        for kind in kinds:
            y = kind(x[0])[None].contiguous()
            check_scores(P.ivfpq_token_logprobs(y, targets, top=64), y, targets, 64)


@pytest.mark.parametrize("n", [4, 1100])
def test_nan_and_infinity_stay_in_their_rows(P, n):
    x = logits_of(n, 9000, torch.float32, seed=9)
    clean = x.clone()
    x[1, 4321] = math.nan
    x[2, 8999] = math.inf
    x[3] = math.nan
    targets = torch.full((n,), 17, dtype=torch.int32, device="cuda")
    got = P.ivfpq_token_logprobs(x, targets, top=5)
    want = P.ivfpq_token_logprobs(clean, targets, top=5)
    for r in (1, 2, 3):
        assert torch.isnan(got.logprobs[r]) and torch.isnan(got.entropy[r]) and torch.isnan(got.norms[r, 1])
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[1:4] = False
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep])
    grad = P.ivfpq_token_logprobs_backward(x, targets, got.norms, got.entropy, torch.ones(n, device="cuda"), torch.ones(n, device="cuda"))
    assert torch.isnan(grad[1]).all() and torch.isnan(grad[2]).all() and torch.isfinite(grad[keep]).all()


def test_targets_outside_of_the_vocabulary(P):
    x = logits_of(6, 333, torch.bfloat16, seed=1)
    targets = torch.tensor([-1, 333, 2 ** 31 - 1, -(2 ** 31), 0, 332], dtype=torch.int32, device="cuda")
    got = P.ivfpq_token_logprobs(x, targets)
    assert got.logprobs[:4].eq(0).all() and got.logprobs[4:].lt(0).all() and got.top_tokens is None
    grad = P.ivfpq_token_logprobs_backward(x, targets, got.norms, None, torch.ones(6, device="cuda"))
    assert grad[:4].eq(0).all() and grad[4:].ne(0).any(dim=1).all()
    alone = P.ivfpq_token_logprobs(x)
    assert alone.logprobs is None and torch.equal(alone.entropy, got.entropy)


def listed_for(n, vocab, k, seed, x):
    gen = torch.Generator().manual_seed(seed)
    tokens = torch.stack([torch.randperm(vocab, generator=gen)[:k] for _ in range(n)]).int()
    if n > 1:
        tokens[:, : k // 2] = torch.topk(x.cpu().float(), k // 2, dim=1).indices.int()       # half of them likely ones
        for r in range(n):                                                                   # ... all distinct
            seen = set()
            for j in range(k):
                t = int(tokens[r, j])
                while t in seen:
                    t = (t + 1) % vocab
                seen.add(t)
                tokens[r, j] = t
    logq = torch.log_softmax(torch.randn(n, k, generator=gen) * 2, dim=1)
    for r in range(n):
        used = k if r % 3 == 0 else int(torch.randint(0, k + 1, (1,), generator=gen))
        if used:
            logq[r, :used] -= torch.logsumexp(logq[r, :used], 0)
        tokens[r, used:], logq[r, used:] = -1, -math.inf
    return tokens.cuda(), logq.cuda()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab,k,top,weight", [(1, 40, 1, 5, 0.5), (5, 1000, 16, 20, 0.25), (1, 131072, 64, 20, 0.25), (7, 50001, 128, 128, 0.9),
                                                  (1050, 700, 10, 3, 0.01), (3, 5000, 1024, 0, 0.5), (2, 30, 20, 20, 0.3)])
def test_mixture_with_listed_tokens(P, dtype, n, vocab, k, top, weight):
    x = logits_of(n, vocab, dtype, seed=k)
    if n > 4:
        x[4] = -math.inf
    near = listed_for(n, vocab, k, seed=vocab, x=x.clamp(min=-1e4))
    targets = torch.randint(vocab, (n,), generator=torch.Generator().manual_seed(2)).int().cuda()
    some = near[0][:, 0] >= 0
    targets = torch.where(some & (torch.arange(n, device="cuda") % 2 == 0), near[0][:, 0], targets)
    got = P.ivfpq_token_logprobs(x, targets, top=top, neighbours=near, weight=weight)
    logp, _, norms = reference(x)
    tokens, logq = (t.cpu() for t in near)
    used = tokens >= 0
    w = torch.where(used.any(dim=1, keepdim=True), weight, 0.0).double()
    w = torch.where((norms[:, :1] == -math.inf) & used.any(dim=1, keepdim=True), 1.0, w)
    m = (1 - w) * logp.exp()
    m.scatter_add_(1, tokens.clamp(min=0).long(), w * torch.where(used, logq.double().exp(), 0.0))
    logm = m.log()
    entropy = -torch.where(m > 0, m * logm, 0.0).sum(dim=1)
    # the mixture's terms: each part of log m as above, one more addition and a logarithm; the entropy's exchange is in 64 bits
    c = chain(vocab) + 8
    want = logm.gather(1, targets.cpu().long()[:, None])[:, 0]
    finite = lambda v: torch.where(torch.isfinite(v), v.abs(), 0.0).numpy()
    close(got.logprobs, want, E * (c + 8 * finite(want)))
    close(got.entropy, entropy, E * 4 * c * (1 + entropy.numpy()))
    close(got.norms[:, 0], norms[:, 0], 0.0)
    if top:
        values = got.top_logprobs.cpu().double()
        tokens_got = got.top_tokens.cpu().long()
        there = tokens_got >= 0
        assert (there.sum(dim=1) == (m > 0).sum(dim=1).clamp(max=top)).all()
        lp = torch.where(there, logm.gather(1, tokens_got.clamp(min=0)), -math.inf)
        close(got.top_logprobs, lp, E * (c + 8 * finite(lp)))          # the tokens have these probabilities
        best = torch.sort(logm, dim=1, descending=True).values[:, :top]
        pad = torch.full((n, top - best.shape[1]), -math.inf, dtype=torch.float64)
        close(got.top_logprobs, torch.cat([best, pad], dim=1), E * (c + 8 * finite(torch.cat([best, pad], dim=1))))     # and no others have more
        assert (values[:, 1:] <= values[:, :-1]).all()
        for r in range(n):
            assert len(set(tokens_got[r][there[r]].tolist())) == int(there[r].sum())


def gradient_reference(x, targets, g, h, temperature):
    logp, entropy, _ = reference(x, temperature)
    p = logp.exp()
    vocab = x.shape[1]
    inside = ((targets >= 0) & (targets < vocab)).cpu()
    hot = torch.zeros_like(p).scatter_(1, targets.cpu().long().clamp(0, vocab - 1)[:, None], 1.0) * inside[:, None]
    gg = (g.cpu().double() * inside)[:, None]
    hh = h.cpu().double()[:, None]
    plogp = torch.where(p > 0, p * logp, 0.0)
    grad = gg * (hot - p) - hh * (plogp + p * entropy[:, None])
    size = gg.abs() * (hot + p) + hh.abs() * (plogp.abs() + p * entropy[:, None])
    none = (logp == -math.inf).all(dim=1, keepdim=True)
    t = torch.where(p > 0, logp.abs(), 0.0)
    return torch.where(none, 0.0, grad) / temperature, torch.where(none, 0.0, size * (1 + 4 * t / chain(vocab))) / temperature


def check_gradient(got, want, size, dtype, vocab):
    got = got.detach().cpu().double()
    tol = 2 * E * chain(vocab) * size + 1e-37
    low, high = ((want - tol).to(dtype).double(), (want + tol).to(dtype).double()) if dtype != torch.float32 else (want - tol, want + tol)
    assert bool(((low <= got) & (got <= high)).all()), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab,pad,offset,temperature", [(1, 1, 0, 0, 1.0), (3, 7, 2, 1, 1.0), (5, 64, 0, 0, 0.5), (2, 4097, 7, 3, 1.0), (1, 131073, 0, 1, 2.0),
                                                            (1050, 515, 0, 0, 1.0), (33, 9001, 5, 2, 1.0)])
def test_gradient(P, dtype, n, vocab, pad, offset, temperature):
    x = logits_of(n, vocab, dtype, seed=vocab, pad=pad, offset=offset)
    if n > 2:
        x[1] = LOWEST[dtype]
        x[2, : vocab // 2] = -math.inf
        x[n - 1] = -math.inf
    gen = torch.Generator().manual_seed(n)
    targets = torch.randint(-1, vocab, (n,), generator=gen).int().cuda()
    g, h = torch.randn(n, generator=gen).cuda(), torch.randn(n, generator=gen).cuda()
    s = P.ivfpq_token_logprobs(x, targets, temperature=temperature)
    both = P.ivfpq_token_logprobs_backward(x, targets, s.norms, s.entropy, g, h, temperature=temperature)
    assert both.dtype == dtype
    check_gradient(both, *gradient_reference(x, targets, g, h, temperature), dtype, vocab)
    only = P.ivfpq_token_logprobs_backward(x, targets, s.norms, None, g, temperature=temperature)
    check_gradient(only, *gradient_reference(x, targets, g, torch.zeros_like(h), temperature), dtype, vocab)
    entropy_only = P.ivfpq_token_logprobs_backward(x, None, s.norms, s.entropy, None, h, temperature=temperature)
    check_gradient(entropy_only, *gradient_reference(x, targets, torch.zeros_like(g), h, temperature), dtype, vocab)
    # another layout of the result, and over the logits themselves: the same bits
    wide = torch.full((n, vocab + 3), 5.0, dtype=dtype, device="cuda")
    P.ivfpq_token_logprobs_backward(x, targets, s.norms, s.entropy, g, h, temperature=temperature, out=wide[:, 1:vocab + 1])
    assert torch.equal(wide[:, 1:vocab + 1], both)
    assert (wide[:, 0] == 5).all() and (wide[:, vocab + 1:] == 5).all()
    over = P.ivfpq_token_logprobs_backward(x, targets, s.norms, s.entropy, g, h, temperature=temperature, out=x)
    assert over is x and torch.equal(x, both)


def test_gradient_against_differences(P):
    """Central differences of the library's own log-probability and entropy: step 2^-6, off by step^2 / 6 times a third
    derivative (at most 2 of log p, under 10 of these entropies) and by 2 e (66 + 40) / step."""
    vocab, step = 37, 2.0 ** -6
    x = logits_of(1, vocab, torch.float32, seed=8)
    targets = torch.full((2 * vocab,), 11, dtype=torch.int32, device="cuda")
    eye = torch.eye(vocab, device="cuda") * step
    moved = P.ivfpq_token_logprobs(torch.cat([x + eye, x - eye]), targets)
    g, h = 0.75, -1.5
    value = g * moved.logprobs.double() + h * moved.entropy.double()
    differences = (value[:vocab] - value[vocab:]) / (2 * step)
    s = P.ivfpq_token_logprobs(x, targets[:1])
    grad = P.ivfpq_token_logprobs_backward(x, targets[:1], s.norms, s.entropy, torch.tensor([g], device="cuda"), torch.tensor([h], device="cuda"))
    bound = step ** 2 / 6 * (abs(g) * 2 + abs(h) * 10) + (abs(g) + abs(h)) * 2 * E * 106 / step
    assert float((grad[0].double() - differences).abs().max()) < bound


def test_streams_and_graph(P):
    """On another stream than the default one, and captured: replays on new data give what eager calls give."""
    x = logits_of(3, 30000, torch.bfloat16, seed=4)
    targets = torch.tensor([5, 6, 7], dtype=torch.int32, device="cuda")
    ones = torch.ones(3, device="cuda")
    side = torch.cuda.Stream()

    def step():
        s = P.ivfpq_token_logprobs(x, targets, top=8)
        return [*s, P.ivfpq_token_logprobs_backward(x, targets, s.norms, s.entropy, ones, ones)]

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for seed in (10, 11, 12):
        x.copy_(logits_of(3, 30000, torch.bfloat16, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_same_inputs_same_bits(P):
    x = logits_of(1100, 12001, torch.bfloat16, seed=6)
    targets = torch.zeros(1100, dtype=torch.int32, device="cuda")
    first = P.ivfpq_token_logprobs(x, targets, top=50)
    for _ in range(3):
        for a, b in zip(P.ivfpq_token_logprobs(x, targets, top=50), first):
            assert torch.equal(a, b)
    # and a row's results do not depend on how many rows there are, but for the order of its sums
    few = P.ivfpq_token_logprobs(x[:2], targets[:2], top=50)
    assert torch.equal(few.top_tokens, first.top_tokens[:2])


def test_no_rows(P):
    x = torch.empty((0, 100), device="cuda")
    got = P.ivfpq_token_logprobs(x, torch.empty(0, dtype=torch.int32, device="cuda"), top=4)
    assert got.logprobs.shape == (0,) and got.top_tokens.shape == (0, 4)


def test_a_large_matrix_past_32_bit_offsets(P):
    """Rows that begin more than 2^31 values into the matrix."""
    vocab, stride = 1000, 1_100_000
    n = 2 ** 31 // stride + 3
    room = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((n, vocab), (stride, 1))
    x.copy_(logits_of(n, vocab, torch.bfloat16, seed=3))
    targets = torch.arange(n, dtype=torch.int32, device="cuda") % vocab
    ones = torch.ones(n, device="cuda")
    got = P.ivfpq_token_logprobs(x, targets, top=3)
    near = x.contiguous()
    want = P.ivfpq_token_logprobs(near, targets, top=3)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    grad = P.ivfpq_token_logprobs_backward(x, targets, got.norms, got.entropy, ones, ones, out=x)
    assert torch.equal(grad, P.ivfpq_token_logprobs_backward(near, targets, got.norms, got.entropy, ones, ones))
