"""The loss towards a teacher's listed tokens and its gradient, against the definitions in 64 bits.

Tolerances.  e = 2^-24.  As for log-probabilities: log p is off by at most e (vocab / 256 + 64 + 4 |log p|), log P_j by e (64 + 4
|log P_j|) with at most 1024 listed tokens, P_j and p relative to themselves by as much, and the loss adds up to 1024 products in
chains of 4 and a tree of 8: e (16 + ...) of their magnitudes.  A gradient is rounded once more, to nearest."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.float16: -65504.0, torch.bfloat16: torch.finfo(torch.bfloat16).min}


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def logits_of(n, vocab, dtype, seed, pad=0, offset=0):
    gen = torch.Generator().manual_seed(seed)
    room = torch.full((n * (vocab + pad) + offset,), 77.0, dtype=dtype, device="cuda")
    view = room[offset:].as_strided((n, vocab), (vocab + pad, 1), offset)
    view.copy_((torch.randn(n, vocab, generator=gen) * 3.0).to(dtype))
    return view


def teacher_for(n, vocab, k, seed, repeats=False):
    """Listed tokens with unused places (-1, over the vocabulary, at -inf) here and there; rows without any; repeated tokens."""
    gen = torch.Generator().manual_seed(seed)
    tokens = torch.randint(vocab, (n, k), generator=gen)
    if not repeats and k <= vocab:
        tokens = torch.stack([torch.randperm(vocab, generator=gen)[:k] for _ in range(n)])
    values = torch.randn(n, k, generator=gen) * 3
    off = torch.rand(n, k, generator=gen) < 0.2
    off[0] = False
    if n > 2:
        off[2] = True
    which = torch.randint(3, (n, k), generator=gen)
    tokens = torch.where(off & (which == 0), -1, tokens)
    tokens = torch.where(off & (which == 1), vocab + tokens, tokens)
    values = torch.where(off & (which == 2), -math.inf, values)
    return tokens.int().cuda(), values.cuda()


def reference(x, tokens, values, temperature, w=None):
    """-> loss and gradient in 64 bits, and their tolerances before a rounding of the gradient."""
    vocab = x.shape[1]
    raw = x.detach().cpu().double()
    tokens, values = tokens.cpu().long(), values.cpu().double()
    used = (tokens >= 0) & (tokens < vocab) & (values > -math.inf)
    at = torch.where(used, tokens, 0)
    none = (raw == -math.inf).all(dim=1, keepdim=True)
    logp = torch.where(none, -math.inf, torch.log_softmax((raw - torch.where(none, 0.0, raw.amax(dim=1, keepdim=True))) / temperature, dim=1))
    t = torch.where(used, values / temperature, -math.inf)
    any_used = used.any(dim=1, keepdim=True)
    log_share = torch.where(used, t - torch.where(any_used, torch.logsumexp(t, dim=1, keepdim=True), 0.0), -math.inf)
    share = log_share.exp()
    lp = logp.gather(1, at)
    terms = torch.where(share > 0, share * (log_share - lp), 0.0)
    loss = terms.sum(dim=1) * temperature ** 2
    chain = vocab / 256 + 64
    finite = lambda v: torch.where(torch.isfinite(v), v.abs(), 0.0)
    loss_tol = E * (share * (chain + 80 + 8 * finite(log_share) + 8 * finite(lp)) * (1 + finite(log_share) + finite(lp))).sum(dim=1) * temperature ** 2
    grad = loss_tol2 = None
    if w is not None:
        teacher = torch.zeros_like(raw).scatter_add_(1, at, torch.where(used, share, 0.0))
        p = logp.exp() * any_used
        scale = temperature * w.cpu().double()[:, None]
        grad = torch.where(none, 0.0, (p - teacher) * scale)
        loss_tol2 = E * scale.abs() * (p * (chain + 8 + 4 * finite(logp)) + teacher * (80 + tokens.shape[1] + 4 * finite(teacher.log())))
    return loss, grad, loss_tol, loss_tol2


def check_loss(got, want, tol):
    got = got.cpu().double()
    finite = torch.isfinite(want)
    assert torch.equal(got[~finite], want[~finite])
    assert bool(((got - want).abs()[finite] <= tol[finite]).all()), float(((got - want).abs() / tol)[finite].max())


def check_grad(got, want, tol):
    dtype = got.dtype
    got = got.cpu().double()
    tol = tol + 1e-37
    low, high = ((want - tol).to(dtype).double(), (want + tol).to(dtype).double()) if dtype != torch.float32 else (want - tol, want + tol)
    assert bool(((low <= got) & (got <= high)).all()), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab,k,temperature,pad,offset,repeats", [
    (1, 1, 1, 1.0, 0, 0, False), (3, 7, 5, 2.0, 2, 1, False), (5, 64, 64, 1.0, 0, 0, False), (4, 4097, 100, 0.5, 7, 3, False), (1, 131073, 20, 1.0, 0, 1, False),
    (8, 50001, 1024, 1.0, 0, 0, True), (1050, 515, 65, 4.0, 0, 0, True), (1100, 3001, 10, 1.0, 3, 1, False), (6, 30, 300, 1.0, 0, 0, True),
    (3, 140000, 33, 1.0, 0, 0, False), (1030, 70001, 20, 1.0, 1, 0, False),
    (20, 50001, 100, 1.0, 0, 1, True), (17, 30000, 64, 2.0, 4, 0, False)])
def test_loss_and_gradient(P, dtype, n, vocab, k, temperature, pad, offset, repeats):
    x = logits_of(n, vocab, dtype, seed=n + k, pad=pad, offset=offset)
    tokens, values = teacher_for(n, vocab, k, seed=vocab, repeats=repeats)
    if n > 3:
        x[1, 0] = -math.inf
        tokens[1, 0] = 0
        values[1, 0] = 1.0                       # the teacher's token is masked: the loss is infinite
        x[3] = LOWEST[dtype]
    if n > 4:
        x[4] = -math.inf
    w = torch.randn(n, generator=torch.Generator().manual_seed(n)).cuda()
    loss, norms = P.ivfpq_distill_topk(x, tokens, values, temperature=temperature)
    grad = P.ivfpq_distill_topk_backward(x, norms, tokens, values, w, temperature=temperature)
    want_loss, want_grad, tol_loss, tol_grad = reference(x, tokens, values, temperature, w)
    check_loss(loss, want_loss, tol_loss)
    check_grad(grad, want_grad, tol_grad)
    step_loss, step_grad = P.ivfpq_distill_topk_step(x, tokens, values, w, temperature=temperature)
    check_loss(step_loss, want_loss, tol_loss)
    check_grad(step_grad, want_grad, tol_grad)
    ones = P.ivfpq_distill_topk_step(x, tokens, values, temperature=temperature)[1]
    check_grad(ones, *(reference(x, tokens, values, temperature, torch.ones(n))[i] for i in (1, 3)))
    # another layout of the gradient, and over the logits: the same bits
    wide = torch.full((n, vocab + 5), 3.0, dtype=dtype, device="cuda")
    P.ivfpq_distill_topk_step(x, tokens, values, w, temperature=temperature, out=wide[:, 1:vocab + 1])
    assert torch.equal(wide[:, 1:vocab + 1], step_grad) and (wide[:, 0] == 3).all() and (wide[:, vocab + 1:] == 3).all()
    copy = x.clone()
    P.ivfpq_distill_topk_backward(copy, norms, tokens, values, w, temperature=temperature, out=copy)
    assert torch.equal(copy, grad)
    _, over = P.ivfpq_distill_topk_step(x, tokens, values, w, temperature=temperature, out=x)
    assert over is x and torch.equal(x, step_grad)


def test_nan_stays_in_its_row(P):
    n, vocab = 6, 5000
    x = logits_of(n, vocab, torch.float32, seed=2)
    tokens, values = teacher_for(n, vocab, 8, seed=3)
    clean = P.ivfpq_distill_topk_step(x, tokens, values)
    x[0, 4000] = math.nan
    values[5, 0], tokens[5, 0] = math.nan, 1
    loss, grad = P.ivfpq_distill_topk_step(x, tokens, values)
    assert torch.isnan(loss[[0, 5]]).all() and torch.isnan(grad[0]).all()
    assert torch.equal(loss[1:5], clean[0][1:5]) and torch.equal(grad[1:5], clean[1][1:5])


def test_gradient_against_differences(P):
    """Central differences of the library's own loss: step 2^-6, off by step^2 / 6 times a third derivative (under 1) and by
    2 e (66 + 80 + 80) / step."""
    vocab, step, temperature = 41, 2.0 ** -6, 1.5
    x = logits_of(1, vocab, torch.float32, seed=8)
    tokens, values = teacher_for(1, vocab, 12, seed=4, repeats=True)
    eye = torch.eye(vocab, device="cuda") * step
    n = 2 * vocab
    value, _ = P.ivfpq_distill_topk(torch.cat([x + eye, x - eye]), tokens.expand(n, -1), values.expand(n, -1), temperature=temperature)
    differences = (value[:vocab].double() - value[vocab:].double()) / (2 * step)
    _, grad = P.ivfpq_distill_topk_step(x, tokens, values, temperature=temperature)
    bound = step ** 2 / 6 + temperature ** 2 * 2 * E * 226 * 8 / step
    assert float((grad[0].double() - differences).abs().max()) < bound


def test_alternatives_as_a_teacher(P):
    """The best tokens of one model's rows are what another one is trained towards: at the teacher's own logits the gradient is that
    of what the list leaves out."""
    x = logits_of(9, 2000, torch.float32, seed=6)
    best = P.ivfpq_token_logprobs(x, top=128)
    loss, grad = P.ivfpq_distill_topk_step(x, best.top_tokens, best.top_logprobs)
    kept = best.top_logprobs.double().exp().sum(dim=1)
    # P = p / kept on the list: the loss is -log kept, and each listed token's gradient p - p / kept
    assert float((loss.double() + kept.log()).abs().max()) < E * 400
    listed = grad.gather(1, best.top_tokens.long()).double()
    p = best.top_logprobs.double().exp()
    assert float((listed - (p - p / kept[:, None])).abs().max()) < E * 400


def test_streams_and_graph(P):
    x = logits_of(40, 9000, torch.bfloat16, seed=4)
    tokens, values = teacher_for(40, 9000, 30, seed=1)
    side = torch.cuda.Stream()

    def step():
        return P.ivfpq_distill_topk_step(x, tokens, values)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for seed in (10, 11, 12):
        x.copy_(logits_of(40, 9000, torch.bfloat16, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
