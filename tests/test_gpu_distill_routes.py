"""The one-call distillation on either side of the sizes where its route changes, against the definitions in 64 bits, with the tolerances
derived for the same rows elsewhere."""
import pytest
import torch

from test_gpu_distill import check_grad, check_loss, reference, teacher_for

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


@pytest.mark.parametrize("dtype,n,vocab", [
    (torch.bfloat16, 5, 80000), (torch.bfloat16, 5, 80001), (torch.bfloat16, 111, 80001), (torch.bfloat16, 112, 80001), (torch.float16, 16, 131072),
    (torch.float16, 112, 131072), (torch.float16, 112, 131073), (torch.bfloat16, 15, 50000), (torch.bfloat16, 15, 50001), (torch.float16, 16, 50001),
    (torch.float32, 1, 65536), (torch.float32, 3, 65536), (torch.float32, 3, 65537)])
@pytest.mark.parametrize("offset", [0, 1])
def test_both_sides(P, dtype, n, vocab, offset):
    gen = torch.Generator(device="cuda").manual_seed(n + vocab)
    room = torch.full((n * (vocab + 5) + 1,), 77.0, dtype=dtype, device="cuda")
    x = room[offset:].as_strided((n, vocab), (vocab + 5 if offset else vocab, 1), offset)
    x.copy_((torch.randn(n, vocab, generator=gen, device="cuda") * 3.0).to(dtype))
    few = teacher_for(min(n, 5), vocab, 33, seed=vocab)
    tokens, values = (t.repeat(-(-n // t.shape[0]), 1)[:n].contiguous() for t in few)
    w = torch.randn(n, generator=torch.Generator().manual_seed(n)).cuda()
    loss, grad = P.ivfpq_distill_topk_step(x, tokens, values, w, temperature=1.5)
    want_loss, want_grad, tol_loss, tol_grad = reference(x, tokens, values, 1.5, w)
    check_loss(loss, want_loss, tol_loss)
    check_grad(grad, want_grad, tol_grad)
    kept = x.clone()
    _, over = P.ivfpq_distill_topk_step(x, tokens, values, w, temperature=1.5, out=x)
    assert over is x and torch.equal(x, grad)
    if offset:
        assert (room.as_strided((n, 5), (vocab + 5, 1), offset + vocab)[: n - 1] == 77).all()
    forward, norms = P.ivfpq_distill_topk(kept, tokens, values, temperature=1.5)
    check_loss(forward, want_loss, tol_loss)
    check_grad(P.ivfpq_distill_topk_backward(kept, norms, tokens, values, w, temperature=1.5), want_grad, tol_grad)
