"""What the language-model calls refuse, through the C ABI and the binding.  A refused call returns before it touches any pointer, so
the addresses here are numbers only; no GPU is needed."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def P():
    import os
    import paper_2301_06672_amd as pkg
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2301_06672_amd.build import build
        build()
    pkg.lib()
    return pkg


A = 1 << 20          # an aligned address
F = ctypes.c_float


def refused(P, call, args, status, needle):
    assert getattr(P.lib(), call)(*args) == status, call
    assert needle in P.lib().ivfpq_last_error().decode(), P.lib().ivfpq_last_error()


SCORE = dict(logits=A, dtype=0, n=4, vocab=100, stride=100, targets=A, temperature=1.0, top=5, near_tokens=0, near_logprobs=0, k=0, weight=0.0, logprobs=A,
             entropy=A, norms=A, top_tokens=A, top_logprobs=A, ws=A, ws_bytes=1 << 30, stream=0)
BACK = dict(logits=A, dtype=0, n=4, vocab=100, stride=100, targets=A, temperature=1.0, norms=A, entropy=A, by_logprob=A, by_entropy=A, grad=A, grad_stride=100, stream=0)
DISTILL = dict(logits=A, dtype=0, n=4, vocab=100, stride=100, tokens=A, values=A, k=3, temperature=1.0, loss=A, norms=A, ws=A, ws_bytes=1 << 30, stream=0)
DBACK = dict(logits=A, dtype=0, n=4, vocab=100, stride=100, norms=A, tokens=A, values=A, k=3, temperature=1.0, w=0, grad=A, grad_stride=100, stream=0)
STEP = dict(logits=A, dtype=0, n=4, vocab=100, stride=100, tokens=A, values=A, k=3, temperature=1.0, w=0, loss=A, grad=A, grad_stride=100, ws=A, ws_bytes=1 << 30, stream=0)
NEAR = dict(ids=A, dists=A, nq=3, k=10, table=A, n_ids=50, temperature=1.0, tokens=A, logprobs=A, stream=0)
Q8 = dict(a=A, a_stride=64, sa=A, m=3, b=A, b_stride=64, sb=A, n=5, k=50, bias=0, out=A, dtype=0, out_stride=5, stream=0)
QUANT = dict(rows=A, dtype=0, n=3, d=50, stride=50, codes=A, code_stride=64, scales=A, stream=0)

ROWS = [
    (dict(dtype=3), "EINVAL", "dtype"), (dict(dtype=-1), "EINVAL", "dtype"), (dict(n=-1), "EINVAL", "shape"), (dict(vocab=0), "EINVAL", "shape"),
    (dict(vocab=(1 << 30) + 1, stride=1 << 31), "EUNSUPPORTED", "vocab"), (dict(n=(1 << 21) + 1), "EUNSUPPORTED", "rows"), (dict(stride=99), "EINVAL", "stride"),
    (dict(logits=0), "EINVAL", "null"), (dict(logits=A + 2), "EINVAL", "aligned"), (dict(temperature=0.0), "EINVAL", "temperature"),
    (dict(temperature=-1.0), "EINVAL", "temperature"), (dict(temperature=math.nan), "EINVAL", "temperature"), (dict(temperature=math.inf), "EINVAL", "temperature"),
    (dict(temperature=1e-7), "EINVAL", "temperature"),
]
GRADS = [(dict(grad=0), "EINVAL", "null"), (dict(grad=A + 1), "EINVAL", "aligned"), (dict(grad_stride=99), "EINVAL", "gradient stride"),
         (dict(grad=A + 400), "EINVAL", "overlaps"), (dict(grad_stride=101), "EINVAL", "overlaps")]
LISTS = [(dict(k=0), "EINVAL", "k=0"), (dict(k=1025), "EINVAL", "k=1025"), (dict(tokens=0), "EINVAL", "null"), (dict(values=0), "EINVAL", "null")]

CASES = (
    [("ivfpq_token_logprobs", SCORE, *c) for c in ROWS + [
        (dict(top=-1), "EINVAL", "top"), (dict(top=129), "EINVAL", "top"), (dict(k=-1), "EINVAL", "n_neighbours"), (dict(k=1025), "EINVAL", "n_neighbours"),
        (dict(top=128, k=129, weight=0.5), "EUNSUPPORTED", "neighbours"), (dict(k=3, weight=0.0), "EINVAL", "weight"), (dict(k=3, weight=1.0), "EINVAL", "weight"),
        (dict(k=3, weight=math.nan), "EINVAL", "weight"), (dict(k=3, weight=0.5), "EINVAL", "null"), (dict(targets=0), "EINVAL", "together"),
        (dict(logprobs=0), "EINVAL", "together"), (dict(top_tokens=0), "EINVAL", "null"), (dict(top_logprobs=0), "EINVAL", "null"),
        (dict(vocab=100000, stride=100000, ws=0), "EINVAL", "null workspace"), (dict(vocab=100000, stride=100000, ws=A + 16), "EINVAL", "aligned"),
        (dict(vocab=100000, stride=100000, ws_bytes=100), "ENOSPACE", "workspace")]]
    + [("ivfpq_token_logprobs_backward", BACK, *c) for c in [(dict(c[0], grad=c[0].get("grad", A)), *c[1:]) for c in ROWS] + GRADS + [
        (dict(norms=0), "EINVAL", "null"), (dict(by_logprob=0, by_entropy=0), "EINVAL", "neither"), (dict(targets=0), "EINVAL", "targets"),
        (dict(entropy=0), "EINVAL", "entropies")]]
    + [("ivfpq_distill_topk", DISTILL, *c) for c in ROWS + LISTS + [
        (dict(loss=0), "EINVAL", "null"), (dict(norms=0), "EINVAL", "null"), (dict(ws_bytes=0), "ENOSPACE", "workspace"), (dict(ws=0), "EINVAL", "workspace")]]
    + [("ivfpq_distill_topk_backward", DBACK, *c) for c in ROWS + LISTS + GRADS + [(dict(norms=0), "EINVAL", "null")]]
    + [("ivfpq_distill_topk_step", STEP, *c) for c in ROWS + LISTS + GRADS + [(dict(loss=0), "EINVAL", "null"), (dict(ws_bytes=0), "ENOSPACE", "workspace")]]
    + [("ivfpq_neighbour_tokens", NEAR, *c) for c in [
        (dict(nq=-1), "EINVAL", "shape"), (dict(n_ids=-1), "EINVAL", "shape"), (dict(k=0), "EINVAL", "k=0"), (dict(k=1025), "EINVAL", "k=1025"),
        (dict(temperature=0.0), "EINVAL", "temperature"), (dict(temperature=math.nan), "EINVAL", "temperature"), (dict(ids=0), "EINVAL", "null"),
        (dict(dists=0), "EINVAL", "null"), (dict(table=0), "EINVAL", "null"), (dict(tokens=0), "EINVAL", "null"), (dict(logprobs=0), "EINVAL", "null")]]
    + [("ivfpq_q8_matmul", Q8, *c) for c in [
        (dict(dtype=9), "EINVAL", "dtype"), (dict(m=-1), "EINVAL", "shape"), (dict(n=-1), "EINVAL", "shape"), (dict(k=0), "EINVAL", "k=0"),
        (dict(k=65537), "EINVAL", "k=65537"), (dict(a_stride=48), "EINVAL", "strides"), (dict(b_stride=72), "EINVAL", "strides"), (dict(a_stride=(1 << 24) + 16), "EUNSUPPORTED", "strides"),
        (dict(b_stride=1 << 25), "EUNSUPPORTED", "strides"), (dict(a=A + 8), "EINVAL", "16 bytes"),
        (dict(b=A + 1), "EINVAL", "16 bytes"), (dict(out=A + 2), "EINVAL", "aligned"), (dict(out_stride=4), "EINVAL", "output stride"), (dict(a=0), "EINVAL", "null"),
        (dict(sa=0), "EINVAL", "null"), (dict(b=0), "EINVAL", "null"), (dict(sb=0), "EINVAL", "null"), (dict(out=0), "EINVAL", "null")]]
    + [("ivfpq_quantize_rows", QUANT, *c) for c in [
        (dict(dtype=9), "EINVAL", "dtype"), (dict(n=-1), "EINVAL", "shape"), (dict(d=0), "EINVAL", "d=0"), (dict(d=65537), "EINVAL", "d=65537"),
        (dict(stride=49), "EINVAL", "stride"), (dict(code_stride=49), "EINVAL", "stride"), (dict(rows=0), "EINVAL", "null"), (dict(codes=0), "EINVAL", "null"),
        (dict(scales=0), "EINVAL", "null"), (dict(rows=A + 2), "EINVAL", "aligned")]]
)


@pytest.mark.parametrize("call,base,change,status,needle", CASES)
def test_refused(P, call, base, change, status, needle):
    args = dict(base, **change)
    if "grad" in args and "grad" not in change and "overlaps" not in needle:
        args["grad"] = 1 << 40
    refused(P, call, list(args.values()), getattr(P, status), needle)


@pytest.mark.parametrize("call,base,count", [("ivfpq_token_logprobs", SCORE, "n"), ("ivfpq_token_logprobs_backward", BACK, "n"), ("ivfpq_distill_topk", DISTILL, "n"),
                                             ("ivfpq_distill_topk_backward", DBACK, "n"), ("ivfpq_distill_topk_step", STEP, "n"), ("ivfpq_neighbour_tokens", NEAR, "nq"),
                                             ("ivfpq_q8_matmul", Q8, "m"), ("ivfpq_q8_matmul", Q8, "n"), ("ivfpq_quantize_rows", QUANT, "n")])
def test_no_rows_is_no_work(P, call, base, count):
    assert getattr(P.lib(), call)(*dict(base, **{count: 0}).values()) == P.OK


def test_columns_of_one_matrix_may_hold_logits_and_gradient(P):
    """Side by side in rows twice as long they share no value; the missing norms are then what is refused."""
    args = dict(DBACK, stride=200, grad=A + 400, grad_stride=200, norms=0)
    refused(P, "ivfpq_distill_topk_backward", list(args.values()), P.EINVAL, "null")
    args.update(grad=A + 396)
    refused(P, "ivfpq_distill_topk_backward", list(args.values()), P.EINVAL, "overlaps")


def test_workspace_sizes(P):
    L = P.lib()
    assert L.ivfpq_token_logprobs_workspace_bytes(4096, 50000, 20, 0) == 0          # one workgroup a row
    assert L.ivfpq_token_logprobs_workspace_bytes(1, 100000, 20, 0) > L.ivfpq_token_logprobs_workspace_bytes(1, 100000, 0, 0) > 0
    for bad in ((0, 100, 1, 0), (4, 0, 1, 0), (4, 100, -1, 0), (4, 100, 129, 0), (4, 100, 1, 1025)):
        assert L.ivfpq_token_logprobs_workspace_bytes(*bad) == 0
    assert L.ivfpq_distill_topk_workspace_bytes(7, 1000) > 0 and L.ivfpq_distill_topk_workspace_bytes(0, 1000) == 0


def test_the_binding_refuses_tensors_elsewhere(P):
    if torch.cuda.is_available():
        pytest.skip("on the CPU the device check needs no GPU to fail")
    x = torch.zeros(2, 10)
    with pytest.raises((P.IvfpqError, RuntimeError, AssertionError)):
        P.ivfpq_token_logprobs(x)
