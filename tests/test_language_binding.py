"""What the binding of the language-model calls refuses by itself: sizes that no 32-bit argument of the C ABI holds.  Nothing here reaches a
GPU: the tensors have no memory."""
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


def meta(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta")


INT = torch.int32
WIDE = 2 ** 32 + 100            # 100 in 32 bits
CALLS = {
    "quantize_rows": lambda P, k: P.ivfpq_quantize_rows(meta(1, k)),
    "q8_matmul": lambda P, k: P.ivfpq_q8_matmul(meta(1, k, dtype=torch.int8), meta(1), meta(1, k, dtype=torch.int8), meta(1)),
    "neighbour_tokens": lambda P, k: P.ivfpq_neighbour_tokens(meta(1, k, dtype=torch.int64), meta(1, k), meta(5, dtype=INT), 1.0),
    "token_logprobs, vocabulary": lambda P, k: P.ivfpq_token_logprobs(meta(1, k)),
    "token_logprobs, alternatives": lambda P, k: P.ivfpq_token_logprobs(meta(1, 50), top=k),
    "token_logprobs, no alternatives": lambda P, k: P.ivfpq_token_logprobs(meta(1, 50), top=-k),
    "token_logprobs, neighbours": lambda P, k: P.ivfpq_token_logprobs(meta(1, 50), neighbours=(meta(1, k, dtype=INT), meta(1, k)), weight=0.5),
    "token_logprobs_backward": lambda P, k: P.ivfpq_token_logprobs_backward(meta(1, k), meta(1, dtype=INT), meta(1, 2), None, meta(1)),
    "distill_topk, vocabulary": lambda P, k: P.ivfpq_distill_topk(meta(1, k), meta(1, 3, dtype=INT), meta(1, 3)),
    "distill_topk, teacher": lambda P, k: P.ivfpq_distill_topk(meta(1, 50), meta(1, k, dtype=INT), meta(1, k)),
    "distill_topk_backward, vocabulary": lambda P, k: P.ivfpq_distill_topk_backward(meta(1, k), meta(1, 2), meta(1, 3, dtype=INT), meta(1, 3)),
    "distill_topk_backward, teacher": lambda P, k: P.ivfpq_distill_topk_backward(meta(1, 50), meta(1, 2), meta(1, k, dtype=INT), meta(1, k)),
    "distill_topk_step, vocabulary": lambda P, k: P.ivfpq_distill_topk_step(meta(1, k), meta(1, 3, dtype=INT), meta(1, 3)),
    "distill_topk_step, teacher": lambda P, k: P.ivfpq_distill_topk_step(meta(1, 50), meta(1, k, dtype=INT), meta(1, k)),
}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("size", [2 ** 31, WIDE])
def test_sizes_over_32_bits(P, monkeypatch, call, size):
    monkeypatch.setattr(P.binding, "_on_device", lambda what, *tensors: None)
    monkeypatch.setattr(P.binding, "_stream", lambda: None)
    with pytest.raises(P.IvfpqError) as e:
        CALLS[call](P, size)
    assert e.value.status == P.EINVAL and "ivfpq_" + call.split(",")[0] in str(e.value) and str(size) in str(e.value)
