"""What the binding of the language-model calls refuses by itself: sizes that no 32-bit argument of the C ABI holds, and tensors
that are not on the current device.  Nothing here reaches a GPU: refusals come before any launch, and tensors have no memory or are small ones
of the CPU."""
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


class OnDevice(torch.Tensor):
    """A tensor of the CPU that says it is on the current device."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def here(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


ARGUMENTS = {
    "ivfpq_quantize_rows": lambda: dict(rows=here(2, 32)),
    "ivfpq_q8_matmul": lambda: dict(a_codes=here(2, 32, dtype=torch.int8), a_scales=here(2), b_codes=here(3, 32, dtype=torch.int8), b_scales=here(3),
                                    bias=here(3), out=here(2, 3)),
    "ivfpq_neighbour_tokens": lambda: dict(ids=here(2, 4, dtype=torch.int64), dists=here(2, 4), id_tokens=here(9, dtype=INT)),
    "ivfpq_token_logprobs": lambda: dict(logits=here(2, 50), targets=here(2, dtype=INT), neighbour_tokens=here(2, 4, dtype=INT), neighbour_logprobs=here(2, 4)),
    "ivfpq_token_logprobs_backward": lambda: dict(logits=here(2, 50), targets=here(2, dtype=INT), norms=here(2, 2), entropy=here(2), grad_logprobs=here(2),
                                                  grad_entropy=here(2), out=here(2, 50)),
    "ivfpq_distill_topk": lambda: dict(logits=here(2, 50), teacher_tokens=here(2, 4, dtype=INT), teacher_logits=here(2, 4)),
    "ivfpq_distill_topk_backward": lambda: dict(logits=here(2, 50), norms=here(2, 2), teacher_tokens=here(2, 4, dtype=INT), teacher_logits=here(2, 4),
                                                row_grads=here(2), out=here(2, 50)),
    "ivfpq_distill_topk_step": lambda: dict(logits=here(2, 50), teacher_tokens=here(2, 4, dtype=INT), teacher_logits=here(2, 4), row_grads=here(2),
                                            out=here(2, 50)),
}


def call(P, name, args):
    args = dict(args)
    if name == "ivfpq_neighbour_tokens":
        args["temperature"] = 1.0
    if name == "ivfpq_token_logprobs":
        args.update(neighbours=(args.pop("neighbour_tokens"), args.pop("neighbour_logprobs")), weight=0.5)
    return getattr(P, name)(**args)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the tensors that say they are on a device are not")
@pytest.mark.parametrize("name,argument", [(name, argument) for name, make in ARGUMENTS.items() for argument in make()])
@pytest.mark.parametrize("where", ["cpu", "another device", "an array"])
def test_every_tensor_has_to_be_on_the_current_device(P, monkeypatch, name, argument, where):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    args = ARGUMENTS[name]()
    if where == "cpu":
        args[argument] = args[argument].as_subclass(torch.Tensor)
    elif where == "another device":
        args[argument].get_device = lambda: 1
    else:
        args[argument] = args[argument].numpy()
    with pytest.raises(P.IvfpqError) as e:
        call(P, name, args)
    assert e.value.status == P.EINVAL and "not on the current CUDA device" in str(e.value)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the tensors that say they are on a device are not")
@pytest.mark.parametrize("name", ARGUMENTS)
def test_tensors_on_the_current_device_pass(P, monkeypatch, name):
    """... up to the first allocation, which there is no device for."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(P.binding, "lib", lambda: pytest.fail("no launch here"))
    with pytest.raises((RuntimeError, AssertionError)) as e:
        args = ARGUMENTS[name]()
        if "out" in args:
            args["out"] = here(1, 1)               # of another shape: refused behind the check of its device
        call(P, name, args)
    assert "not on the current CUDA device" not in str(e.value)
