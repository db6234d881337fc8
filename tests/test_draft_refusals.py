"""What the calls around drafted tokens refuse, through the C ABI and the binding.  A refused call returns before it touches any pointer, so the addresses
here are numbers only; no GPU is needed."""
import math

import pytest
import torch

A = 1 << 20          # an aligned address
INT = torch.int32


@pytest.fixture(scope="module")
def P():
    import os
    import paper_2301_06672_amd as pkg
    if not os.path.exists(pkg.LIB_PATH):
        from paper_2301_06672_amd.build import build
        build()
    pkg.lib()
    return pkg


DRAFTS = dict(ids=A, dists=A, nq=3, k=10, text=A, n_ids=50, last=A, temperature=1.0, depth=5, m=8, tokens=A, parents=A, depths=A, logprobs=A, counts=A, stream=0)
LAYOUT = dict(n_pages=20, kv_heads=2, page=16, d=64, pages=A, max_pages=9, lens=A)
APPEND = dict(q=A, q_stride=256, heads=4, k=A, k_stride=128, v=A, v_stride=128, dtype=2, n=3, m=5, depths=0, counts=0, inv_freq=A, rotated=64, interleaved=0, amplitude=1.0,
              q_out=A, k_cache=A, v_cache=A, cache_dtype=2, **LAYOUT, stream=0)
ATTENTION = dict(q=A, q_stride=256, heads=4, n=3, m=5, parents=0, counts=0, k_cache=A, v_cache=A, cache_dtype=2, **LAYOUT, max_places=144, scale=0.125, out=A,
                 out_stride=256, lse=0, ws=A, ws_bytes=1 << 30, stream=0)
VERIFY = dict(logits=A, dtype=2, n=3, m=5, vocab=100, stride=100, tokens=A, parents=0, counts=0, uniforms=A, temperature=1.0, drafts=0, draft_stride=0, accept=0, path=A, kept=A,
              following=A, logprobs=A, ws=A, ws_bytes=1 << 30, stream=0)
KEEP = dict(k_cache=A, v_cache=A, cache_dtype=1, layers=2, **LAYOUT, n=3, m=5, path=A, kept=A, stream=0)

CACHES = [
    (dict(cache_dtype=0), "EINVAL", "dtype"), (dict(cache_dtype=7), "EINVAL", "dtype"), (dict(n=-1), "EINVAL", "shape"), (dict(m=0), "EINVAL", "shape"),
    (dict(n_pages=-1), "EINVAL", "shape"), (dict(kv_heads=0), "EINVAL", "shape"), (dict(max_pages=-1), "EINVAL", "shape"), (dict(page=8), "EINVAL", "page=8"),
    (dict(page=48), "EINVAL", "page=48"), (dict(page=512), "EINVAL", "page=512"), (dict(page=0), "EINVAL", "page=0"), (dict(d=0), "EINVAL", "d=0"), (dict(d=60), "EINVAL", "d=60"),
    (dict(d=264), "EINVAL", "d=264"), (dict(kv_heads=4097), "EUNSUPPORTED", "kv_heads"), (dict(n_pages=1 << 31), "EUNSUPPORTED", "n_pages"),
    (dict(max_pages=(1 << 27) - 1), "EUNSUPPORTED", "places"), (dict(n=(1 << 20) + 1), "EUNSUPPORTED", "sequences"), (dict(n=1 << 20, m=17), "EUNSUPPORTED", "rows"),
    (dict(k_cache=0), "EINVAL", "null"), (dict(v_cache=0), "EINVAL", "null"), (dict(pages=0), "EINVAL", "null"), (dict(lens=0), "EINVAL", "null"),
    (dict(k_cache=A + 8), "EINVAL", "16 bytes"), (dict(v_cache=A + 2), "EINVAL", "16 bytes"),
]
CASES = (
    [("ivfpq_neighbour_drafts", DRAFTS, *c) for c in [
        (dict(nq=-1), "EINVAL", "shape"), (dict(n_ids=-1), "EINVAL", "shape"), (dict(k=0), "EINVAL", "k=0"), (dict(k=1025), "EINVAL", "k=1025"), (dict(depth=0), "EINVAL", "depth=0"),
        (dict(depth=16), "EINVAL", "depth=16"), (dict(m=0), "EINVAL", "m=0"), (dict(m=65), "EINVAL", "m=65"), (dict(temperature=0.0), "EINVAL", "temperature"),
        (dict(temperature=math.nan), "EINVAL", "temperature"), (dict(temperature=1e31), "EINVAL", "temperature")] +
        [({name: 0}, "EINVAL", "null") for name in ("ids", "dists", "text", "last", "tokens", "parents", "depths", "logprobs", "counts")]]
    + [("ivfpq_cache_append", APPEND, *c) for c in CACHES + [
        (dict(dtype=3), "EINVAL", "dtype"), (dict(dtype=1), "EINVAL", "16-bit"), (dict(heads=-1), "EINVAL", "heads"), (dict(heads=0), "EINVAL", "heads"), (dict(q=0), "EINVAL", "heads"),
        (dict(q_out=0), "EINVAL", "heads"), (dict(heads=65537, q_stride=1 << 30), "EUNSUPPORTED", "heads"), (dict(rotated=-2), "EINVAL", "rotated"), (dict(rotated=66), "EINVAL", "rotated"),
        (dict(rotated=7), "EINVAL", "rotated"), (dict(inv_freq=0), "EINVAL", "null"), (dict(k=0), "EINVAL", "null"), (dict(v=0), "EINVAL", "null"), (dict(q_stride=255), "EINVAL", "stride"),
        (dict(k_stride=127), "EINVAL", "stride"), (dict(v_stride=-128), "EINVAL", "stride"), (dict(k=A + 1), "EINVAL", "aligned"), (dict(v=A + 1), "EINVAL", "aligned"),
        (dict(q=A + 1), "EINVAL", "aligned"), (dict(q_out=A + 8), "EINVAL", "16 bytes"), (dict(n=1, m=(1 << 20) + 1), "EUNSUPPORTED", "m=")]]
    + [("ivfpq_draft_attention", ATTENTION, *c) for c in CACHES + [
        (dict(heads=3), "EINVAL", "multiple"), (dict(heads=0), "EINVAL", "multiple"), (dict(parents=A, m=65), "EUNSUPPORTED", "tree"), (dict(max_places=-1), "EINVAL", "max_places"),
        (dict(max_places=1 << 31), "EUNSUPPORTED", "max_places"), (dict(scale=math.nan), "EINVAL", "scale"), (dict(scale=math.inf), "EINVAL", "scale"), (dict(q=0), "EINVAL", "null"),
        (dict(out=0), "EINVAL", "null"), (dict(q_stride=255), "EINVAL", "stride"), (dict(q_stride=260), "EINVAL", "stride"), (dict(out_stride=258), "EINVAL", "stride"),
        (dict(out_stride=252), "EINVAL", "stride"), (dict(q=A + 8), "EINVAL", "aligned"), (dict(out=A + 4), "EINVAL", "aligned"), (dict(lse=A + 2), "EINVAL", "aligned"),
        (dict(n=1 << 16, m=1 << 8, heads=8, q_stride=512, out_stride=512), "EUNSUPPORTED", "limits"), (dict(n=1 << 20, kv_heads=16, heads=16, q_stride=1024, out_stride=1024, m=1), "EUNSUPPORTED", "workgroups"),
        (dict(max_places=4096, ws=0), "EINVAL", "null workspace"), (dict(max_places=4096, ws=A + 16), "EINVAL", "aligned"), (dict(max_places=4096, ws_bytes=100), "ENOSPACE", "workspace")]]
    + [("ivfpq_verify_drafts", VERIFY, *c) for c in [
        (dict(dtype=3), "EINVAL", "dtype"), (dict(n=-1), "EINVAL", "shape"), (dict(m=0), "EINVAL", "shape"), (dict(vocab=0), "EINVAL", "shape"), (dict(m=65), "EUNSUPPORTED", "m=65"),
        (dict(vocab=(1 << 30) + 1, stride=1 << 31), "EUNSUPPORTED", "vocab"), (dict(temperature=0.0), "EINVAL", "temperature"), (dict(temperature=math.nan), "EINVAL", "temperature"),
        (dict(temperature=1e7), "EINVAL", "temperature"), (dict(drafts=A, accept=A, draft_stride=100, parents=A), "EINVAL", "chain"), (dict(drafts=A, draft_stride=100), "EINVAL", "random numbers"),
        (dict(drafts=A, draft_stride=100, accept=A, uniforms=0), "EINVAL", "random numbers"), (dict(n=1 << 20, m=2), "EUNSUPPORTED", "limits"), (dict(stride=99), "EINVAL", "stride"),
        (dict(drafts=A, accept=A, draft_stride=99), "EINVAL", "draft stride"), (dict(logits=A + 1), "EINVAL", "aligned"), (dict(drafts=A + 1, accept=A, draft_stride=100), "EINVAL", "aligned"),
        (dict(ws=0), "EINVAL", "null workspace"), (dict(ws=A + 16), "EINVAL", "aligned"), (dict(ws_bytes=100), "ENOSPACE", "workspace")] +
        [({name: 0}, "EINVAL", "null") for name in ("logits", "tokens", "path", "kept", "following", "logprobs")]]
    + [("ivfpq_cache_keep", KEEP, *c) for c in CACHES + [
        (dict(layers=0), "EINVAL", "layers"), (dict(layers=4097), "EINVAL", "layers"), (dict(path=0), "EINVAL", "null"), (dict(kept=0), "EINVAL", "null"),
        (dict(layers=4096, kv_heads=4096, d=256), "EUNSUPPORTED", "components"), (dict(n=1, m=(1 << 20) + 1), "EUNSUPPORTED", "m=")]]
)


@pytest.mark.parametrize("call,base,change,status,needle", CASES)
def test_refused(P, call, base, change, status, needle):
    args = list(dict(base, **change).values())
    assert getattr(P.lib(), call)(*args) == getattr(P, status), call
    assert needle in P.lib().ivfpq_last_error().decode() and call in P.lib().ivfpq_last_error().decode(), P.lib().ivfpq_last_error()


@pytest.mark.parametrize("call,base", [("ivfpq_neighbour_drafts", DRAFTS), ("ivfpq_cache_append", APPEND), ("ivfpq_draft_attention", ATTENTION), ("ivfpq_verify_drafts", VERIFY),
                                       ("ivfpq_cache_keep", KEEP)])
def test_no_sequences_are_no_work(P, call, base):
    assert getattr(P.lib(), call)(*dict(base, **{"nq" if "nq" in base else "n": 0}).values()) == P.OK


def test_workspace_sizes(P):
    L = P.lib()
    assert L.ivfpq_draft_attention_workspace_bytes(512, 1, 32, 8, 128, 100_000) == 0             # workgroups enough without dividing the places
    assert L.ivfpq_draft_attention_workspace_bytes(1, 1, 32, 8, 128, 100) == 0                   # nothing to divide
    assert L.ivfpq_draft_attention_workspace_bytes(1, 1, 32, 8, 128, 100_000) > 0
    for bad in ((0, 1, 32, 8, 128, 100_000), (1, 0, 32, 8, 128, 100_000), (1, 1, 33, 8, 128, 100_000), (1, 1, 32, 0, 128, 100_000), (1, 1, 32, 8, 257, 100_000), (1, 1, 32, 8, 128, -1),
                (1, 1, 32, 8, 128, 1 << 40)):
        assert L.ivfpq_draft_attention_workspace_bytes(*bad) == 0
    assert L.ivfpq_verify_drafts_workspace_bytes(3, 5, 100, 1) > L.ivfpq_verify_drafts_workspace_bytes(3, 5, 100, 0) > 0
    assert L.ivfpq_verify_drafts_workspace_bytes(0, 5, 100, 1) == L.ivfpq_verify_drafts_workspace_bytes(3, 65, 100, 1) == L.ivfpq_verify_drafts_workspace_bytes(1 << 20, 2, 100, 0) == 0


# ---- the binding

class OnDevice(torch.Tensor):
    """A tensor of the CPU that says it is on the current device."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def here(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


BF16 = torch.bfloat16
CACHE = lambda: dict(k_cache=here(6, 2, 16, 64, dtype=BF16), v_cache=here(6, 2, 2, 64, 8, dtype=BF16), pages=here(3, 2, dtype=INT), lens=here(3, dtype=INT))
ARGUMENTS = {
    "ivfpq_neighbour_drafts": lambda: dict(ids=here(2, 4, dtype=torch.int64), dists=here(2, 4), text=here(9, dtype=INT), last_tokens=here(2, dtype=INT)),
    "ivfpq_cache_append": lambda: dict(k=here(3, 5, 2, 64, dtype=BF16), v=here(3, 5, 2, 64, dtype=BF16), **CACHE(), q=here(3, 5, 4, 64, dtype=BF16), inv_freq=here(32),
                                       depths=here(3, 5, dtype=INT), counts=here(3, dtype=INT)),
    "ivfpq_draft_attention": lambda: dict(q=here(3, 5, 4, 64, dtype=BF16), **CACHE(), parents=here(3, 5, dtype=INT), counts=here(3, dtype=INT), out=here(3, 5, 4, 64, dtype=BF16)),
    "ivfpq_verify_drafts": lambda: dict(logits=here(6, 50), tokens=here(2, 3, dtype=INT), parents=here(2, 3, dtype=INT), counts=here(2, dtype=INT), uniforms=here(2, 3),
                                        draft_logits=here(4, 50), accept=here(2, 3)),
    "ivfpq_cache_keep": lambda: dict(**CACHE(), path=here(3, 5, dtype=INT), kept=here(3, dtype=INT)),
}


def call(P, name, args):
    more = {"temperature": 1.0} if name == "ivfpq_neighbour_drafts" else {}
    return getattr(P, name)(**args, **more)


@pytest.fixture()
def pretend(P, monkeypatch):
    if torch.cuda.is_available():
        pytest.skip("the tensors that say they are on a device are not")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(P.binding, "_stream", lambda: None)


@pytest.mark.parametrize("name,argument", [(name, argument) for name, make in ARGUMENTS.items() for argument in make()])
@pytest.mark.parametrize("where", ["cpu", "another device", "an array"])
def test_every_tensor_has_to_be_on_the_current_device(P, pretend, name, argument, where):
    args = ARGUMENTS[name]()
    if where == "cpu":
        args[argument] = args[argument].as_subclass(torch.Tensor)
    elif where == "another device":
        args[argument].get_device = lambda: 1
    else:
        args[argument] = args[argument].float().numpy()
    with pytest.raises(P.IvfpqError) as e:
        call(P, name, args)
    assert e.value.status == P.EINVAL and "not on the current CUDA device" in str(e.value)


WRONG = [
    ("ivfpq_neighbour_drafts", dict(ids=(8, torch.int64)), "matrix"), ("ivfpq_neighbour_drafts", dict(dists=(2, 5)), "expected"), ("ivfpq_neighbour_drafts", dict(last_tokens=(3, INT)), "expected"),
    ("ivfpq_neighbour_drafts", dict(text=(9, torch.int64)), "expected"), ("ivfpq_neighbour_drafts", dict(ids=(2, 4, INT)), "expected"),
    ("ivfpq_cache_append", dict(k=(3, 5, 2, 32, BF16)), "rows are"), ("ivfpq_cache_append", dict(k=(2, 5, 2, 64, BF16)), "rows are"), ("ivfpq_cache_append", dict(v=(3, 4, 2, 64, BF16)), "keys"),
    ("ivfpq_cache_append", dict(v=(3, 5, 2, 64)), "rows of"), ("ivfpq_cache_append", dict(q=(3, 4, 4, 64, BF16)), "queries"), ("ivfpq_cache_append", dict(q=(3, 5, 4, 64)), "rows of"),
    ("ivfpq_cache_append", dict(k_cache=(6, 2, 16, 64)), "keys are"), ("ivfpq_cache_append", dict(v_cache=(6, 2, 16, 64, BF16)), "values are"), ("ivfpq_cache_append", dict(lens=(4, INT)), "expected"),
    ("ivfpq_cache_append", dict(depths=(3, 4, INT)), "expected"), ("ivfpq_cache_append", dict(inv_freq=(32, BF16)), "expected"), ("ivfpq_cache_append", dict(pages=(3, INT)), "matrix"),
    ("ivfpq_draft_attention", dict(q=(3, 5, 4, 64)), "queries of"), ("ivfpq_draft_attention", dict(q=(3, 0, 4, 64, BF16)), "queries"), ("ivfpq_draft_attention", dict(parents=(3, 4, INT)), "expected"),
    ("ivfpq_draft_attention", dict(out=(3, 5, 2, 64, BF16)), "out"), ("ivfpq_draft_attention", dict(out=(3, 5, 4, 64)), "out"), ("ivfpq_draft_attention", dict(v_cache=(6, 2, 2, 8, 64, BF16)), "values are"),
    ("ivfpq_verify_drafts", dict(logits=(5, 50)), "rows of logits"), ("ivfpq_verify_drafts", dict(tokens=(6, INT)), "matrix"), ("ivfpq_verify_drafts", dict(draft_logits=(5, 50)), "draft logits"),
    ("ivfpq_verify_drafts", dict(draft_logits=(4, 50, BF16)), "draft logits"), ("ivfpq_verify_drafts", dict(uniforms=(2, 2)), "expected"), ("ivfpq_verify_drafts", dict(logits=(6, 50, torch.float64)), "matrix"),
    ("ivfpq_cache_keep", dict(path=(3, INT)), "matrix"), ("ivfpq_cache_keep", dict(kept=(2, INT)), "expected"), ("ivfpq_cache_keep", dict(k_cache=(16, 64, BF16)), "keys are"),
]


@pytest.mark.parametrize("name,change,needle", WRONG)
def test_shapes_and_types_refused(P, pretend, monkeypatch, name, change, needle):
    monkeypatch.setattr(torch, "empty", lambda *a, **k: here(1))                     # no device to allocate on
    args = ARGUMENTS[name]()
    for key, spec in change.items():
        dtype = spec[-1] if isinstance(spec[-1], torch.dtype) else torch.float32
        args[key] = here(*(x for x in spec if not isinstance(x, torch.dtype)), dtype=dtype)
    with pytest.raises(P.IvfpqError) as e:
        call(P, name, args)
    assert e.value.status == P.EINVAL and name in str(e.value) and needle in str(e.value), str(e.value)


def test_caches_are_taken_as_they_are(P, pretend):
    """A cache is written in place, so a view that would have to be copied is refused."""
    for name in ("ivfpq_cache_append", "ivfpq_draft_attention", "ivfpq_cache_keep"):
        args = ARGUMENTS[name]()
        args["k_cache"] = here(2, 6, 16, 64, dtype=BF16).transpose(0, 1)
        with pytest.raises(P.IvfpqError) as e:
            call(P, name, args)
        assert "contiguous" in str(e.value)


def meta(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta")


WIDE = {
    "neighbour_drafts": lambda P, x: P.ivfpq_neighbour_drafts(meta(1, x, dtype=torch.int64), meta(1, x), meta(5, dtype=INT), meta(1, dtype=INT), 1.0),
    "neighbour_drafts, rows": lambda P, x: P.ivfpq_neighbour_drafts(meta(1, 5, dtype=torch.int64), meta(1, 5), meta(5, dtype=INT), meta(1, dtype=INT), 1.0, rows=x),
    "neighbour_drafts, depth": lambda P, x: P.ivfpq_neighbour_drafts(meta(1, 5, dtype=torch.int64), meta(1, 5), meta(5, dtype=INT), meta(1, dtype=INT), 1.0, depth=x),
    "cache_append, rows": lambda P, x: P.ivfpq_cache_append(meta(1, x, 1, 8, dtype=BF16), meta(1, x, 1, 8, dtype=BF16), meta(1, 1, 16, 8, dtype=BF16), meta(1, 1, 2, 8, 8, dtype=BF16),
                                                           meta(1, 1, dtype=INT), meta(1, dtype=INT)),
    "cache_append, frequencies": lambda P, x: P.ivfpq_cache_append(meta(1, 1, 1, 8, dtype=BF16), meta(1, 1, 1, 8, dtype=BF16), meta(1, 1, 16, 8, dtype=BF16),
                                                                  meta(1, 1, 2, 8, 8, dtype=BF16), meta(1, 1, dtype=INT), meta(1, dtype=INT), inv_freq=meta(x // 2)),
    "draft_attention, heads": lambda P, x: P.ivfpq_draft_attention(meta(1, 1, x, 8, dtype=BF16), meta(1, 1, 16, 8, dtype=BF16), meta(1, 1, 2, 8, 8, dtype=BF16), meta(1, 1, dtype=INT), meta(1, dtype=INT)),
    "draft_attention, pages": lambda P, x: P.ivfpq_draft_attention(meta(1, 1, 1, 8, dtype=BF16), meta(1, 1, 16, 8, dtype=BF16), meta(1, 1, 2, 8, 8, dtype=BF16), meta(1, x, dtype=INT), meta(1, dtype=INT)),
    "verify_drafts": lambda P, x: P.ivfpq_verify_drafts(meta(1, x), meta(1, 1, dtype=INT)),
    "verify_drafts, rows": lambda P, x: P.ivfpq_verify_drafts(meta(x, 5), meta(1, x, dtype=INT)),
    "cache_keep": lambda P, x: P.ivfpq_cache_keep(meta(1, 1, 16, 8, dtype=BF16), meta(1, 1, 2, 8, 8, dtype=BF16), meta(1, 1, dtype=INT), meta(1, dtype=INT), meta(1, x, dtype=INT), meta(1, dtype=INT)),
}


@pytest.mark.parametrize("name", WIDE)
@pytest.mark.parametrize("size", [2 ** 31, 2 ** 32 + 100])
def test_sizes_over_32_bits(P, monkeypatch, name, size):
    monkeypatch.setattr(P.binding, "_on_device", lambda what, *tensors: None)
    monkeypatch.setattr(P.binding, "_stream", lambda: None)
    with pytest.raises(P.IvfpqError) as e:
        WIDE[name](P, size)
    assert e.value.status == P.EINVAL and "ivfpq_" + name.split(",")[0] in str(e.value) and str(size) in str(e.value)
