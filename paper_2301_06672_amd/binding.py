"""ctypes binding of libivfpq.so: argument marshalling only.

Function names mirror the C ABI in include/ivfpq.h.  PyTorch is used for device memory
(`torch.empty(..., device="cuda")`) and for the current HIP stream -- nothing is computed here.
There is no CPU fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional

import numpy as np
import torch  # imported before the library so that both share one HIP runtime

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libivfpq.so")

LUT_FP32, LUT_FP16, LUT_FP8_E5M3, LUT_FP8_E4M4 = 0, 1, 2, 3
LUT_NAMES = {LUT_FP32: "fp32", LUT_FP16: "fp16", LUT_FP8_E5M3: "e5m3", LUT_FP8_E4M4: "e4m4"}
LUT_BYTES = {LUT_FP32: 4, LUT_FP16: 2, LUT_FP8_E5M3: 1, LUT_FP8_E4M4: 1}
ROUND_NEAREST, ROUND_TRUNCATE = 0, 1
MAX_K = 1024
MAX_PROBES = 1024
STATIC_SCRATCH_BYTES = 64 << 20
TUNE_SCAN_THREADS, TUNE_ORDER_BLOCK, TUNE_SCAN_SHARE, TUNE_EARLY_EXIT, TUNE_LDS_PAD, TUNE_SCAN_ROUTE = 0, 1, 2, 3, 4, 5

MAX_TOP, MAX_LISTED, MAX_MIXED, MAX_Q8_K = 128, 1024, 256, 65536
MAX_DRAFT, MAX_DRAFT_DEPTH, MAX_HEAD = 64, 15, 256
VALUES_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

OK, EINVAL, ENOSPACE, EHIP, EUNSUPPORTED, ESTATE = 0, -1, -2, -3, -4, -5

# every symbol include/ivfpq.h declares
EXPORTS = (
    "ivfpq_build_host", "ivfpq_build_device", "ivfpq_build_device_workspace_bytes", "ivfpq_assign_device",
    "ivfpq_assign_device_workspace_bytes", "ivfpq_index_from_arrays", "ivfpq_index_info", "ivfpq_index_export", "ivfpq_free",
    "ivfpq_set_e4m4_bias", "ivfpq_set_fp8_encoding", "ivfpq_set_workspace_limit", "ivfpq_set_tuning",
    "ivfpq_device_bytes", "ivfpq_upload", "ivfpq_search_workspace_bytes", "ivfpq_search", "ivfpq_search_static",
    "ivfpq_select_probes", "ivfpq_search_with_probes", "ivfpq_dump_lut", "ivfpq_scan_list", "ivfpq_refine",
    "ivfpq_set_stage_timing", "ivfpq_stage_times_ms", "ivfpq_scan_kernel_info", "ivfpq_stream_read", "ivfpq_last_error",
    "ivfpq_quantize_rows", "ivfpq_q8_matmul", "ivfpq_neighbour_tokens", "ivfpq_token_logprobs_workspace_bytes",
    "ivfpq_token_logprobs", "ivfpq_token_logprobs_backward", "ivfpq_distill_topk_workspace_bytes", "ivfpq_distill_topk",
    "ivfpq_distill_topk_backward", "ivfpq_distill_topk_step",
    "ivfpq_neighbour_drafts", "ivfpq_cache_append", "ivfpq_draft_attention_workspace_bytes", "ivfpq_draft_attention",
    "ivfpq_verify_drafts_workspace_bytes", "ivfpq_verify_drafts", "ivfpq_cache_keep",
)


class IvfpqError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"ivfpq status {status}: {message}")
        self.status = status


_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """Loads libivfpq.so (built by `python -m paper_2301_06672_amd.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2301_06672_amd.build` "
                "(there is no fallback implementation)")
        L = ctypes.CDLL(LIB_PATH)
        _declare(L)
        _lib = L
    return _lib


def _declare(L):
    c = ctypes
    vp, i64, i32, u32, u64, sz = c.c_void_p, c.c_int64, c.c_int32, c.c_uint32, c.c_uint64, c.c_size_t
    pp = c.POINTER(c.c_void_p)
    L.ivfpq_build_host.argtypes = [vp, i64, i32, i32, i32, i32, i32, u64, pp]
    L.ivfpq_build_device_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i64, i64]
    L.ivfpq_build_device_workspace_bytes.restype = sz
    L.ivfpq_build_device.argtypes = [vp, i64, i32, i32, i32, i32, i32, vp, i64, vp, vp, i64, vp, u64, vp, sz, vp, pp]
    L.ivfpq_assign_device_workspace_bytes.argtypes = [i64, i32, i32]
    L.ivfpq_assign_device_workspace_bytes.restype = sz
    L.ivfpq_assign_device.argtypes = [vp, i64, i32, vp, i32, vp, vp, sz, vp]
    L.ivfpq_index_from_arrays.argtypes = [i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, pp]
    L.ivfpq_index_info.argtypes = [vp, c.POINTER(i64), c.POINTER(i32), c.POINTER(i32), c.POINTER(i32), c.POINTER(i32)]
    L.ivfpq_index_export.argtypes = [vp, vp, vp, vp, vp, vp]
    L.ivfpq_free.argtypes = [vp]
    L.ivfpq_set_e4m4_bias.argtypes = [vp, i32]
    L.ivfpq_set_workspace_limit.argtypes = [vp, sz]
    L.ivfpq_set_fp8_encoding.argtypes = [vp, i32, i32, i32, i32]
    L.ivfpq_set_tuning.argtypes = [vp, i32, i32]
    L.ivfpq_search_static.argtypes = [vp, vp, i64, i32, i32, i32, vp, vp, vp]
    L.ivfpq_free.restype = None
    L.ivfpq_device_bytes.argtypes = [vp]
    L.ivfpq_device_bytes.restype = sz
    L.ivfpq_upload.argtypes = [vp, vp, sz, vp]
    L.ivfpq_search_workspace_bytes.argtypes = [vp, i64, i32, i32, i32]
    L.ivfpq_search_workspace_bytes.restype = sz
    L.ivfpq_search.argtypes = [vp, vp, i64, i32, i32, i32, vp, vp, vp, sz, vp]
    L.ivfpq_select_probes.argtypes = [vp, vp, i64, i32, vp, vp, vp, sz, vp]
    L.ivfpq_search_with_probes.argtypes = [vp, vp, i64, vp, i32, i32, i32, vp, vp, vp, sz, vp]
    L.ivfpq_dump_lut.argtypes = [vp, vp, u32, i32, vp, vp]
    L.ivfpq_refine.argtypes = [vp, i64, i32, vp, i64, vp, i32, i32, vp, vp, vp]
    L.ivfpq_scan_list.argtypes = [vp, vp, u32, i32, vp, vp]
    L.ivfpq_set_stage_timing.argtypes = [vp, i32]
    L.ivfpq_stage_times_ms.argtypes = [vp, c.POINTER(c.c_float * 8)]
    L.ivfpq_scan_kernel_info.argtypes = [vp, i32, c.c_char_p, sz]
    L.ivfpq_stream_read.argtypes = [vp, sz, vp, i32, vp]
    f32 = c.c_float
    logits = [vp, i32, i64, i32, i64]
    L.ivfpq_quantize_rows.argtypes = [vp, i32, i64, i32, i64, vp, i64, vp, vp]
    L.ivfpq_q8_matmul.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, vp, i32, i64, vp]
    L.ivfpq_neighbour_tokens.argtypes = [vp, vp, i64, i32, vp, i64, f32, vp, vp, vp]
    L.ivfpq_token_logprobs_workspace_bytes.argtypes = [i64, i32, i32, i32]
    L.ivfpq_token_logprobs_workspace_bytes.restype = sz
    L.ivfpq_token_logprobs.argtypes = logits + [vp, f32, i32, vp, vp, i32, f32, vp, vp, vp, vp, vp, vp, sz, vp]
    L.ivfpq_token_logprobs_backward.argtypes = logits + [vp, f32, vp, vp, vp, vp, vp, i64, vp]
    L.ivfpq_distill_topk_workspace_bytes.argtypes = [i64, i32]
    L.ivfpq_distill_topk_workspace_bytes.restype = sz
    L.ivfpq_distill_topk.argtypes = logits + [vp, vp, i32, f32, vp, vp, vp, sz, vp]
    L.ivfpq_distill_topk_backward.argtypes = logits + [vp, vp, vp, i32, f32, vp, vp, i64, vp]
    L.ivfpq_distill_topk_step.argtypes = logits + [vp, vp, i32, f32, vp, vp, vp, i64, vp, sz, vp]
    f64 = c.c_double
    L.ivfpq_neighbour_drafts.argtypes = [vp, vp, i64, i32, vp, i64, vp, f64, i32, i32, vp, vp, vp, vp, vp, vp]
    layout = [i64, i32, i32, i32, vp, i32, vp]
    L.ivfpq_cache_append.argtypes = [vp, i64, i32, vp, i64, vp, i64, i32, i64, i32, vp, vp, vp, i32, i32, f32, vp, vp, vp, i32] + layout + [vp]
    L.ivfpq_draft_attention_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i64]
    L.ivfpq_draft_attention_workspace_bytes.restype = sz
    L.ivfpq_draft_attention.argtypes = [vp, i64, i32, i64, i32, vp, vp, vp, vp, i32] + layout + [i64, f32, vp, i64, vp, vp, sz, vp]
    L.ivfpq_verify_drafts_workspace_bytes.argtypes = [i64, i32, i32, i32]
    L.ivfpq_verify_drafts_workspace_bytes.restype = sz
    L.ivfpq_verify_drafts.argtypes = [vp, i32, i64, i32, i32, i64, vp, vp, vp, vp, f64, vp, i64, vp, vp, vp, vp, vp, vp, sz, vp]
    L.ivfpq_cache_keep.argtypes = [vp, vp, i32, i32] + layout + [i64, i32, vp, vp, vp]
    L.ivfpq_last_error.restype = c.c_char_p
    for name in EXPORTS:
        fn = getattr(L, name)
        if fn.restype is c.c_int:      # default: status code
            fn.restype = c.c_int


def _check(status: int):
    if status != OK:
        raise IvfpqError(status, lib().ivfpq_last_error().decode("utf-8", "replace"))


def _np(a, dtype):
    return np.ascontiguousarray(a, dtype=dtype)


def _hp(a: np.ndarray):
    return a.ctypes.data_as(ctypes.c_void_p)


def _dp(t: Optional[torch.Tensor]):
    # an int, which ctypes takes for a pointer by the declared types; an object for it would take as long as the conversion of ten
    return t.data_ptr() if t is not None else None


def _stream():
    # the current stream's handle; torch.cuda.current_stream() makes an object for it first, which takes longer than a launch
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _dev_f32(x) -> torch.Tensor:
    if isinstance(x, torch.Tensor):
        assert x.is_cuda and x.dtype == torch.float32
        return x.contiguous()
    return torch.from_numpy(_np(x, np.float32)).cuda()


def ivfpq_assign_device(rows, centres) -> torch.Tensor:
    """-> int32 CUDA tensor: the nearest centre of every row (k-means assignment step)."""
    x, c = _dev_f32(rows), _dev_f32(centres)
    assert x.shape[1] == c.shape[1]
    need = lib().ivfpq_assign_device_workspace_bytes(int(x.shape[0]), int(x.shape[1]), int(c.shape[0]))
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    labels = torch.empty(int(x.shape[0]), dtype=torch.int32, device="cuda")
    _check(lib().ivfpq_assign_device(_dp(x), int(x.shape[0]), int(x.shape[1]), _dp(c), int(c.shape[0]), _dp(labels),
                                     _dp(ws), need, _stream()))
    torch.cuda.current_stream().synchronize()
    return labels


def ivfpq_refine(data: torch.Tensor, queries, cand_ids: torch.Tensor, k: int):
    """-> (ids [nq][k] int64, dists [nq][k] fp32): candidates re-ranked by exact distance to rows of `data` (CUDA)."""
    assert data.is_cuda and data.dtype == torch.float32 and data.is_contiguous()
    q = _dev_f32(queries)
    cand = cand_ids.contiguous()
    assert cand.is_cuda and cand.dtype == torch.int64 and cand.shape[0] == q.shape[0]
    ids = torch.empty((q.shape[0], k), dtype=torch.int64, device="cuda")
    dists = torch.empty((q.shape[0], k), dtype=torch.float32, device="cuda")
    _check(lib().ivfpq_refine(_dp(data), int(data.shape[0]), int(data.shape[1]), _dp(q), int(q.shape[0]), _dp(cand),
                              int(cand.shape[1]), int(k), _dp(ids), _dp(dists), _stream()))
    return ids, dists


def ivfpq_stream_read(buf: torch.Tensor, n_out: int = 8192) -> torch.Tensor:
    """-> uint32-as-int32 [n_out]: per-workgroup XOR of the 32-bit words of `buf` (CUDA, size a multiple of 16 bytes)."""
    assert buf.is_cuda and buf.is_contiguous()
    out = torch.empty(n_out, dtype=torch.int32, device="cuda")
    _check(lib().ivfpq_stream_read(_dp(buf), buf.numel() * buf.element_size(), _dp(out), int(n_out), _stream()))
    return out


# ---- language models around a search.  Inputs are CUDA tensors on the current device; rows may have any stride, the values
# of a row are contiguous.

class TokenLogprobs(NamedTuple):
    logprobs: Optional[torch.Tensor]       # [n] of the targets; None without targets
    entropy: torch.Tensor                  # [n]
    norms: torch.Tensor                    # [n][2], for the backward call
    top_tokens: Optional[torch.Tensor]     # [n][top] int32, None with top = 0
    top_logprobs: Optional[torch.Tensor]   # [n][top]


def _refuse(message: str):
    raise IvfpqError(EINVAL, message)


def _on_device(what: str, *tensors):
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and not (isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() == device):
            _refuse(f"{what}: a tensor is not on the current CUDA device")


def _plain(what: str, t: torch.Tensor, dtype, *shape):
    """A contiguous tensor of this type and shape."""
    if t.dtype != dtype or t.shape != shape:
        _refuse(f"{what}: expected {dtype} {shape}, got {t.dtype} {tuple(t.shape)}")
    return t.contiguous()


def _fits_int32(what: str, size: int):
    """Row lengths are int32 in the C ABI, and ctypes cuts what is over that without a word."""
    if size > 2 ** 31 - 1:
        _refuse(f"{what}: rows of {size} values (limit 2^31 - 1)")


def _value_rows(what: str, x: torch.Tensor) -> torch.Tensor:
    if x.dim() != 2 or x.dtype not in VALUES_DTYPES:
        _refuse(f"{what}: expected a matrix of float32, float16 or bfloat16, got {x.dtype} {tuple(x.shape)}")
    _fits_int32(what, x.shape[1])
    return x if _rows_apart(x) else x.contiguous()


def _rows_apart(x: torch.Tensor) -> bool:
    """Whether a row's values are contiguous and rows do not overlap."""
    n, d = x.shape
    return (d <= 1 or x.stride(1) == 1) and (n <= 1 or x.stride(0) >= d)


def _grad_like(what: str, logits: torch.Tensor, out: Optional[torch.Tensor]) -> torch.Tensor:
    if out is None:
        return torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _on_device(what, out)
    if out.shape != logits.shape or out.dtype != logits.dtype or not _rows_apart(out):
        _refuse(f"{what}: out has another shape, type or layout than the logits")
    return out


def _listed(what: str, tokens: torch.Tensor, values: torch.Tensor, n: int):
    if tokens.dim() != 2:
        _refuse(f"{what}: listed tokens are a matrix")
    k = tokens.shape[1]
    _fits_int32(what, k)
    return _plain(what, tokens, torch.int32, n, k), _plain(what, values, torch.float32, n, k)


def _scratch(nbytes: int) -> Optional[torch.Tensor]:
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def _logits(x: torch.Tensor):
    return _dp(x), VALUES_DTYPES[x.dtype], x.shape[0], x.shape[1], x.stride(0)


def ivfpq_quantize_rows(rows: torch.Tensor):
    """-> (codes int8 [n][d], scales fp32 [n]); the codes' rows lie a multiple of 16 bytes apart, zeros in between."""
    _on_device("ivfpq_quantize_rows", rows)
    x = _value_rows("ivfpq_quantize_rows", rows)
    n, d = x.shape
    codes = torch.empty((n, -(-d // 16) * 16), dtype=torch.int8, device="cuda")
    scales = torch.empty(n, dtype=torch.float32, device="cuda")
    _check(lib().ivfpq_quantize_rows(_dp(x), VALUES_DTYPES[x.dtype], n, d, x.stride(0), _dp(codes), codes.shape[1], _dp(scales), _stream()))
    return codes[:, :d], scales


def _code_rows(what: str, codes: torch.Tensor):
    """-> (codes, row stride): rows of 16-byte pieces that can all be read, as ivfpq_quantize_rows makes them; other layouts are copied."""
    if codes.dim() != 2 or codes.dtype != torch.int8:
        _refuse(f"{what}: codes are a matrix of int8, got {codes.dtype} {tuple(codes.shape)}")
    n, k = codes.shape
    _fits_int32(what, k)
    width = -(-k // 16) * 16
    stride = codes.stride(0) if n > 1 else width
    fits = (k <= 1 or codes.stride(1) == 1) and stride % 16 == 0 and width <= stride <= 1 << 24 and codes.data_ptr() % 16 == 0 and (
        codes.storage_offset() + (n - 1) * stride + width <= codes.untyped_storage().nbytes())
    if n == 0 or fits:
        return codes, max(stride, width)
    padded = torch.zeros((n, width), dtype=torch.int8, device=codes.device)
    padded[:, :k] = codes
    return padded, width


def ivfpq_q8_matmul(a_codes: torch.Tensor, a_scales: torch.Tensor, b_codes: torch.Tensor, b_scales: torch.Tensor, bias=None,
                    out_dtype=torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """-> [m][n]: a_scales[i] * b_scales[j] * (a_codes[i] . b_codes[j]) + bias[j]."""
    what = "ivfpq_q8_matmul"
    _on_device(what, a_codes, a_scales, b_codes, b_scales, bias, out)
    a, a_stride = _code_rows(what, a_codes)
    b, b_stride = _code_rows(what, b_codes)
    (m, k), n = a_codes.shape, b_codes.shape[0]
    if b_codes.shape[1] != k:
        _refuse(f"{what}: rows of {k} and {b_codes.shape[1]} codes")
    sa, sb = _plain(what, a_scales, torch.float32, m), _plain(what, b_scales, torch.float32, n)
    bias = None if bias is None else _plain(what, bias, torch.float32, n)
    if out is None:
        if out_dtype not in VALUES_DTYPES:
            _refuse(f"{what}: out_dtype {out_dtype}")
        out = torch.empty((m, n), dtype=out_dtype, device="cuda")
    if out.shape != (m, n) or out.dtype not in VALUES_DTYPES or not _rows_apart(out):
        _refuse(f"{what}: out has another shape, type or layout")
    _check(lib().ivfpq_q8_matmul(_dp(a), a_stride, _dp(sa), m, _dp(b), b_stride, _dp(sb), n, k, _dp(bias), _dp(out),
                                 VALUES_DTYPES[out.dtype], out.stride(0), _stream()))
    return out


def ivfpq_neighbour_tokens(ids: torch.Tensor, dists: torch.Tensor, id_tokens: torch.Tensor, temperature: float):
    """-> (tokens int32 [nq][k], log-probabilities fp32 [nq][k]) of search results; id_tokens [n_ids] int32 is the token of every id."""
    what = "ivfpq_neighbour_tokens"
    _on_device(what, ids, dists, id_tokens)
    if ids.dim() != 2:
        _refuse(f"{what}: ids are a matrix")
    nq, k = ids.shape
    _fits_int32(what, k)
    ids, dists = _plain(what, ids, torch.int64, nq, k), _plain(what, dists, torch.float32, nq, k)
    table = _plain(what, id_tokens, torch.int32, id_tokens.numel())
    tokens = torch.empty((nq, k), dtype=torch.int32, device="cuda")
    logprobs = torch.empty((nq, k), dtype=torch.float32, device="cuda")
    _check(lib().ivfpq_neighbour_tokens(_dp(ids), _dp(dists), nq, k, _dp(table), table.numel(), temperature, _dp(tokens), _dp(logprobs), _stream()))
    return tokens, logprobs


def ivfpq_token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 0, temperature: float = 1.0,
                         neighbours=None, weight: float = 0.0) -> TokenLogprobs:
    """Log-probabilities of `targets` (int32 [n]), entropy and the `top` best tokens of rows of logits; neighbours: (tokens,
    log-probabilities) as ivfpq_neighbour_tokens gives them, mixed in with this weight."""
    what = "ivfpq_token_logprobs"
    _on_device(what, logits, targets, *(neighbours or ()))
    x = _value_rows(what, logits)
    n, vocab = x.shape
    if not 0 <= top <= MAX_TOP:
        _refuse(f"{what}: top={top} outside [0, {MAX_TOP}]")
    targets = None if targets is None else _plain(what, targets, torch.int32, n)
    near_tokens, near_logprobs = (None, None) if neighbours is None else _listed(what, *neighbours, n)
    k = 0 if near_tokens is None else near_tokens.shape[1]
    logprobs = None if targets is None else torch.empty(n, dtype=torch.float32, device="cuda")
    entropy = torch.empty(n, dtype=torch.float32, device="cuda")
    norms = torch.empty((n, 2), dtype=torch.float32, device="cuda")
    best = (torch.empty((n, top), dtype=torch.int32, device="cuda"), torch.empty((n, top), dtype=torch.float32, device="cuda")) if top > 0 else (None, None)
    need = lib().ivfpq_token_logprobs_workspace_bytes(n, vocab, top, k)
    ws = _scratch(need)
    _check(lib().ivfpq_token_logprobs(*_logits(x), _dp(targets), temperature, top, _dp(near_tokens), _dp(near_logprobs), k, weight,
                                      _dp(logprobs), _dp(entropy), _dp(norms), _dp(best[0]), _dp(best[1]), _dp(ws), need, _stream()))
    return TokenLogprobs(logprobs, entropy, norms, *best)


def ivfpq_token_logprobs_backward(logits: torch.Tensor, targets: Optional[torch.Tensor], norms: torch.Tensor, entropy: Optional[torch.Tensor],
                                  grad_logprobs: Optional[torch.Tensor], grad_entropy: Optional[torch.Tensor] = None,
                                  temperature: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """-> the gradient with respect to the logits (written to `out`, which may be the logits themselves); norms and entropy of a call
    without neighbours."""
    what = "ivfpq_token_logprobs_backward"
    _on_device(what, logits, targets, norms, entropy, grad_logprobs, grad_entropy)
    x = _value_rows(what, logits)
    n = x.shape[0]
    row = lambda t, dtype=torch.float32: None if t is None else _plain(what, t, dtype, n)
    targets, entropy, by_logprob, by_entropy = row(targets, torch.int32), row(entropy), row(grad_logprobs), row(grad_entropy)
    norms = _plain(what, norms, torch.float32, n, 2)
    grad = _grad_like(what, x, out)
    _check(lib().ivfpq_token_logprobs_backward(*_logits(x), _dp(targets), temperature, _dp(norms), _dp(entropy), _dp(by_logprob),
                                               _dp(by_entropy), _dp(grad), grad.stride(0), _stream()))
    return grad


def ivfpq_distill_topk(logits: torch.Tensor, teacher_tokens: torch.Tensor, teacher_logits: torch.Tensor, temperature: float = 1.0):
    """-> (loss fp32 [n], norms [n][2]): divergence of the rows' distributions from a teacher's listed tokens."""
    what = "ivfpq_distill_topk"
    _on_device(what, logits, teacher_tokens, teacher_logits)
    x = _value_rows(what, logits)
    n, vocab = x.shape
    tokens, values = _listed(what, teacher_tokens, teacher_logits, n)
    loss = torch.empty(n, dtype=torch.float32, device="cuda")
    norms = torch.empty((n, 2), dtype=torch.float32, device="cuda")
    need = lib().ivfpq_distill_topk_workspace_bytes(n, vocab)
    ws = _scratch(need)
    _check(lib().ivfpq_distill_topk(*_logits(x), _dp(tokens), _dp(values), tokens.shape[1], temperature, _dp(loss), _dp(norms), _dp(ws),
                                    need, _stream()))
    return loss, norms


def ivfpq_distill_topk_backward(logits: torch.Tensor, norms: torch.Tensor, teacher_tokens: torch.Tensor, teacher_logits: torch.Tensor,
                                row_grads: Optional[torch.Tensor] = None, temperature: float = 1.0,
                                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """-> the gradient of sum(row_grads * loss) with respect to the logits (written to `out`, which may be the logits themselves)."""
    what = "ivfpq_distill_topk_backward"
    _on_device(what, logits, norms, teacher_tokens, teacher_logits, row_grads)
    x = _value_rows(what, logits)
    n = x.shape[0]
    tokens, values = _listed(what, teacher_tokens, teacher_logits, n)
    norms = _plain(what, norms, torch.float32, n, 2)
    row_grads = None if row_grads is None else _plain(what, row_grads, torch.float32, n)
    grad = _grad_like(what, x, out)
    _check(lib().ivfpq_distill_topk_backward(*_logits(x), _dp(norms), _dp(tokens), _dp(values), tokens.shape[1], temperature, _dp(row_grads),
                                             _dp(grad), grad.stride(0), _stream()))
    return grad


def ivfpq_distill_topk_step(logits: torch.Tensor, teacher_tokens: torch.Tensor, teacher_logits: torch.Tensor,
                            row_grads: Optional[torch.Tensor] = None, temperature: float = 1.0, out: Optional[torch.Tensor] = None):
    """-> (loss [n], gradient): ivfpq_distill_topk and its backward call in one."""
    what = "ivfpq_distill_topk_step"
    _on_device(what, logits, teacher_tokens, teacher_logits, row_grads)
    x = _value_rows(what, logits)
    n, vocab = x.shape
    tokens, values = _listed(what, teacher_tokens, teacher_logits, n)
    row_grads = None if row_grads is None else _plain(what, row_grads, torch.float32, n)
    grad = _grad_like(what, x, out)
    loss = torch.empty(n, dtype=torch.float32, device="cuda")
    need = lib().ivfpq_distill_topk_workspace_bytes(n, vocab)
    ws = _scratch(need)
    _check(lib().ivfpq_distill_topk_step(*_logits(x), _dp(tokens), _dp(values), tokens.shape[1], temperature, _dp(row_grads), _dp(loss),
                                         _dp(grad), grad.stride(0), _dp(ws), need, _stream()))
    return loss, grad


# ---- drafted tokens.  n sequences of m rows a pass: row 0 the last token that was kept, the others drafts.

class DraftTrees(NamedTuple):
    tokens: torch.Tensor       # [n][m] int32; -1 behind a tree's rows
    parents: torch.Tensor      # [n][m] int32: the row that each row follows; -1 for row 0
    depths: torch.Tensor       # [n][m] int32: tokens since row 0
    logprobs: torch.Tensor     # [n][m] fp32: of the way to a row, among the neighbours
    counts: torch.Tensor       # [n] int32: rows of each tree


class Verified(NamedTuple):
    path: torch.Tensor         # [n][m] int32: the kept rows, then -1
    kept: torch.Tensor         # [n] int32: how many
    next_tokens: torch.Tensor  # [n] int32: the token behind the last kept row
    logprobs: torch.Tensor     # [n][m] fp32: of the token behind each kept row


def _optional(what: str, t: Optional[torch.Tensor], dtype, *shape):
    return None if t is None else _plain(what, t, dtype, *shape)


def _cache(what: str, k_cache: torch.Tensor, v_cache: torch.Tensor, pages: torch.Tensor, lens: torch.Tensor, layers: bool = False):
    """-> (layers, the arguments that describe a cache's layout, n, page, tensors that the call reads): caches are written or read in place, so they have to
    be contiguous."""
    if k_cache.dim() != 4 + layers or k_cache.dtype not in (torch.float16, torch.bfloat16):
        _refuse(f"{what}: keys are float16 or bfloat16 {'[layers]' if layers else ''}[pages][heads][page][d], got {k_cache.dtype} {tuple(k_cache.shape)}")
    *more, n_pages, kv_heads, page, d = k_cache.shape
    if v_cache.dtype != k_cache.dtype or v_cache.shape != (*more, n_pages, kv_heads, page // 8, d, 8):
        _refuse(f"{what}: values are {k_cache.dtype} {(*more, n_pages, kv_heads, page // 8, d, 8)}, got {v_cache.dtype} {tuple(v_cache.shape)}")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()):
        _refuse(f"{what}: a cache is not contiguous")
    if pages.dim() != 2 or lens.dim() != 1:
        _refuse(f"{what}: pages are a matrix, lengths a vector")
    n, most = pages.shape
    for size in (kv_heads, page, d, most, *more):
        _fits_int32(what, size)
    pages, lens = _plain(what, pages, torch.int32, n, most), _plain(what, lens, torch.int32, n)
    return (more[0] if layers else 1), (n_pages, kv_heads, page, d, _dp(pages), most, _dp(lens)), n, page, (pages, lens)


def _head_rows(what: str, x: torch.Tensor, n: int, d: int, align: int = 1):
    """-> (x, row stride): [n][m][heads][d] whose heads lie behind each other and whose rows lie a stride apart; other layouts are copied."""
    if x.dim() != 4 or x.shape[0] != n or x.shape[3] != d:
        _refuse(f"{what}: rows are [{n}][m][heads][{d}], got {tuple(x.shape)}")
    _, m, heads, _ = x.shape
    _fits_int32(what, m)
    _fits_int32(what, heads)
    if x.numel() == 0 or x.is_contiguous():
        return x, heads * d
    sn, sm, sh, sd = x.stride()
    stride = sm if m > 1 else sn
    fits = (sd == 1 or d == 1) and (sh == d or heads == 1) and (n == 1 or sn == m * stride) and stride >= heads * d and stride % align == 0
    return (x, stride) if fits else (x.contiguous(), heads * d)


def ivfpq_neighbour_drafts(ids: torch.Tensor, dists: torch.Tensor, text: torch.Tensor, last_tokens: torch.Tensor, temperature: float, depth: int = 8,
                           rows: int = MAX_DRAFT) -> DraftTrees:
    """Trees of `rows` rows from search results: text [n_ids] int32 is the token that followed each stored state, states in the order of their text."""
    what = "ivfpq_neighbour_drafts"
    _on_device(what, ids, dists, text, last_tokens)
    if ids.dim() != 2:
        _refuse(f"{what}: ids are a matrix")
    nq, k = ids.shape
    _fits_int32(what, k)
    if not 1 <= depth <= MAX_DRAFT_DEPTH:
        _refuse(f"{what}: depth={depth} outside [1, {MAX_DRAFT_DEPTH}]")
    if not 1 <= rows <= MAX_DRAFT:
        _refuse(f"{what}: rows={rows} outside [1, {MAX_DRAFT}]")
    ids, dists = _plain(what, ids, torch.int64, nq, k), _plain(what, dists, torch.float32, nq, k)
    text, last = _plain(what, text, torch.int32, text.numel()), _plain(what, last_tokens, torch.int32, nq)
    three = torch.empty((3, nq, rows), dtype=torch.int32, device="cuda")
    tokens, parents, depths = three[0], three[1], three[2]
    logprobs = torch.empty((nq, rows), dtype=torch.float32, device="cuda")
    counts = torch.empty(nq, dtype=torch.int32, device="cuda")
    _check(lib().ivfpq_neighbour_drafts(_dp(ids), _dp(dists), nq, k, _dp(text), text.numel(), _dp(last), temperature, depth, rows, _dp(tokens), _dp(parents),
                                        _dp(depths), _dp(logprobs), _dp(counts), _stream()))
    return DraftTrees(tokens, parents, depths, logprobs, counts)


def ivfpq_cache_append(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, pages: torch.Tensor, lens: torch.Tensor,
                       q: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None, depths: Optional[torch.Tensor] = None,
                       counts: Optional[torch.Tensor] = None, interleaved: bool = False, amplitude: float = 1.0) -> Optional[torch.Tensor]:
    """Keys and values [n][m][heads][d] to their places, keys turned by their positions; -> the queries turned alike (None without q).  inv_freq [rotated / 2] fp32."""
    what = "ivfpq_cache_append"
    _on_device(what, k, v, k_cache, v_cache, pages, lens, q, inv_freq, depths, counts)
    _, layout, n, _, held = _cache(what, k_cache, v_cache, pages, lens)
    kv_heads, d = k_cache.shape[1], k_cache.shape[3]
    if k.dtype not in VALUES_DTYPES or v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
        _refuse(f"{what}: rows of {k.dtype} and {v.dtype}")
    k, k_stride = _head_rows(what, k, n, d)
    v, v_stride = _head_rows(what, v, n, d)
    m = k.shape[1]
    if k.shape != v.shape or k.shape[2] != kv_heads:
        _refuse(f"{what}: keys {tuple(k.shape)} and values {tuple(v.shape)} for a cache of {kv_heads} heads")
    heads, q_stride, turned = 0, 0, None
    if q is not None:
        q, q_stride = _head_rows(what, q, n, d)
        if q.shape[1] != m or q.shape[2] < 1:
            _refuse(f"{what}: queries {tuple(q.shape)} for {m} rows")
        heads = q.shape[2]
        turned = torch.empty(q.shape, dtype=k_cache.dtype, device="cuda")
    half = 0 if inv_freq is None else inv_freq.numel()
    _fits_int32(what, 2 * half)
    inv_freq = _optional(what, inv_freq, torch.float32, half)
    depths, counts = _optional(what, depths, torch.int32, n, m), _optional(what, counts, torch.int32, n)
    _check(lib().ivfpq_cache_append(_dp(q), q_stride, heads, _dp(k), k_stride, _dp(v), v_stride, VALUES_DTYPES[k.dtype], n, m, _dp(depths), _dp(counts),
                                    _dp(inv_freq), 2 * half, int(interleaved), amplitude, _dp(turned), _dp(k_cache), _dp(v_cache),
                                    VALUES_DTYPES[k_cache.dtype], *layout, _stream()))
    return turned


def ivfpq_draft_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, pages: torch.Tensor, lens: torch.Tensor,
                          parents: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                          max_places: Optional[int] = None, out: Optional[torch.Tensor] = None, with_lse: bool = False):
    """-> [n][m][heads][d] (with_lse: and lse [n][m][heads] fp32): attention of a pass's rows over the cache, whose last m places hold theirs.
    scale: d ** -0.5 if None.  max_places: about how many places the longest sequence has with its rows (as many as `pages` has if None); it
    decides how the work is divided, not what is seen."""
    what = "ivfpq_draft_attention"
    _on_device(what, q, k_cache, v_cache, pages, lens, parents, counts, out)
    _, layout, n, page, held = _cache(what, k_cache, v_cache, pages, lens)
    kv_heads, d = k_cache.shape[1], k_cache.shape[3]
    if q.dtype != k_cache.dtype:
        _refuse(f"{what}: queries of {q.dtype} over a cache of {k_cache.dtype}")
    q, q_stride = _head_rows(what, q, n, d, 8)
    if q.data_ptr() % 16:
        q, q_stride = q.clone(memory_format=torch.contiguous_format), q.shape[2] * d
    m, heads = q.shape[1], q.shape[2]
    if m < 1 or heads < 1:
        _refuse(f"{what}: queries {tuple(q.shape)}")
    parents, counts = _optional(what, parents, torch.int32, n, m), _optional(what, counts, torch.int32, n)
    if out is None:
        out = torch.empty((n, m, heads, d), dtype=q.dtype, device="cuda")
    if out.shape != (n, m, heads, d) or out.dtype != q.dtype or not out.is_contiguous():
        _refuse(f"{what}: out has another shape, type or layout than the queries")
    lse = torch.empty((n, m, heads), dtype=torch.float32, device="cuda") if with_lse else None
    if max_places is None:
        max_places = pages.shape[1] * page
    if not 0 <= max_places < 2 ** 62:
        _refuse(f"{what}: max_places={max_places}")
    need = lib().ivfpq_draft_attention_workspace_bytes(n, m, heads, kv_heads, d, max_places)
    ws = _scratch(need)
    _check(lib().ivfpq_draft_attention(_dp(q), q_stride, heads, n, m, _dp(parents), _dp(counts), _dp(k_cache), _dp(v_cache), VALUES_DTYPES[q.dtype], *layout,
                                       max_places, d ** -0.5 if scale is None else scale, _dp(out), heads * d, _dp(lse), _dp(ws), need, _stream()))
    return (out, lse) if with_lse else out


def ivfpq_verify_drafts(logits: torch.Tensor, tokens: torch.Tensor, parents: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
                        uniforms: Optional[torch.Tensor] = None, temperature: float = 1.0, draft_logits: Optional[torch.Tensor] = None,
                        accept: Optional[torch.Tensor] = None) -> Verified:
    """Which rows of tokens [n][m] the model's logits [n * m][vocab] keep, and the token behind them.  uniforms [n][m]: where in its distribution each row's
    token is (None: the most likely one).  draft_logits [n * (m - 1)][vocab] and accept [n][m]: for drafts that were drawn from a student's distribution."""
    what = "ivfpq_verify_drafts"
    _on_device(what, logits, tokens, parents, counts, uniforms, draft_logits, accept)
    x = _value_rows(what, logits)
    if tokens.dim() != 2:
        _refuse(f"{what}: tokens are a matrix")
    n, m = tokens.shape
    _fits_int32(what, m)
    if x.shape[0] != n * m:
        _refuse(f"{what}: {x.shape[0]} rows of logits for {n} x {m} tokens")
    tokens, parents, counts = _plain(what, tokens, torch.int32, n, m), _optional(what, parents, torch.int32, n, m), _optional(what, counts, torch.int32, n)
    uniforms, accept = _optional(what, uniforms, torch.float32, n, m), _optional(what, accept, torch.float32, n, m)
    if draft_logits is not None:
        drafts = _value_rows(what, draft_logits)
        if drafts.shape != (n * (m - 1), x.shape[1]) or drafts.dtype != x.dtype:
            _refuse(f"{what}: draft logits {drafts.dtype} {tuple(drafts.shape)} for {n} x {m} tokens")
        if uniforms is None or accept is None:
            _refuse(f"{what}: drafts that were drawn need both random numbers")
        if m <= 1:
            draft_logits = None                            # nothing was drafted
    if draft_logits is None:
        drafts = None
    path = torch.empty((n, m), dtype=torch.int32, device="cuda")
    logprobs = torch.empty((n, m), dtype=torch.float32, device="cuda")
    kept, following = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    need = lib().ivfpq_verify_drafts_workspace_bytes(n, m, x.shape[1], drafts is not None)
    ws = _scratch(need)
    _check(lib().ivfpq_verify_drafts(_dp(x), VALUES_DTYPES[x.dtype], n, m, x.shape[1], x.stride(0), _dp(tokens), _dp(parents), _dp(counts), _dp(uniforms),
                                     temperature, _dp(drafts), 0 if drafts is None else drafts.stride(0), _dp(accept), _dp(path), _dp(kept),
                                     _dp(following), _dp(logprobs), _dp(ws), need, _stream()))
    return Verified(path, kept, following, logprobs)


def ivfpq_cache_keep(k_cache: torch.Tensor, v_cache: torch.Tensor, pages: torch.Tensor, lens: torch.Tensor, path: torch.Tensor, kept: torch.Tensor):
    """The kept rows (path, kept of Verified) move up behind each other in the caches [layers][pages][heads][page][d] (values [layers][pages][heads][page / 8][d][8];
    one layer's without the first dimension); raise `lens` by `kept` afterwards."""
    what = "ivfpq_cache_keep"
    _on_device(what, k_cache, v_cache, pages, lens, path, kept)
    layers, layout, n, _, held = _cache(what, k_cache, v_cache, pages, lens, layers=k_cache.dim() == 5)
    if path.dim() != 2:
        _refuse(f"{what}: paths are a matrix")
    m = path.shape[1]
    _fits_int32(what, m)
    path, kept = _plain(what, path, torch.int32, n, m), _plain(what, kept, torch.int32, n)
    _check(lib().ivfpq_cache_keep(_dp(k_cache), _dp(v_cache), VALUES_DTYPES[k_cache.dtype], layers, *layout, n, m, _dp(path), _dp(kept), _stream()))


class Index:
    """Owns one ivfpq_index_t handle plus the torch tensors that back its device image and scratch."""

    def __init__(self, handle: ctypes.c_void_p):
        self._h = handle
        self._image: Optional[torch.Tensor] = None
        self._ws: Optional[torch.Tensor] = None
        n, d, nl, s, p = ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
        _check(lib().ivfpq_index_info(self._h, n, d, nl, s, p))
        self.n, self.d, self.n_lists, self.pq_dim, self.pq_bits = n.value, d.value, nl.value, s.value, p.value

    # ---- construction
    @staticmethod
    def ivfpq_build_host(data, n_lists: int, pq_dim: int, pq_bits: int, kmeans_iters: int = 10, seed: int = 0) -> "Index":
        data = _np(data, np.float32)
        h = ctypes.c_void_p()
        _check(lib().ivfpq_build_host(_hp(data), data.shape[0], data.shape[1], n_lists, pq_dim, pq_bits,
                                      kmeans_iters, seed, ctypes.byref(h)))
        return Index(h)

    @staticmethod
    def ivfpq_build_device(data, n_lists: int, pq_dim: int, pq_bits: int, kmeans_iters: int = 10, seed: int = 0,
                           coarse_train_rows=None, coarse_init_rows=None, pq_train_rows=None,
                           pq_init_rows=None) -> "Index":
        """data: a CUDA tensor or a numpy array (copied to the device) [n][d] fp32."""
        x = _dev_f32(data)
        n, d = int(x.shape[0]), int(x.shape[1])
        opt = lambda a: None if a is None else _np(a, np.int64)
        ctr, cir, ptr, pir = opt(coarse_train_rows), opt(coarse_init_rows), opt(pq_train_rows), opt(pq_init_rows)
        n_ct = 0 if ctr is None else int(ctr.size)
        n_pt = 0 if ptr is None else int(ptr.size)
        if cir is not None:
            assert cir.size == n_lists
        if pir is not None:
            assert pir.size == pq_dim * (1 << pq_bits)
        need = lib().ivfpq_build_device_workspace_bytes(n, d, n_lists, pq_dim, pq_bits, n_ct, n_pt)
        if need == 0:
            raise IvfpqError(EINVAL, lib().ivfpq_last_error().decode("utf-8", "replace"))
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        h = ctypes.c_void_p()
        hp = lambda a: None if a is None else _hp(a)
        _check(lib().ivfpq_build_device(_dp(x), n, d, n_lists, pq_dim, pq_bits, kmeans_iters, hp(ctr), n_ct, hp(cir),
                                        hp(ptr), n_pt, hp(pir), seed, _dp(ws), need, _stream(), ctypes.byref(h)))
        del ws
        return Index(h)

    @staticmethod
    def ivfpq_index_from_arrays(d: int, n_lists: int, pq_dim: int, pq_bits: int, centroids, codebooks,
                                list_offsets, codes, ids) -> "Index":
        centroids, codebooks = _np(centroids, np.float32), _np(codebooks, np.float32)
        list_offsets, codes, ids = _np(list_offsets, np.int64), _np(codes, np.uint8), _np(ids, np.int64)
        ksub, m, cb = 1 << pq_bits, d // max(pq_dim, 1), pq_dim * pq_bits // 8
        n = int(ids.shape[0])
        assert centroids.size == n_lists * d and codebooks.size == pq_dim * ksub * m
        assert list_offsets.size == n_lists + 1 and codes.size == n * cb
        h = ctypes.c_void_p()
        _check(lib().ivfpq_index_from_arrays(n, d, n_lists, pq_dim, pq_bits, _hp(centroids), _hp(codebooks),
                                             _hp(list_offsets), _hp(codes), _hp(ids), ctypes.byref(h)))
        return Index(h)

    def ivfpq_index_export(self):
        ksub, m, cb = 1 << self.pq_bits, self.d // self.pq_dim, self.pq_dim * self.pq_bits // 8
        centroids = np.empty((self.n_lists, self.d), np.float32)
        codebooks = np.empty((self.pq_dim, ksub, m), np.float32)
        list_offsets = np.empty(self.n_lists + 1, np.int64)
        codes = np.empty((self.n, cb), np.uint8)
        ids = np.empty(self.n, np.int64)
        _check(lib().ivfpq_index_export(self._h, _hp(centroids), _hp(codebooks), _hp(list_offsets), _hp(codes), _hp(ids)))
        return centroids, codebooks, list_offsets, codes, ids

    def ivfpq_set_fp8_encoding(self, lut_dtype: int, bias: int, rounding: int = ROUND_NEAREST, per_table_bias: bool = False):
        _check(lib().ivfpq_set_fp8_encoding(self._h, int(lut_dtype), int(bias), int(rounding), int(per_table_bias)))

    def ivfpq_set_workspace_limit(self, nbytes: int):
        _check(lib().ivfpq_set_workspace_limit(self._h, int(nbytes)))
        self._ws = None

    def ivfpq_set_tuning(self, knob: int, value: int):
        _check(lib().ivfpq_set_tuning(self._h, int(knob), int(value)))

    def ivfpq_set_e4m4_bias(self, bias: int):
        _check(lib().ivfpq_set_e4m4_bias(self._h, int(bias)))

    def ivfpq_free(self):
        if self._h:
            lib().ivfpq_free(self._h)
            self._h = None
            self._image = None
            self._ws = None

    def __del__(self):
        try:
            self.ivfpq_free()
        except Exception:
            pass

    # ---- device residency
    def ivfpq_device_bytes(self) -> int:
        return int(lib().ivfpq_device_bytes(self._h))

    def ivfpq_upload(self) -> "Index":
        nbytes = self.ivfpq_device_bytes()
        self._image = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        _check(lib().ivfpq_upload(self._h, _dp(self._image), nbytes, _stream()))
        return self

    def ivfpq_search_workspace_bytes(self, nq: int, n_probes: int, k: int, lut_dtype: int) -> int:
        return int(lib().ivfpq_search_workspace_bytes(self._h, nq, n_probes, k, lut_dtype))

    def _workspace(self, nq, n_probes, k, lut_dtype) -> torch.Tensor:
        need = self.ivfpq_search_workspace_bytes(nq, n_probes, k, lut_dtype)
        if self._ws is None or self._ws.numel() < need:
            self._ws = None
            self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        return self._ws

    # ---- search
    def ivfpq_search(self, queries, n_probes: int, k: int, lut_dtype: int = LUT_FP8_E5M3, out=None):
        q = _dev_f32(queries)
        nq = q.shape[0]
        ids, dists = out if out is not None else (
            torch.empty((nq, k), dtype=torch.int64, device="cuda"),
            torch.empty((nq, k), dtype=torch.float32, device="cuda"))
        ws = self._workspace(nq, n_probes, k, lut_dtype)
        _check(lib().ivfpq_search(self._h, _dp(q), nq, n_probes, k, lut_dtype, _dp(ids), _dp(dists),
                                  _dp(ws), ws.numel(), _stream()))
        return ids, dists

    def ivfpq_search_static(self, queries, n_probes: int, k: int, lut_dtype: int = LUT_FP8_E5M3, out=None):
        """ivfpq_search on the library's fixed scratch: no workspace is allocated or passed."""
        q = _dev_f32(queries)
        nq = q.shape[0]
        ids, dists = out if out is not None else (
            torch.empty((nq, k), dtype=torch.int64, device="cuda"),
            torch.empty((nq, k), dtype=torch.float32, device="cuda"))
        _check(lib().ivfpq_search_static(self._h, _dp(q), nq, n_probes, k, lut_dtype, _dp(ids), _dp(dists), _stream()))
        return ids, dists

    def ivfpq_select_probes(self, queries, n_probes: int):
        q = _dev_f32(queries)
        nq = q.shape[0]
        probes = torch.empty((nq, n_probes), dtype=torch.int32, device="cuda")   # u32 payload
        pd = torch.empty((nq, n_probes), dtype=torch.float32, device="cuda")
        ws = self._workspace(nq, n_probes, 1, LUT_FP32)
        _check(lib().ivfpq_select_probes(self._h, _dp(q), nq, n_probes, _dp(probes), _dp(pd), _dp(ws),
                                         ws.numel(), _stream()))
        return probes, pd

    def ivfpq_search_with_probes(self, queries, probes, k: int, lut_dtype: int = LUT_FP8_E5M3):
        q = _dev_f32(queries)
        nq = q.shape[0]
        if not isinstance(probes, torch.Tensor):
            probes = torch.from_numpy(_np(probes, np.uint32).view(np.int32)).cuda()
        probes = probes.contiguous()
        assert probes.is_cuda and probes.dtype == torch.int32 and probes.shape[0] == nq
        n_probes = probes.shape[1]
        ids = torch.empty((nq, k), dtype=torch.int64, device="cuda")
        dists = torch.empty((nq, k), dtype=torch.float32, device="cuda")
        ws = self._workspace(nq, n_probes, k, lut_dtype)
        _check(lib().ivfpq_search_with_probes(self._h, _dp(q), nq, _dp(probes), n_probes, k, lut_dtype,
                                              _dp(ids), _dp(dists), _dp(ws), ws.numel(), _stream()))
        return ids, dists

    def ivfpq_dump_lut(self, query, list_id: int, lut_dtype: int) -> torch.Tensor:
        q = _dev_f32(query).reshape(-1)
        nbytes = self.pq_dim * (1 << self.pq_bits) * LUT_BYTES[lut_dtype]
        out = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        _check(lib().ivfpq_dump_lut(self._h, _dp(q), list_id, lut_dtype, _dp(out), _stream()))
        return out

    def ivfpq_scan_list(self, query, list_id: int, lut_dtype: int, list_len: int) -> torch.Tensor:
        q = _dev_f32(query).reshape(-1)
        out = torch.empty(max(list_len, 1), dtype=torch.float32, device="cuda")
        _check(lib().ivfpq_scan_list(self._h, _dp(q), list_id, lut_dtype, _dp(out), _stream()))
        return out[:list_len]

    # ---- measurement aid
    def ivfpq_set_stage_timing(self, enabled: bool):
        _check(lib().ivfpq_set_stage_timing(self._h, int(enabled)))

    def ivfpq_scan_kernel_info(self, lut_dtype: int) -> str:
        buf = ctypes.create_string_buffer(256)
        _check(lib().ivfpq_scan_kernel_info(self._h, int(lut_dtype), buf, 256))
        return buf.value.decode()

    def ivfpq_stage_times_ms(self):
        ms = (ctypes.c_float * 8)()
        _check(lib().ivfpq_stage_times_ms(self._h, ctypes.byref(ms)))
        return {"probe_select": ms[0], "scan": ms[1], "topk": ms[2], "total": ms[3],
                "rank_gemm": ms[4], "scan_nearest_kernel": ms[5], "scan_filtered_kernel": ms[6]}
