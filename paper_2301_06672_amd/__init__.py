"""MI355X-native IVFPQ search (arXiv 2301.06672): thin Python binding over libivfpq.so."""
from .binding import (  # noqa: F401
    Index, IvfpqError, lib, EXPORTS, LIB_PATH, ivfpq_assign_device, ivfpq_refine, ivfpq_stream_read,
    TokenLogprobs, ivfpq_quantize_rows, ivfpq_q8_matmul, ivfpq_neighbour_tokens, ivfpq_token_logprobs,
    ivfpq_token_logprobs_backward, ivfpq_distill_topk, ivfpq_distill_topk_backward, ivfpq_distill_topk_step,
    DraftTrees, Verified, ivfpq_neighbour_drafts, ivfpq_cache_append, ivfpq_draft_attention, ivfpq_verify_drafts, ivfpq_cache_keep,
    MAX_DRAFT, MAX_DRAFT_DEPTH, MAX_HEAD, MAX_TOP, MAX_LISTED, MAX_MIXED, MAX_Q8_K, VALUES_DTYPES,
    LUT_FP32, LUT_FP16, LUT_FP8_E5M3, LUT_FP8_E4M4, LUT_NAMES, LUT_BYTES, MAX_K, MAX_PROBES,
    ROUND_NEAREST, ROUND_TRUNCATE, STATIC_SCRATCH_BYTES,
    TUNE_SCAN_THREADS, TUNE_ORDER_BLOCK, TUNE_SCAN_SHARE, TUNE_EARLY_EXIT, TUNE_LDS_PAD, TUNE_SCAN_ROUTE,
    OK, EINVAL, ENOSPACE, EHIP, EUNSUPPORTED, ESTATE,
)
