"""CMC two-tier KV-cache decode path for GB300 (sm_103a).

Question-guided top-K selection of Context Memory Embeddings (Tier-1), a
local-window ring (Tier-2) and GQA decode attention over [Tier-1 | Tier-2],
as hand-written CUDA kernels behind the C ABI of include/cmc.h.
"""

from .cmc import (  # noqa: F401
    CmcDims,
    DecodeWorkspace,
    DEVFLAG_BAD_INDEX,
    DEVFLAG_BAD_POS,
    DEVFLAG_TIMEOUT,
    bridge_epilogue,
    decode_attn_plan,
    decode_attn_q8_plan,
    decode_attn_q8_workspace_size,
    decode_q8_status,
    decode_attn_workspace_size,
    decode_step,
    decode_attn_weighted_plan,
    decode_attn_weighted_workspace_size,
    decode_step_q8,
    decode_step_weighted,
    denoise,
    dequantize_cache,
    dims_of,
    evict_cache,
    q8_scale_bytes,
    qk_norm_rope,
    quantize_cache,
    question_select,
    score_select,
    score_select_workspace_size,
    set_l2_prefetch_tiles,
    stage_copies,
    tier1_gather,
    two_tier_decode_attn,
    two_tier_decode_attn_q8,
    two_tier_decode_attn_weighted,
    weighted_cache_status,
    window_append,
    window_append_q8,
    window_prefill,
)
from ._lib import CmcError, EXPORTS, LIB_PATH, lib  # noqa: F401
