"""MI355X (gfx950) dynamic sparse prefill attention: Python binding of the C ABI in include/sa.h."""
from .binding import (  # noqa: F401
    SA_BLOCK_CLUSTER, SA_CACHE_E4M3, SA_CACHE_E5M2, SA_INTERVAL_SLASH, SA_PATTERN_AUTO, SA_ROTARY_HALF,
    SA_ROTARY_INTERLEAVED, SA_SCALING_BASE, SA_SCALING_LINEAR, SA_SCALING_NONE, SA_SCALING_RAMP, SA_SCALING_WAVELENGTH,
    SA_TRIANGULAR, Cache, Rotary, SaCache, SaConfig, SaError, SaIndex, SaRotaryConfig, SaRows, SaScores, Session, library,
    sa_build_index, sa_cache_append, sa_cache_attend, sa_cache_attend_plan, sa_cache_attend_scratch_bytes, sa_cache_bytes, sa_cache_decode, sa_create,
    sa_default_budgets, sa_destroy, sa_estimate_and_index, sa_estimate_patterns, sa_index_bytes, sa_last_error,
    sa_rotary_create, sa_rotary_destroy, sa_rotary_embed,
    sa_scores_bytes, sa_search_patterns, sa_search_scratch_bytes, sa_set_workspace, sa_sparse_decode, sa_sparse_decode_static, sa_sparse_prefill,
    sa_sparse_prefill_counted, sa_version, sa_workspace_bytes,
)
