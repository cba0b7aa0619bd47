"""SageBwd hot path for MI355X (gfx950): fused INT8 attention forward and
backward behind a C-ABI library, with a thin binding, and serving from a paged
key/value cache held in 4 or 8 bits (cache.py)."""
from .binding import (  # noqa: F401
    SageParams,
    lib_path,
    load_library,
    workspace_bytes,
    sagebwd_quantize,
    sagebwd_fwd,
    sagebwd_bwd,
    sagebwd_strerror,
)
from .cache import (  # noqa: F401
    CacheCompaction,
    CacheParams,
    CachePlan,
    alloc_cache,
    alloc_shares,
    cache_page_bytes,
    cache_workspace_bytes,
    sagebwd_cache_append,
    sagebwd_cache_attention,
    sagebwd_cache_compact,
    sagebwd_cache_fork,
    sagebwd_cache_free,
    sagebwd_cache_own,
    sagebwd_cache_plan,
    sagebwd_cache_read,
    sagebwd_cache_trim,
)
