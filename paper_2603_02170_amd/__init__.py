"""SageBwd hot path for MI355X (gfx950): fused INT8 attention forward and
backward behind a C-ABI library, with a thin binding, and serving from a paged
4-bit key/value cache (cache.py)."""
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
    CacheParams,
    CachePlan,
    alloc_cache,
    cache_page_bytes,
    cache_workspace_bytes,
    sagebwd_cache_append,
    sagebwd_cache_attention,
    sagebwd_cache_plan,
    sagebwd_cache_read,
    sagebwd_cache_trim,
)
