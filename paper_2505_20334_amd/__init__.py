"""MI355X-native hot path of Lookahead Q-Cache (LAQ) re-eviction (paper Sec. 4.3, Eq. 4).

The work is done by hand-written HIP kernels behind the C ABI declared in
``include/laq.h``, ``laq_fp4.h`` and ``laq_cache.h``; this package only marshals arguments (``binding``, ``fp4``, ``paged``) and knows how
to compile the library (``_build``).  There is no CPU fallback: if the shared
library is missing the first call builds it with hipcc, and raises if that fails.
"""
from .binding import (LaqError, laq_compact, laq_init, laq_workspace_status, laq_score_kernel, laq_decode_attention, laq_decode_workspace_bytes, laq_evict, laq_qcache_store, laq_recall, laq_score, laq_select,  # noqa: F401
                      laq_select_sink_recent, laq_strerror, laq_workspace_bytes, lib_path, load_library, packed_rows)
from .fp4 import (Fp4Cache, laq_block_map, laq_block_pool, laq_fp4_attention, laq_fp4_attention_workspace_bytes, laq_fp4_cache,  # noqa: F401
                  laq_fp4_compact, laq_fp4_load, laq_fp4_store)
from .paged import (PagedCache, Rope, laq_cache, laq_cache_append, laq_cache_attention, laq_cache_attention_workspace_bytes, laq_cache_compact,  # noqa: F401
                    laq_cache_load, laq_rope, laq_rope_frequencies)

__all__ = ["LaqError", "laq_compact", "laq_init", "laq_workspace_status", "laq_score_kernel", "laq_decode_attention", "laq_decode_workspace_bytes", "laq_evict", "laq_qcache_store", "laq_recall", "laq_score", "laq_select", "laq_select_sink_recent", "laq_strerror",
           "laq_workspace_bytes", "lib_path", "load_library", "packed_rows", "Fp4Cache", "laq_block_map", "laq_block_pool", "laq_fp4_attention",
           "laq_fp4_attention_workspace_bytes", "laq_fp4_cache", "laq_fp4_compact", "laq_fp4_load", "laq_fp4_store",
           "PagedCache", "Rope", "laq_cache", "laq_cache_append", "laq_cache_attention", "laq_cache_attention_workspace_bytes", "laq_cache_compact",
           "laq_cache_load", "laq_rope", "laq_rope_frequencies"]
