"""L2A token-wise conditional attention for MI355X (gfx950): hand-written HIP kernels behind a
C-ABI library (l2a_route_compact, l2a_attn_fwd, l2a_attn_bwd; for serving l2a_router_decide, l2a_attn_decode and, on a paged KV
cache, l2a_cache_write, l2a_cache_read, l2a_attn_extend; for long generations l2a_cache_weights, l2a_cache_evict, and l2a_rope) and a
thin ctypes binding."""
